"""PagedAttention where counts pass 32 bits."""
import pytest

from attention_cases import paged_graph
from paper_1707_08265_b200 import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("starts", [False, True])
def test_new_rows_times_heads_beyond_32_bits(starts):
    """2^24 new rows of 128 heads that share one: 2^31 together (34 GB of queries, and of results).  Each row sees itself alone, so
    that its result is its value, bit by bit; the sequence's pages are all the same one."""
    import torch
    rows, heads, width, page = 2 ** 24, 128, 8, 2 ** 20
    if torch.cuda.mem_get_info()[0] < 80 * 2 ** 30:
        pytest.skip("needs 80 GB")
    g, ids, inputs, outputs = paged_graph(rows, 1, heads, 1, width, page, rows // page, 1, window=1, starts=starts, write=False)
    v = torch.randn(page, width, device="cuda").to(torch.bfloat16)
    table = [torch.zeros(1, rows // page, dtype=torch.int32, device="cuda"), torch.tensor([rows], dtype=torch.int32, device="cuda")]
    if starts:
        table.append(torch.tensor([0, rows], dtype=torch.int32, device="cuda"))
    q = torch.zeros(rows, heads * width, dtype=torch.bfloat16, device="cuda")
    y = torch.full_like(q, float("nan"))
    f = B.Graph.from_desc(g.desc).function(inputs, outputs)
    f.run_torch([q, torch.ones_like(v), v] + table, [y])
    assert f.status() == 0
    for part in y.split(page):
        assert torch.equal(part.view(page, heads, width), v[:, None].expand(page, heads, width))


def one_page_everywhere(new, length, window, pages):
    """A sequence of `length` tokens whose pages are all the same one of 2^20 rows, and a window."""
    import torch
    width, page = 8, 2 ** 20
    g, ids, inputs, outputs = paged_graph(new, 1, 2, 1, width, page, pages, 1, window=window, write=False, y="f32")
    k, v = (torch.randn(page, width, device="cuda").to(torch.bfloat16) for _ in range(2))
    q = torch.randn(new, 2 * width, device="cuda").to(torch.bfloat16)
    y = torch.full((new, 2 * width), float("nan"), device="cuda")
    f = B.Graph.from_desc(g.desc).function(inputs, outputs)
    f.run_torch([q, k, v, torch.zeros(1, pages, dtype=torch.int32, device="cuda"), torch.tensor([length], dtype=torch.int32, device="cuda")], [y])
    return f, q.double().view(new, 2, width), k.double(), v.double(), y.double().view(new, 2, width)


@pytest.mark.parametrize("new", [1, 40])
@pytest.mark.parametrize("length", [2 ** 31 - 256, 2 ** 31 - 300, 2 ** 30 + 7])
def test_the_longest_sequences(new, length):
    import torch
    window, page = 70, 2 ** 20
    f, q, k, v, y = one_page_everywhere(new, length, window, 2048)
    assert f.status() == 0
    at = (torch.arange(length - new, length, device="cuda")[:, None] - torch.arange(window, device="cuda")) % page
    s = torch.einsum("rhd,rjd->rhj", q, k[at]) / 8 ** 0.5
    p = torch.softmax(s, -1)
    want, size = torch.einsum("rhj,rjd->rhd", p, v[at]), torch.einsum("rhj,rjd->rhd", p, v[at].abs())
    # probabilities to bf16 (2^-8 of each), and fp32 sums of 8 and of 70 products with what they are made of: 2^-8 once more covers them
    assert bool(((y - want).abs() <= 2 * 2.0 ** -8 * size).all())


@pytest.mark.parametrize("new", [1, 40])
@pytest.mark.parametrize("length", [2 ** 31 - 1, 2 ** 31 - 255])
def test_longer_ones_are_reported(new, length):
    import torch
    f, q, k, v, y = one_page_everywhere(new, length, 70, 2048)
    assert f.status() == B.ERR_INVALID_ARG and bool(torch.isfinite(y).all())
