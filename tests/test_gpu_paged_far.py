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
