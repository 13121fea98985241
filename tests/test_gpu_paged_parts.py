"""PagedAttention over long contexts, split into parts that are put together: parts of sequences with few new rows beside those of
chunks, numbered by rows or by sequences."""
import numpy as np
import pytest

from attention_cases import paged_bounds, paged_feeds, paged_graph, within
from lm_cases import run_gpu
from oracle import interp

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads,kv,width,page,window,new,lengths,first", [
    (8, 2, 64, 16, 0, [1, 300, 2, 0, 1], [3000, 2000, 2500, 40, 700], 0),       # both kinds of part
    (8, 2, 128, 32, 0, [1, 1, 1, 1], [3000, 2000, 2500, 700], 0),               # single rows only
    (8, 2, 128, 32, 0, [1, 2, 1, 3], [3000, 2000, 2500, 700], 3),               # some rows of no sequence in front
    (32, 32, 32, 16, 0, [1, 1200, 2], [2000, 1300, 900], 0),                    # tiles in one part: only rows of few are put together
    (40, 2, 64, 64, 0, [1, 90, 1], [1500, 1200, 40], 2),                        # 20 heads of a group
    (6, 2, 72, 16, 900, [5, 1, 70], [2600, 1, 1900], 0),                        # a window, 3 heads of a group
    (33, 1, 64, 16, 0, [1, 3], [1200, 2000], 1),                                # more heads of a group than the kernel for few rows takes
])
@pytest.mark.parametrize("y", ["bf16", "f32"])
def test_parts_of_few_rows_beside_parts_of_chunks(heads, kv, width, page, window, new, lengths, first, y):
    starts = first + np.concatenate([[0], np.cumsum(new)])
    rows = int(starts[-1]) + 3
    most = max(-(-n // page) for n in lengths) + 2
    pool = sum(-(-n // page) for n in lengths) + 2
    g, ids, inputs, outputs = paged_graph(rows, len(new), heads, kv, width, page, most, pool, window, starts=True, write=False, y=y)
    feeds = paged_feeds(g, inputs, heads + width, lengths, page, pool, starts)
    got, f = run_gpu(g.desc, inputs, outputs, feeds)
    want = interp.run_function(g.desc, inputs, outputs, feeds)
    assert within(got[0], want[0], paged_bounds(g, inputs, outputs, feeds), y) <= 1
    assert (got[0][:first] == 0).all() and (got[0][-3:] == 0).all()
    again, _ = run_gpu(g.desc, inputs, outputs, feeds, f)
    assert np.array_equal(again[0], got[0])
