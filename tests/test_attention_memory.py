"""What the attention operators ask for as workspace, without a GPU."""
import pytest

from attention_cases import attention_graph, paged_graph
from paper_1707_08265_b200 import binding as B


def workspace(built):
    g, ids, inputs, outputs = built
    return B.Graph.from_desc(g.desc).function(inputs, outputs).workspace_bytes()


# rows, sequences, heads, kv heads, width, page, pages of the table
CHUNKS = [(8192, 1, 32, 8, 128, 64, 2048), (16384, 1, 64, 8, 128, 64, 2048), (8192, 2, 64, 8, 128, 64, 2048), (6000, 4, 8, 1, 128, 64, 2048), (4096, 1, 8, 1, 128, 64, 2048),
          (4500, 6, 16, 4, 128, 32, 297), (64, 64, 32, 8, 128, 16, 250), (3, 3, 16, 4, 64, 16, 13), (300000, 7, 4, 4, 64, 16, 70000)]


@pytest.mark.parametrize("rows,sequences,heads,kv,width,page,most", CHUNKS)
def test_parts_of_paged_attention_do_not_grow_with_the_rows(rows, sequences, heads, kv, width, page, most):
    """Keys are split over as many CTAs as the GPU holds at once, some 740 of 16 rows and heads or 440 of 32: with starts too, where any
    sequence may turn out to have few rows, and for tiles of up to 256 rows and heads, one an SM.  A part is width + 1 floats of each."""
    bound = (740 * 32 + 2 * 148 * 256) * (width + 1) * 4 + 4096
    assert workspace(paged_graph(rows, sequences, heads, kv, width, page, most, 8, starts=True, write=False)) <= bound


def test_single_new_rows_take_no_more_with_starts_than_without():
    """One new row each of 64 sequences: parts are numbered by rows where that is less than room for every sequence's most."""
    with_starts, without = (workspace(paged_graph(64, 64, 32, 8, 128, 16, 250, 8, starts=s, write=False)) for s in (True, False))
    assert with_starts <= without + 4096
