"""Attention where every score of a row is -inf: nothing is left of the row, and it gets 0."""
import numpy as np
import pytest

from attention_cases import attention_feeds, attention_graph, paged_feeds, paged_graph, within
from lm_cases import run_gpu
from oracle import interp

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,heads,kv,width,causal", [(300, 2, 1, 64, 1), (3001, 1, 1, 32, 1), (200, 3, 1, 72, 0), (1500, 2, 1, 128, 0)])
def test_rows_whose_scores_are_all_minus_infinity(rows, heads, kv, width, causal):
    g, ids, inputs, outputs = attention_graph(rows, heads, kv, width, causal)
    feeds = attention_feeds(g, inputs, rows)
    feeds[0], feeds[1][:] = np.abs(feeds[0]) + 1, -np.inf
    got, _ = run_gpu(g.desc, inputs, outputs, feeds)
    assert (got[0] == 0).all() and (interp.run_function(g.desc, inputs, outputs, feeds)[0] == 0).all()


def test_rows_of_which_some_scores_are_minus_infinity():
    """The first 140 keys give -inf: rows that see only them get 0, the others the softmax of the rest."""
    g, ids, inputs, outputs = attention_graph(300, 2, 1, 64)
    feeds = attention_feeds(g, inputs, 3)
    feeds[0] = np.abs(feeds[0]) + 1
    feeds[1][:140] = -np.inf
    got, _ = run_gpu(g.desc, inputs, outputs, feeds)
    want = interp.run_function(g.desc, inputs, outputs, feeds)
    assert (got[0][:140] == 0).all() and (want[0][:140] == 0).all()
    # the probabilities of a row add up to 1, and each is off by 2^-8 of itself (its rounding) and some 2^-12 (its score, a sum of 64
    # products of magnitude 200 together in fp32, and the exponential)
    assert within(got[0][140:], want[0][140:], 1.1 * 2.0 ** -8 * np.abs(feeds[2]).max(), "bf16") <= 1


@pytest.mark.parametrize("new,length", [(1, 300), (40, 300), (1, 20000)])
def test_paged_rows_whose_scores_are_all_minus_infinity(new, length):
    pool = -(-length // 16) + 1
    g, ids, inputs, outputs = paged_graph(new, 1, 4, 2, 64, 16, pool, pool, write=False)
    feeds = paged_feeds(g, inputs, new, [length], 16, pool)
    feeds[0], feeds[1][:] = np.abs(feeds[0]) + 1, -np.inf
    got, _ = run_gpu(g.desc, inputs, outputs, feeds)
    assert (got[0] == 0).all() and (interp.run_function(g.desc, inputs, outputs, feeds)[0] == 0).all()
