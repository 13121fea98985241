"""The oracle's language-model operators at values that are no ordinary numbers, worked by hand."""
import numpy as np

from oracle import interp
from paper_1707_08265_b200 import workloads as wl


def clipped(values, norm, limit=2.0):
    g = wl.GraphDesc()
    t, n = g.tensor("t", [len(values)]), g.tensor("n", [])
    c = g.op("ClipByNorm", [t, n], "c", attrs=[limit], out_shape=[len(values)])
    return interp.run_function(g.desc, [t, n], [c], [np.array(values, dtype=np.float64), np.array(norm)])[0]


def test_clipping_by_a_norm_that_is_no_number():
    assert np.isnan(clipped([1.0, 0.0], np.nan)).all()
    assert np.array_equal(clipped([1.0, -3.0], np.inf), [0.0, 0.0])
    assert np.array_equal(clipped([1.0, -3.0], 2.0), [1.0, -3.0]) and np.array_equal(clipped([1.0, -3.0], 4.0), [0.5, -1.5])
    assert np.array_equal(clipped([1.0, -3.0], 0.0), [1.0, -3.0])


def test_scan_passes_nothing_over_a_reset():
    g = wl.GraphDesc()
    gate, x, h0, r = g.tensor("gate", [3, 1]), g.tensor("x", [3, 1]), g.tensor("h0", [1, 1]), g.tensor("r", [3], "i32")
    h = g.op("GatedScan", [gate, x, h0, r], "h", [3, 1])
    got = interp.run_function(g.desc, [gate, x, h0, r], [h], [np.zeros((3, 1)), np.full((3, 1), 4.0), np.full((1, 1), np.nan), np.array([0, 1, 0], np.int32)])[0]
    assert np.isnan(got[0, 0]) and np.array_equal(got[1:, 0], [2.0, 3.0])
