"""The language-model operators on the GPU where values leave the ordinary range: precision of every value by itself."""
import numpy as np
import pytest

from lm_cases import U32, run_gpu
from oracle import interp
from paper_1707_08265_b200 import workloads as wl

pytestmark = pytest.mark.gpu

# a gate f = 1 / (1 + t) and 1 - f = t f with t = exp(-z): 2^u of the hardware to 4 units of 2^-24 and the correction's own rounding
# to 1 (t: 5), 1 + t to 1, the reciprocal to 2, the product to 1, the operator's product and sum with 0 and 1 to none
GATE = 10 * U32


@pytest.mark.parametrize("cols", [512, 513])
@pytest.mark.parametrize("length", [1, 70])
def test_gate_keeps_full_relative_precision(cols, length):
    """Rows that all start afresh: h = (1 - f) x + f h0 shows 1 - f (x = 1, h0 = 0) or f (x = 0, h0 = 1) itself, and its
    gradient dx = (1 - f) dh, dh0 = f dh.  |z| up to 86, where both are normal numbers."""
    g = wl.GraphDesc()
    seqs = 6
    rows = seqs * length
    gate, x, h0, d = g.tensor("gate", [rows, cols]), g.tensor("x", [rows, cols]), g.tensor("h0", [seqs, cols]), g.tensor("d", [rows, cols])
    h = g.op("GatedScan", [gate, x, h0], "h", [rows, cols], attrs=[seqs])
    dx, dh0 = g.grad([g.op("Mul", [h, d], "along")], [x, h0])
    rng = np.random.default_rng(cols)
    z = rng.uniform(-86, 86, (rows, cols)).astype(np.float32).astype(np.float64)
    first = np.arange(rows) % length == 0
    xv, start, dv = np.zeros((rows, cols)), np.zeros((seqs, cols)), np.zeros((rows, cols))
    xv[:, 1::2][first] = 1.0
    start[:, ::2] = 1.0
    dv[first] = 1.0
    got, _ = run_gpu(g.desc, [gate, x, h0, d], [h, dx, dh0], [z, xv, start, dv])
    f, keep = 1 / (1 + np.exp(-z[first])), 1 / (1 + np.exp(z[first]))
    want = np.where(np.arange(cols) % 2 == 0, f, keep)
    for name, a, b in (("h", got[0][first], want), ("dx", got[1][first], keep), ("dh0", got[2], f)):
        far = np.abs(a - b) / b
        assert far.max() <= GATE, "%s: %.1f units of 2^-24 at gate %g" % (name, far.max() / U32, z[first].reshape(-1)[far.argmax()])


def test_gates_at_the_ends_of_the_range():
    """Infinite and huge gates keep or replace the state exactly, tiny ones are one half, NaN stays in its column."""
    g = wl.GraphDesc()
    gate, x, h0 = g.tensor("gate", [1, 8]), g.tensor("x", [1, 8]), g.tensor("h0", [1, 8])
    h = g.op("GatedScan", [gate, x, h0], "h", [1, 8])
    z = np.array([[np.inf, -np.inf, 3e38, -3e38, 1e-45, -0.0, np.nan, 104.5]])
    (got,), _ = run_gpu(g.desc, [gate, x, h0], [h], [z, np.full((1, 8), 3.0), np.full((1, 8), 5.0)])
    assert np.array_equal(got[0, :6], [5.0, 3.0, 5.0, 3.0, 4.0, 4.0]) and np.isnan(got[0, 6]) and got[0, 7] == 5.0
