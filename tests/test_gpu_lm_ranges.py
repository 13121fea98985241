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


@pytest.mark.parametrize("M,N,K", [(3, 300, 4096), (20, 130, 272), (50, 257, 400), (100, 200, 2064), (300, 520, 640), (2433, 2049, 272), (2400, 2056, 144)])
def test_scaled_product_whose_scales_multiply_to_a_denormal(M, N, K):
    """Scales of 1e-21 on both sides: their product has its documented error, a denormal's half step, in both kernels; rows
    whose scales multiply to a normal number have none of it, and a row of zeros stays zero."""
    g, kb, nb = wl.GraphDesc(), -(-K // 128), -(-N // 128)
    t = [g.tensor("xq", [M, K], "f8e4m3"), g.tensor("sx", [M, kb]), g.tensor("wq", [N, K], "f8e4m3"), g.tensor("sw", [nb, kb])]
    y = g.op("ScaledInnerProduct", t, "y", [M, N])
    rng = np.random.default_rng(M)
    xq, wq = (interp.round_e4m3(rng.standard_normal((r, K)) * 120.0) for r in (M, N))
    xq[0] = 0
    sx, sw = ((1e-21 * np.exp(rng.standard_normal(shape) * 0.5)).astype(np.float32).astype(np.float64) for shape in ((M, kb), (nb, kb)))
    sx[1::3] = np.float32(1e-10)
    (got,), _ = run_gpu(g.desc, t, [y], [xq, sx, wq, sw])
    want = interp.run_function(g.desc, t, [y], [xq, sx, wq, sw])[0]
    plain = np.abs(xq) @ np.abs(wq).T
    mag = (np.abs(xq) * interp._spread(sx, (M, K), 1)) @ (np.abs(wq) * interp._spread(sw, (N, K), 128)).T
    assert (got[0] == 0).all() and np.isfinite(got).all()
    # exact products, at most 128 additions in a block, a factor (half a unit, or half of 2^-149) and one addition a block
    bound = (128 + kb + 2) * U32 * mag + kb * 2.0 ** -149
    bound += np.where(np.arange(M)[:, None] % 3 == 1, 0, plain * 2.0 ** -150 * (1 + 200 * U32))
    assert (np.abs(got - want) <= bound).all()
    assert (np.abs(want[1::3]) > 2.0 ** -110).mean() > 0.9      # (ordinary numbers, for which 2^-149 is nothing)
