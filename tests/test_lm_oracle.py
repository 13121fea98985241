"""Pins of the oracle's language-model operators: values worked by hand, closed forms and central differences."""
import numpy as np
import pytest

from oracle import interp
from paper_1707_08265_b200 import workloads as wl


def run(build, feeds):
    g = wl.GraphDesc()
    ids, outs = build(g)
    return interp.run_function(g.desc, ids, outs, feeds)


def test_norm_of_a_row_of_equal_values_is_the_gain():
    def build(g):
        h, w = g.tensor("h", [2, 4]), g.tensor("g", [4])
        return [h, w], [g.op("RMSNorm", [h, w], "y", [2, 4], attrs=[0.0])]
    (y,) = run(build, [np.full((2, 4), -3.0), np.arange(4.0)])
    assert np.allclose(y, -np.arange(4.0)[None].repeat(2, 0), atol=1e-15)


def test_norm_has_unit_mean_square():
    def build(g):
        h, w = g.tensor("h", [5, 33]), g.tensor("g", [33])
        return [h, w], [g.op("RMSNorm", [h, w], "y", [5, 33], attrs=[0.0])]
    (y,) = run(build, [np.random.default_rng(0).standard_normal((5, 33)) * 7, np.ones(33)])
    assert np.allclose((y ** 2).mean(1), 1.0, atol=1e-12)


def test_e4m3_rounding_against_the_list_of_all_values():
    import torch
    table = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    table = np.unique(table[np.isfinite(table)])
    assert np.array_equal(interp.round_e4m3(table), table)                       # every value stays itself
    mid = (table[1:] + table[:-1]) / 2
    lo, hi = table[:-1], table[1:]
    assert np.array_equal(interp.round_e4m3(np.nextafter(mid, -np.inf)), lo)
    assert np.array_equal(interp.round_e4m3(np.nextafter(mid, np.inf)), hi)
    tie = interp.round_e4m3(mid)
    bits = {float(v): i for i, v in enumerate(table[table >= 0])}                 # the code's last bit is even
    assert all(bits[abs(float(t))] % 2 == 0 for t in tie)
    assert np.array_equal(interp.round_e4m3([1e9, -np.inf]), [448.0, -448.0]) and np.isnan(interp.round_e4m3([np.nan]))[0]


def test_scales_and_values_of_a_ragged_block():
    def build(g):
        x = g.tensor("x", [130, 129])
        s = g.op("BlockScale", [x], "s", [2, 2], attrs=[128])
        return [x], [s, g.op("Quantize", [x, s], "q", [130, 129], "f8e4m3")]
    x = np.zeros((130, 129))
    x[0, 0], x[129, 128], x[5, 7] = 896.0, -2.0, 3.0
    s, q = run(build, [x])
    assert np.allclose(s, [[2.0, 2.0 ** -126], [2.0 ** -126, 2.0 / 448]])
    assert q[0, 0] == 448 and q[129, 128] == -448 and q[5, 7] == 1.5


def test_scaled_product_against_its_sum():
    rng = np.random.default_rng(3)
    M, N, K = 3, 130, 144
    xq, wq = interp.round_e4m3(rng.standard_normal((M, K)) * 50), interp.round_e4m3(rng.standard_normal((N, K)) * 50)
    sx, sw = rng.uniform(0.1, 1, (M, 2)), rng.uniform(0.1, 1, (2, 2))

    def build(g):
        t = [g.tensor("xq", [M, K], "f8e4m3"), g.tensor("sx", [M, 2]), g.tensor("wq", [N, K], "f8e4m3"), g.tensor("sw", [2, 2])]
        return t, [g.op("ScaledInnerProduct", t, "y", [M, N])]
    (y,) = run(build, [xq, sx, wq, sw])
    for m, n in [(0, 0), (2, 129), (1, 127), (1, 128)]:
        want = sum(xq[m, k] * wq[n, k] * sx[m, k // 128] * sw[n // 128, k // 128] for k in range(K))
        assert abs(y[m, n] - want) <= 1e-9 * max(1, abs(want))


def test_norm_of_many_tensors_and_clipping():
    def build(g):
        a, b = g.tensor("a", [2]), g.tensor("b", [1, 2])
        n = g.op("GlobalNorm", [a, b], "n", [])
        return [a, b], [n, g.op("ClipByNorm", [a, n], "ca", [2], attrs=[2.5]), g.op("ClipByNorm", [b, n], "cb", [1, 2], attrs=[6.0])]
    n, ca, cb = run(build, [np.array([3.0, 0.0]), np.array([[0.0, -4.0]])])
    assert n == 5.0 and np.array_equal(ca, [1.5, 0.0]) and np.array_equal(cb, [[0.0, -4.0]])


def test_scan_with_constant_gate_is_a_geometric_mean():
    f, L = 0.75, 9
    gate = np.full((2 * L, 1), np.log(f / (1 - f)))
    h0 = np.array([[2.0], [0.0]])

    def build(g):
        a, x, h = g.tensor("gate", [2 * L, 1]), g.tensor("x", [2 * L, 1]), g.tensor("h0", [2, 1])
        return [a, x, h], [g.op("GatedScan", [a, x, h], "h", [2 * L, 1], attrs=[2])]
    (y,) = run(build, [gate, np.ones((2 * L, 1)), h0])
    t = np.arange(1, L + 1)
    assert np.allclose(y[:L, 0], f ** t * 2 + 1 - f ** t) and np.allclose(y[L:, 0], 1 - f ** t)


def test_scan_reset_cuts_the_sequence():
    rng = np.random.default_rng(1)
    gate, x, h0 = rng.standard_normal((7, 3)), rng.standard_normal((7, 3)), rng.standard_normal((1, 3))
    reset = np.array([0, 0, 0, 5, 0, 0, -1], dtype=np.int32)

    def build(with_reset, rows, state):
        def b(g):
            t = [g.tensor("gate", [rows, 3]), g.tensor("x", [rows, 3])]
            t += [g.tensor("h0", [1, 3])] if state else []
            t += [g.tensor("reset", [rows], "i32")] if with_reset else []
            return t, [g.op("GatedScan", t, "h", [rows, 3])]
        return b
    (y,) = run(build(True, 7, True), [gate, x, h0, reset])
    (a,) = run(build(False, 3, True), [gate[:3], x[:3], h0])
    (b,) = run(build(False, 3, False), [gate[3:6], x[3:6]])
    (c,) = run(build(False, 1, False), [gate[6:], x[6:]])
    assert np.array_equal(y, np.concatenate([a, b, c]))


@pytest.mark.parametrize("case", ["norm", "scan", "scan_reset", "norm_same"])
def test_gradients_against_central_differences(case):
    rng = np.random.default_rng(7)
    g = wl.GraphDesc()
    if case.startswith("norm"):
        h, w, d = g.tensor("h", [3, 5]), g.tensor("g", [5]), g.tensor("d", [3, 5])
        src = g.op("Mul", [h, h], "hh") if case == "norm_same" else h
        y = g.op("RMSNorm", [src, w], "y", [3, 5], attrs=[1e-3])
        ids, feeds, wrts = [h, w, d], [rng.standard_normal((3, 5)), rng.standard_normal(5), rng.standard_normal((3, 5))], [h, w]
    else:
        gate, x, h0, d = g.tensor("gate", [6, 2]), g.tensor("x", [6, 2]), g.tensor("h0", [2, 2]), g.tensor("d", [6, 2])
        ins = [gate, x, h0]
        ids, feeds = [gate, x, h0, d], [rng.standard_normal((6, 2)), rng.standard_normal((6, 2)), rng.standard_normal((2, 2)), rng.standard_normal((6, 2))]
        if case == "scan_reset":
            r = g.tensor("reset", [6], "i32")
            ins, ids, feeds = ins + [r], ids + [r], feeds + [np.array([0, 1, 0, 1, 0, 0], dtype=np.int32)]
        y = g.op("GatedScan", ins, "h", [6, 2], attrs=[2])
        wrts = [gate, x, h0]
    obj = g.op("Mul", [y, d], "obj")
    grads = g.grad([obj], wrts)
    got = interp.run_function(g.desc, ids, grads, feeds)
    for w, a in zip(wrts, got):
        fd = interp.finite_difference(g.desc, ids, feeds, [obj], w)
        assert np.allclose(a, fd, rtol=1e-6, atol=1e-7), w
