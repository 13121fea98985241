"""The language-model operators on the GPU against the fp64 oracle, at the sizes, types and values where they can go wrong."""
import numpy as np
import pytest

from lm_cases import (U16, U32, as_type, e4m3_half_step, norm_graph, normals, run_gpu, scan_bounds, scan_graph, to_gpu)
from oracle import interp
from paper_1707_08265_b200 import workloads as wl

pytestmark = pytest.mark.gpu


def close(got, want, bound, dtype, what):
    # the oracle's bf16 value is itself rounded: each of the two is off by at most half a step from its exact value, so values
    # whose fp32 forms lie on two sides of a tie are a whole step (2 U16 of the value) apart
    bound = bound + (2 * U16 * np.abs(want) * (1 + U16) if dtype == "bf16" else 0) + U32 * np.abs(want)
    bad = ~(np.abs(got - want) <= bound + 1e-37)
    assert not bad.any(), "%s: %d of %d outside, worst %.3g of its bound" % (
        what, bad.sum(), bad.size, np.nanmax(np.abs(got - want)[bad] / (bound[bad] + 1e-37)))


NORM_SIZES = [(1, 1), (3, 7), (2, 8), (5, 96), (4, 128), (9, 250), (130, 1000), (7, 1001), (600, 136), (3, 4096), (2, 5000), (2, 8200), (3, 8195),
              (2, 16384), (2, 16392), (1, 20001), (9700, 40)]
# rstd: a sum of squares in at most 32 terms a thread and a tree (each rounding halved by the root), rsqrt to 2 units, two products
NORM_REL = 32 * U32


@pytest.mark.parametrize("rows,cols", NORM_SIZES)
@pytest.mark.parametrize("types", [("bf16", "bf16", "bf16", "bf16", "f32"), ("f32", "f32", "f32", "f32", "f32"), ("f32", "bf16", "bf16", "f32", "bf16"),
                                   ("bf16", None, None, "f32", "f32"), ("f32", None, None, "bf16", "f32")])
def test_norm(rows, cols, types):
    x, r, h, y, gain = types
    g, ids, inputs, outputs = norm_graph(rows, cols, x, r, h or "bf16", y, gain)
    feeds = normals(g.desc, inputs, rows * 100003 + cols, {"r": 3.0})
    got, f = run_gpu(g.desc, inputs, outputs, feeds)
    want = interp.run_function(g.desc, inputs, outputs, feeds)
    assert f.num_launches() == 1
    if r:
        close(got[0], want[0], 0 * want[0], h, "h")
    close(got[-1], want[-1], NORM_REL * np.abs(want[-1]), y, "y")


@pytest.mark.parametrize("rows,cols", NORM_SIZES)
@pytest.mark.parametrize("types", [("bf16", "bf16", "f32"), ("f32", "f32", "bf16"), ("f32", None, "f32")])
@pytest.mark.parametrize("fetch_y", [True, False])
def test_norm_with_eight_bit_output(rows, cols, types, fetch_y):
    x, r, y = types
    g, ids, inputs, outputs = norm_graph(rows, cols, x, r, "bf16", y, eight_bit=True if fetch_y else "only")
    feeds = normals(g.desc, inputs, rows * 100003 + cols, {"r": 3.0})
    got, f = run_gpu(g.desc, inputs, outputs, feeds)
    assert f.num_launches() == 1
    want = dict(zip(outputs, interp.run_function(g.desc, inputs, outputs, feeds)))
    got = dict(zip(outputs, got))
    yv = interp.run_function(g.desc, inputs, [ids["y"]], feeds)[0]
    rel = NORM_REL + (2 * U16 if y == "bf16" else 0)      # a bf16 y may have been rounded the other way
    s, q = got[ids["s"]], got[ids["q"]]
    assert (np.abs(s - want[ids["s"]]) <= (rel + 2 * U32) * want[ids["s"]]).all()
    v = yv / interp._spread(want[ids["s"]], yv.shape, 1)
    assert (np.abs(q - v) <= e4m3_half_step(v) + 2 * (rel + 3 * U32) * np.abs(v)).all()
    if fetch_y:                                          # with the y and s that came out, each value is the nearest one
        v = got[ids["y"]] / interp._spread(s, yv.shape, 1)
        assert (np.abs(q - v) <= e4m3_half_step(v) + 3 * U32 * np.abs(v)).all()


@pytest.mark.parametrize("rows,cols", NORM_SIZES)
@pytest.mark.parametrize("types", [("bf16", "bf16", "bf16", "bf16", "bf16"), ("f32", "f32", "f32", "f32", None), ("bf16", None, None, "f32", "f32"),
                                   ("f32", None, None, "bf16", None), ("f32", "bf16", "bf16", "f32", "f32")])
def test_norm_gradient(rows, cols, types):
    x, r, h, y, skip = types
    g, ids, inputs, outputs = norm_graph(rows, cols, x, r, h or "bf16", y, grad=True, skip=skip)
    feeds = normals(g.desc, inputs, rows * 100003 + cols, {"r": 3.0})
    got, f = run_gpu(g.desc, inputs, outputs, feeds)
    got = dict(zip(outputs, got))
    (want, val, _) = interp.run_function(g.desc, inputs, outputs, feeds, return_all=True)
    want = dict(zip(outputs, want))
    hv, dy, gain = val[ids["h"]], val[ids["dy"]], val[ids["g"]]
    rstd = 1 / np.sqrt((hv ** 2).mean(1, keepdims=True) + 1e-6)
    t = np.abs(dy * gain)
    mag = rstd * (t + np.abs(hv) * rstd ** 2 * (t * np.abs(hv)).mean(1, keepdims=True))
    mag = mag + (np.abs(val[ids["dskip"]]) if skip else 0)
    close(got[ids["dx"]], want[ids["dx"]], 2 * NORM_REL * mag, "f32", "dx")
    # at most rows terms in the running fp32 sum of a column, each with rstd's error
    close(got[ids["dg"]], want[ids["dg"]], (NORM_REL + (rows + 3) * U32) * (np.abs(dy * hv) * rstd).sum(0), "f32", "dg")


def test_norm_gradient_in_the_middle_of_a_graph():
    """h feeds the norm and a later operator that is no addition of tensors in memory; only dg is wanted, then only dx."""
    g = wl.GraphDesc()
    x, w, a = g.tensor("x", [37, 264]), g.tensor("w", [264]), g.tensor("a", [37, 264])
    h = g.op("Tanh", [x], "h")
    y = g.op("RMSNorm", [h, w], "y", [37, 264])
    z = g.op("Mul", [g.op("Sin", [y], "sy"), g.op("Mul", [h, a], "ha")], "z")
    dx, dw = g.grad([z], [x, w])
    for outs in ([dx], [dw], [z, dx, dw]):
        feeds = normals(g.desc, [x, w, a], 5)
        got, _ = run_gpu(g.desc, [x, w, a], outs, feeds)
        for o, p in zip(got, interp.run_function(g.desc, [x, w, a], outs, feeds)):
            assert np.abs(o - p).max() <= 2e-5 * np.abs(p).max()


def test_norm_of_a_zero_row_and_of_non_finite_rows():
    g, ids, inputs, outputs = norm_graph(5, 256, "f32", None, None, "f32", eight_bit=True)
    x = np.random.default_rng(0).standard_normal((5, 256))
    x[0] = 0
    x[1, 3], x[2, 200] = np.nan, np.inf
    got, _ = run_gpu(g.desc, inputs, outputs, [x, np.ones(256)])
    y, s, q = got
    assert (y[0] == 0).all() and (s[0] == 2.0 ** -126).all() and (q[0] == 0).all()
    assert np.isnan(y[1]).all() and np.isnan(s[1]).all() and np.isnan(q[1]).all()
    assert np.isnan(y[2, 200]) and (np.delete(y[2], 200) == 0).all()
    assert np.isfinite(y[3:]).all() and np.isfinite(q[3:]).all()


# ---- scales and e4m3 values ---------------------------------------------------------------------------------

@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 128), (3, 130), (127, 16), (128, 128), (129, 257), (300, 1000), (5, 4096), (260, 1001)])
@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_quantize(rows, cols, block_rows, dtype):
    g = wl.GraphDesc()
    x = g.tensor("x", [rows, cols], dtype)
    s = g.op("BlockScale", [x], "s", [-(-rows // block_rows), -(-cols // 128)], attrs=[block_rows])
    q = g.op("Quantize", [x, s], "q", [rows, cols], "f8e4m3")
    (feed,) = normals(g.desc, [x], rows + cols)
    feed[rows // 2, cols // 2] = 0
    (sv, qv), f = run_gpu(g.desc, [x], [s, q], [feed])
    assert f.num_launches() == 1
    want = interp.run_function(g.desc, [x], [s], [feed])[0]
    assert (np.abs(sv - want) <= U32 * want).all()
    v = feed / interp._spread(sv, feed.shape, block_rows)
    assert (np.abs(qv - v) <= e4m3_half_step(v) + 3 * U32 * np.abs(v)).all()
    # the same values in scales that are fed, and the scales or the values alone
    (q2,), _ = run_gpu(g.desc, [x, s], [q], [feed, sv])
    (s3,), _ = run_gpu(g.desc, [x], [s], [feed])
    (q3,), _ = run_gpu(g.desc, [x], [q], [feed])
    assert np.array_equal(q2, qv) and np.array_equal(q3, qv) and np.array_equal(s3, sv)


@pytest.mark.parametrize("block_rows", [1, 128])
def test_quantize_extremes(block_rows):
    g = wl.GraphDesc()
    x = g.tensor("x", [4, 640])
    s = g.op("BlockScale", [x], "s", [4 if block_rows == 1 else 1, 5], attrs=[block_rows])
    q = g.op("Quantize", [x, s], "q", [4, 640], "f8e4m3")
    v = np.zeros((4, 640))
    v[:, 128:256] = 1e-45                                   # amax / 448 below the smallest scale
    v[0, 256], v[0, 257] = np.nan, 1.0
    v[0, 384], v[0, 385] = np.inf, 1.0
    v[:, 512:] = np.float32(3e38)
    (sv, qv), _ = run_gpu(g.desc, [x], [s, q], [v])
    assert sv[0, 0] == 2.0 ** -126 and (qv[:, :256] == 0).all() and sv[0, 1] == 2.0 ** -126
    assert np.isnan(sv[0, 2]) and np.isnan(qv[0, 256:384]).all()
    assert np.isinf(sv[0, 3]) and np.isnan(qv[0, 384]) and qv[0, 385] == 0
    assert (qv[:, 512:] == 448).all()


# ---- the product in e4m3 ------------------------------------------------------------------------------------

def product_case(M, N, K, out, seed):
    g, kb = wl.GraphDesc(), -(-K // 128)
    t = [g.tensor("xq", [M, K], "f8e4m3"), g.tensor("sx", [M, kb]), g.tensor("wq", [N, K], "f8e4m3"), g.tensor("sw", [-(-N // 128), kb])]
    y = g.op("ScaledInnerProduct", t, "y", [M, N], out)
    rng = np.random.default_rng(seed)
    feeds = [interp.round_e4m3(rng.standard_normal((M, K)) * 120), as_type(np.exp(rng.standard_normal((M, kb))) / 100, "f32"),
             interp.round_e4m3(rng.standard_normal((N, K)) * 120), as_type(np.exp(rng.standard_normal((-(-N // 128), kb))) / 100, "f32")]
    return g, t, y, feeds


@pytest.mark.parametrize("M,N,K", [(1, 1, 16), (1, 64, 128), (2, 129, 144), (5, 256, 4096), (8, 1000, 272), (16, 512, 2048), (17, 136, 1040), (33, 384, 512), (64, 128, 128),
                                   (65, 300, 400), (128, 256, 128), (129, 257, 384), (200, 1024, 1024), (300, 520, 2064), (512, 768, 640), (1000, 1000, 1008),
                                   # enough tiles of 128 x 256 for every SM: the kernel of many rows, ragged in every extent, more tiles than SMs
                                   (2433, 2049, 272), (2400, 2056, 128), (4900, 1000, 400), (19000, 96, 16),
                                   # ... whose rows start at multiples of 4 and of 8 bytes
                                   (2431, 2050, 160), (1301, 2052, 272)])
@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_scaled_product(M, N, K, out):
    g, t, y, feeds = product_case(M, N, K, out, M * 7 + N * 3 + K)
    (got,), f = run_gpu(g.desc, t, [y], feeds)
    want = interp.run_function(g.desc, t, [y], feeds)[0]
    mag = (np.abs(feeds[0]) * interp._spread(feeds[1], (M, K), 1)) @ (np.abs(feeds[2]) * interp._spread(feeds[3], (N, K), 128)).T
    # products of e4m3 values are exact in fp32; at most 128 additions in a block, one product of scales, one addition a block
    close(got, want, (min(K, 128) + -(-K // 128) + 2) * U32 * mag, out, "y")


def test_scaled_product_keeps_non_finite_values_where_they_are():
    g, t, y, feeds = product_case(70, 200, 256, "f32", 1)
    feeds[0][3, 5] = np.nan
    feeds[1][9, 1] = np.inf
    feeds[3][1, 0] = 0.0
    (got,), _ = run_gpu(g.desc, t, [y], feeds)
    assert np.isnan(got[3]).all() and not np.isfinite(got[9]).any()
    rest = np.delete(got, [3, 9], axis=0)
    assert np.isfinite(rest).all()


@pytest.mark.parametrize("M,N,K", [(3, 300, 1024), (100, 128, 640), (2432, 2048, 1024)])
def test_scaled_product_wait_that_runs_out_is_reported(M, N, K, monkeypatch):
    """Failure detection without a fault: the producer leaves out its first stage, the first wait for it runs out on a short
    budget, the kernel reports DRAGON_ERR_TIMEOUT and returns by itself; the next run of the same function is correct."""
    from paper_1707_08265_b200 import binding as B
    import torch
    g, t, y, feeds = product_case(M, N, K, "f32", 5)
    f = B.Graph.from_desc(g.desc).function(t, [y])
    dev = [to_gpu(a, g.desc["tensors"][i]["dtype"]) for a, i in zip(feeds, t)]
    out = torch.empty(M, N, device="cuda")
    monkeypatch.setenv("DRAGON_GEMM_WAIT_BUDGET", "2000000")
    monkeypatch.setenv("DRAGON_GEMM_DROP_FIRST_LOAD", "1")
    f.run_torch(dev, [out])
    assert f.status() == B.ERR_TIMEOUT
    monkeypatch.delenv("DRAGON_GEMM_WAIT_BUDGET")
    monkeypatch.delenv("DRAGON_GEMM_DROP_FIRST_LOAD")
    run_gpu(g.desc, t, [y], feeds, f)
    f.run_torch(dev, [out])
    assert f.status() == 0
    want = interp.run_function(g.desc, t, [y], feeds)[0]
    mag = (np.abs(feeds[0]) * interp._spread(feeds[1], (M, K), 1)) @ (np.abs(feeds[2]) * interp._spread(feeds[3], (N, K), 128)).T
    close(out.double().cpu().numpy(), want, (128 + -(-K // 128) + 2) * U32 * mag, "f32", "y")


# ---- norm over many tensors and clipping --------------------------------------------------------------------

def clip_graph(shapes, types, limit, out_types=None):
    g = wl.GraphDesc()
    t = [g.tensor("g%d" % i, s, d) for i, (s, d) in enumerate(zip(shapes, types))]
    n = g.op("GlobalNorm", t, "norm", [])
    c = [g.op("ClipByNorm", [a, n], "c%d" % i, s, d, attrs=[limit]) for i, (a, s, d) in enumerate(zip(t, shapes, out_types or types))]
    return g, t, n, c


@pytest.mark.parametrize("shapes", [[[]], [[1]], [[7]], [[8191], [1], [8193], []], [[33, 77], [5], [1000, 100], [64, 64]], [[3]] * 300, [[100, 8192], [17]],
                                    [[4096, 4097], [12], [3000, 1001]]])
@pytest.mark.parametrize("limit", [0.5, 1e6])
@pytest.mark.parametrize("types", [("f32",), ("bf16",), ("f32", "bf16")])
def test_clip(shapes, limit, types):
    types = [types[i % len(types)] for i in range(len(shapes))]
    g, t, n, c = clip_graph(shapes, types, limit)
    feeds = normals(g.desc, t, len(shapes))
    got, f = run_gpu(g.desc, t, [n] + c, feeds)
    want = interp.run_function(g.desc, t, [n] + c, feeds)
    small = sum(-(-int(np.prod(s)) // (4096 if d == "f32" else 8192)) for s, d in zip(shapes, types)) <= 2 * 4 * 148 and len(shapes) <= 256
    assert f.num_launches() == (1 if small else 2 * -(-len(shapes) // 256))
    close(got[0], want[0], 18 * U32 * want[0], "f32", "norm")
    for a, b, d in zip(got[1:], want[1:], types):
        close(a, b, 21 * U32 * np.abs(b), d, "clipped")
    if limit == 1e6:
        for a, b in zip(got[1:], feeds):
            assert np.array_equal(a, b)


@pytest.mark.parametrize("scale", [1e-30, 1e-22, 1e-10, 1e15, 1e25, 1e37])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_norm_over_fp32_range(scale, dtype):
    g, t, n, c = clip_graph([[5000], [100, 3]], [dtype] * 2, 1.0)
    feeds = normals(g.desc, t, 1, {"g0": scale, "g1": scale * 1e-3})
    (got,), _ = run_gpu(g.desc, t, [n], feeds)
    want = np.sqrt(sum((a.astype(np.float64) ** 2).sum() for a in feeds))
    if want < 3.4e38:
        assert abs(got - want) <= 18 * U32 * want
    else:
        assert np.isinf(got)


def test_clip_of_non_finite_gradients():
    g, t, n, c = clip_graph([[100], [50]], ["f32"] * 2, 1.0)
    a, b = np.ones(100), np.ones(50)
    a[3] = np.nan
    got, _ = run_gpu(g.desc, t, [n] + c, [a, b])
    assert np.isnan(got[0]) and np.isnan(got[1]).all() and np.isnan(got[2]).all()
    a[3] = np.inf
    got, _ = run_gpu(g.desc, t, [n] + c, [a, b])
    assert np.isinf(got[0]) and np.isnan(got[1][3]) and (np.delete(got[1], 3) == 0).all() and (got[2] == 0).all()
    got, _ = run_gpu(g.desc, t, [n] + c, [0 * b[:1].repeat(100), 0 * b])
    assert got[0] == 0 and (got[1] == 0).all()


def test_clip_between_types_and_in_an_updater():
    """A clipped tensor of another type, and one that an update consumes: the factor is a scalar of its program."""
    g = wl.GraphDesc()
    a, b, w, lr = g.tensor("a", [300, 20]), g.tensor("b", [77], "bf16"), g.tensor("w", [300, 20]), g.tensor("lr", [])
    n = g.op("GlobalNorm", [a, b], "n", [])
    cb = g.op("ClipByNorm", [b, n], "cb", [77], "f32", attrs=[0.25])
    ca = g.op("ClipByNorm", [a, n], "ca", [300, 20], attrs=[0.25])
    w2 = g.op("Sub", [w, g.op("Mul", [lr, ca], "step")], "w2")
    feeds = normals(g.desc, [a, b, w, lr], 2)
    got, f = run_gpu(g.desc, [a, b, w, lr], [w2, cb, n], feeds)
    for o, p in zip(got, interp.run_function(g.desc, [a, b, w, lr], [w2, cb, n], feeds)):
        assert np.abs(o - p).max() <= 30 * U32 * max(1, np.abs(p).max())
    # a norm that is fed (over several processes, say) and a second limit
    got, _ = run_gpu(g.desc, [a, n, w, lr], [w2], [feeds[0], np.float32(50.0), feeds[2], feeds[3]])
    want = interp.run_function(g.desc, [a, n, w, lr], [w2], [feeds[0], np.array(50.0), feeds[2], feeds[3]])
    assert np.abs(got[0] - want[0]).max() <= 30 * U32 * np.abs(want[0]).max()


# ---- the gated recurrence -----------------------------------------------------------------------------------

SCAN_SIZES = [(1, 1, 1), (1, 1, 64), (64, 1, 70), (1, 2, 3), (1, 127, 2), (1, 128, 64), (1, 129, 66), (2, 128, 8), (3, 50, 1), (3, 300, 65), (5, 700, 33), (1, 2500, 64), (2, 1300, 130),
              (40, 13, 256), (1, 9000, 4), (300, 2, 10)]


@pytest.mark.parametrize("seqs,length,cols", SCAN_SIZES)
@pytest.mark.parametrize("types", [("bf16", "bf16", "bf16", "f32"), ("f32", "f32", "f32", None), ("f32", "bf16", "f32", "bf16")])
@pytest.mark.parametrize("reset", [None, 0.02, 0.5])
def test_scan_and_gradient(seqs, length, cols, types, reset):
    gate, x, h, h0 = types
    g, ids, inputs, outputs = scan_graph(seqs, length, cols, gate, x, h, h0, reset is not None, True)
    feeds = normals(g.desc, inputs, seqs * 1009 + length * 31 + cols, {"gate": 2.0})
    if reset is not None:
        at = inputs.index(ids["reset"])
        feeds[at] = (np.random.default_rng(length).random(seqs * length) < reset).astype(np.int32) * np.int32(-7)
    names = {g.desc["tensors"][t]["name"]: a for t, a in zip(inputs, feeds)}
    bound = scan_bounds(g.desc, ids, names, seqs)
    want = dict(zip(outputs, interp.run_function(g.desc, inputs, outputs, feeds)))
    got = dict(zip(outputs, run_gpu(g.desc, inputs, outputs, feeds)[0]))
    # the oracle's gradient uses its own states; a bf16 h is only an output
    for name in ["h", "dgate", "dx"] + (["dh0"] if h0 else []):
        close(got[ids[name]], want[ids[name]], bound[name], h if name == "h" else "f32", name)
    (alone,), _ = run_gpu(g.desc, inputs, [ids["h"]], feeds)
    assert np.array_equal(alone, got[ids["h"]])
    (dx_alone,), _ = run_gpu(g.desc, inputs, [ids["dx"]], feeds)
    assert np.array_equal(dx_alone, got[ids["dx"]])


@pytest.mark.parametrize("seqs,length,cols,dtype", [(1, 20000, 64, "bf16"), (1, 9000, 33, "f32"), (3, 5000, 200, "f32")])
def test_scan_gives_the_same_bits_every_time(seqs, length, cols, dtype):
    """Tiles of a long sequence hand their states on while they run in any order; what is added to what does not depend on it."""
    g, ids, inputs, outputs = scan_graph(seqs, length, cols, dtype, dtype, "f32", "f32", False, True, dtype)
    feeds = normals(g.desc, inputs, 6, {"gate": 2.0})
    first, f = run_gpu(g.desc, inputs, outputs, feeds)
    for _ in range(10):
        again, _ = run_gpu(g.desc, inputs, outputs, feeds, f)
        assert all(np.array_equal(a, b) for a, b in zip(first, again))


def test_scan_extreme_gates():
    g, ids, inputs, outputs = scan_graph(1, 300, 8, "f32", "f32", "f32", "f32", grad=True)
    feeds = normals(g.desc, inputs, 3)
    gate = feeds[0]
    gate[:, 0], gate[:, 1], gate[:, 2], gate[:, 3], gate[:, 4] = 200.0, -200.0, 88.0, -88.0, np.where(np.arange(300) % 2, 1e30, -1e30)
    want = dict(zip(outputs, interp.run_function(g.desc, inputs, outputs, feeds)))
    got = dict(zip(outputs, run_gpu(g.desc, inputs, outputs, feeds)[0]))
    for t in outputs:
        assert np.isfinite(got[t]).all()
        assert (np.abs(got[t] - want[t]) <= 3e-5 * np.abs(want[t]).max(0) + 1e-30).all()


def test_scan_reset_stops_non_finite_states():
    """What is in front of a reset, a sequence's start or in another column does not reach a row, finite or not."""
    g, ids, inputs, outputs = scan_graph(2, 400, 64, "f32", "f32", "f32", "f32", reset=True, grad=True)
    feeds = normals(g.desc, inputs, 4)
    at = {g.desc["tensors"][t]["name"]: i for i, t in enumerate(inputs)}
    reset = np.zeros(800, np.int32)
    reset[[200, 650]] = 1
    feeds[at["reset"]] = reset
    feeds[at["x"]][150, 3] = np.nan
    feeds[at["x"]][260, 5] = np.inf
    feeds[at["h0"]][1, 7] = np.nan
    feeds[at["dh"]][300, 9] = np.nan
    clean = [a.copy() for a in feeds]
    for n in ("x", "h0", "dh"):
        clean[at[n]] = np.nan_to_num(clean[at[n]], nan=0.0, posinf=0.0)
    want = dict(zip(outputs, interp.run_function(g.desc, inputs, outputs, clean)))
    got = dict(zip(outputs, run_gpu(g.desc, inputs, outputs, feeds)[0]))
    h, dx, dgate = (got[ids[n]] for n in ("h", "dx", "dgate"))
    assert np.isnan(h[150:200, 3]).all() and not np.isfinite(h[260:400, 5]).any() and np.isnan(h[400:650, 7]).all()
    assert np.isnan(dx[200:301, 9]).all()
    expect_bad = np.zeros_like(h, bool)
    expect_bad[150:200, 3] = expect_bad[260:400, 5] = expect_bad[400:650, 7] = True
    assert np.array_equal(~np.isfinite(h), expect_bad)
    assert np.isfinite(dx[:200, 9]).all() and np.isfinite(dx[301:, 9]).all()
    ok = ~expect_bad
    assert np.abs(h - want[ids["h"]])[ok].max() < 1e-5


def test_scan_wait_that_runs_out_is_reported(monkeypatch):
    """Failure detection without a fault: the chain's first tile publishes nothing, the tiles behind it give up on a short
    budget, the kernel ends and reports DRAGON_ERR_TIMEOUT; the next run of the same function is correct."""
    from paper_1707_08265_b200 import binding as B
    g, ids, inputs, outputs = scan_graph(1, 1000, 64, "f32", "f32", "f32", "f32", False, True)
    feeds = normals(g.desc, inputs, 6)
    want, f = run_gpu(g.desc, inputs, outputs, feeds)
    import torch
    dev = [to_gpu(a, g.desc["tensors"][t]["dtype"]) for a, t in zip(feeds, inputs)]
    outs = [torch.empty(g.shape(t), device="cuda") for t in outputs]
    monkeypatch.setenv("DRAGON_SCAN_WAIT_BUDGET", "2000000")
    monkeypatch.setenv("DRAGON_SCAN_WITHHOLD", "1")
    f.run_torch(dev, outs)
    assert f.status() == B.ERR_TIMEOUT
    monkeypatch.delenv("DRAGON_SCAN_WAIT_BUDGET")
    monkeypatch.delenv("DRAGON_SCAN_WITHHOLD")
    again, _ = run_gpu(g.desc, inputs, outputs, feeds, f)
    assert all(np.array_equal(a, b) for a, b in zip(want, again))


@pytest.mark.parametrize("seqs,length", [(1, 70), (5, 1)])
def test_scan_of_one_tensor_in_two_places(seqs, length):
    """gate and x are the same tensor, or x and h0 (one row per sequence): the gradient sums both places."""
    g = wl.GraphDesc()
    rows = seqs * length
    x, d = g.tensor("x", [rows, 6]), g.tensor("d", [rows, 6])
    h = g.op("GatedScan", [x, x] if length > 1 else [x, x, x], "h", [rows, 6], attrs=[seqs])
    dx, = g.grad([g.op("Mul", [h, d], "along")], [x])
    feeds = normals(g.desc, [x, d], 3)
    got, _ = run_gpu(g.desc, [x, d], [h, dx], feeds)
    for o, p in zip(got, interp.run_function(g.desc, [x, d], [h, dx], feeds)):
        assert np.abs(o - p).max() <= 1e-5 * max(1.0, np.abs(p).max())


# ---- how functions of these operators are run --------------------------------------------------------------------

def mixed_functions():
    """One function of each kind of kernel (norm, gradient, quantisation, product of many and few rows, clipping, scan over many tiles)."""
    out = []
    out.append(norm_graph(70, 264, grad=True, skip="bf16"))
    out.append(norm_graph(70, 300, eight_bit=True))
    g, t, y, _ = product_case(40, 300, 400, "bf16", 1)
    out.append((g, {}, t, [y]))
    g, t, y, _ = product_case(2600, 2100, 144, "f32", 1)
    out.append((g, {}, t, [y]))
    g, t, n, c = clip_graph([[100, 33], [7]], ["f32", "bf16"], 0.5)
    out.append((g, {}, t, [n] + c))
    g, t, n, c = clip_graph([[4096, 3000], [7]], ["bf16", "f32"], 0.5)
    out.append((g, {}, t, [n] + c))
    out.append(scan_graph(2, 1000, 66, reset=True, grad=True))
    return out


def feeds_of(g, inputs, seed):
    out = []
    for a, t in zip(normals(g.desc, inputs, seed), inputs):
        out.append((np.abs(a) < 0.05).astype(np.int32) if g.desc["tensors"][t]["dtype"] == "i32" else a)
    return out


@pytest.mark.parametrize("k", range(7))
@pytest.mark.parametrize("eager_first", [True, False])
def test_captured_and_replayed(k, eager_first):
    """A run captured into a CUDA graph before or after a first eager one, two graphs of one function (one workspace), replays
    in any order and eager runs between them, with inputs that change in place: always the bits of a plain run."""
    import torch
    from paper_1707_08265_b200 import binding as B
    g, _, inputs, outputs = mixed_functions()[k]
    f = B.Graph.from_desc(g.desc).function(inputs, outputs)
    f.ensure_workspace()
    f._ws.fill_(0xA5)
    sets = [feeds_of(g, inputs, s) for s in (1, 2)]
    plain = [run_gpu(g.desc, inputs, outputs, s)[0] for s in sets]
    dev = [[to_gpu(a, g.desc["tensors"][t]["dtype"]) for a, t in zip(s, inputs)] for s in sets]
    feeds = [t.clone() for t in dev[0]]
    outs = [torch.empty(g.shape(t), dtype={"f32": torch.float32, "bf16": torch.bfloat16, "f8e4m3": torch.float8_e4m3fn}[g.desc["tensors"][t]["dtype"]], device="cuda")
            for t in outputs]

    def check(which):
        torch.cuda.synchronize()
        for o, p in zip(outs, plain[which]):
            assert np.array_equal(o.double().cpu().numpy(), p)

    def load(which):
        for a, b in zip(feeds, dev[which]):
            a.copy_(b)
        for o in outs:
            o.reshape(-1).view(torch.uint8).fill_(0x7F)

    if eager_first:
        f.run_torch(feeds, outs)
        check(0)
    graphs = []
    for _ in range(2):
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            f.run_torch(feeds, outs)
        graphs.append(gr)
    for which, step in ((1, graphs[1]), (0, graphs[0]), (1, None), (0, graphs[1]), (1, graphs[0]), (0, graphs[0])):
        load(which)
        step.replay() if step else f.run_torch(feeds, outs)
        check(which)


def test_two_streams_and_two_functions_at_once():
    """Functions with workspaces of their own on streams of their own, many runs in flight."""
    import torch
    from paper_1707_08265_b200 import binding as B
    jobs = []
    for k, (g, _, inputs, outputs) in enumerate(mixed_functions()):
        feeds = feeds_of(g, inputs, 9)
        plain = run_gpu(g.desc, inputs, outputs, feeds)[0]
        f = B.Graph.from_desc(g.desc).function(inputs, outputs)
        f.ensure_workspace()
        dev = [to_gpu(a, g.desc["tensors"][t]["dtype"]) for a, t in zip(feeds, inputs)]
        from lm_cases import torch_type
        outs = [torch.empty(g.shape(t), dtype=torch_type(g.desc["tensors"][t]["dtype"]), device="cuda") for t in outputs]
        jobs.append((f, dev, outs, plain, torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(20):
        for f, dev, outs, _, st in jobs:
            f.run_torch(dev, outs, st)
    torch.cuda.synchronize()
    for f, _, outs, plain, _ in jobs:
        assert f.status() == 0
        for o, p in zip(outs, plain):
            assert np.array_equal(o.double().cpu().numpy(), p)


@pytest.mark.parametrize("big", [False, True])
def test_clip_over_its_own_tensors(big):
    """dragon_function_can_alias: the clipped tensors may be the tensors; one that is below the limit stays as it is."""
    import torch
    from paper_1707_08265_b200 import binding as B
    g, t, n, c = clip_graph([[4096, 2100], [4096, 300], [77]] if big else [[1000, 30], [513], [77]], ["bf16", "f32", "f32"], 2.0)
    feeds = normals(g.desc, t, 3)
    want = run_gpu(g.desc, t, [n] + c, feeds)[0]
    f = B.Graph.from_desc(g.desc).function(t, [n] + c)
    assert all(f.can_alias(i, i + 1) for i in range(3)) and not f.can_alias(0, 2)
    dev = [to_gpu(a, g.desc["tensors"][x]["dtype"]) for a, x in zip(feeds, t)]
    norm = torch.empty((), device="cuda")
    f.run_torch(dev, [norm] + dev)
    for o, p in zip([norm] + dev, want):
        assert np.array_equal(o.double().cpu().numpy(), p)
    clipped = [x.clone() for x in dev]
    f.run_torch(dev, [norm] + dev)            # the norm is the limit now, up to rounding
    assert abs(float(norm) - 2.0) < 1e-2
    for o, p in zip(dev, clipped):
        assert (o.float() - p.float()).abs().max() <= 2 * U16 * p.float().abs().max()


def test_host_buffers_and_named_tensors():
    """The same functions through dragon_run_host and through a workspace of named tensors (e4m3 among them)."""
    import torch
    from lm_cases import torch_type
    from paper_1707_08265_b200 import binding as B
    for g, _, inputs, outputs in mixed_functions():
        feeds = feeds_of(g, inputs, 4)
        plain, f = run_gpu(g.desc, inputs, outputs, feeds)
        host = [to_gpu(a, g.desc["tensors"][t]["dtype"]).cpu().pin_memory() for a, t in zip(feeds, inputs)]
        outs = [torch.empty(g.shape(t), dtype=torch_type(g.desc["tensors"][t]["dtype"])).pin_memory() for t in outputs]
        staging = torch.empty(f.staging_bytes() + 256, dtype=torch.uint8, device="cuda")
        base = (staging.data_ptr() + 255) & ~255
        f.run_host([h.data_ptr() for h in host], [o.data_ptr() for o in outs], base, f.staging_bytes(), torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        for o, p in zip(outs, plain):
            assert np.array_equal(o.double().numpy(), p)
        ws = B.Workspace()
        f2 = B.Graph.from_desc(g.desc).function(inputs, outputs)
        for h, t in zip(host, inputs):
            info = g.desc["tensors"][t]
            ws.feed(info["name"], B.DTYPES[info["dtype"]], info["shape"], h.data_ptr())
        for _ in range(2):
            ws.run(f2)
        torch.cuda.synchronize()
        for t, p in zip(outputs, plain):
            info = g.desc["tensors"][t]
            o = torch.empty(info["shape"], dtype=torch_type(info["dtype"]))
            ws.fetch(info["name"], o.data_ptr(), o.numel() * o.element_size())
            torch.cuda.synchronize()
            assert np.array_equal(o.double().numpy(), p)
        f2.close()
        ws.close()
