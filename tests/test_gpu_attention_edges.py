"""The attention operators where they could go wrong: values that are not finite in a gradient, offsets beyond 32 bits, waits that
run out, steps that share a launch, operands that are the same tensor, host buffers."""
import numpy as np
import pytest

from attention_cases import (as_type, attention_bounds, attention_feeds, attention_graph, head_bounds, head_feeds, head_graph, paged_bounds, paged_feeds,
                             paged_graph, within)
from lm_cases import run_gpu, to_gpu, torch_type
from oracle import interp
from paper_1707_08265_b200 import binding as B
from paper_1707_08265_b200 import workloads as wl

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("types_of", [("f32", "bf16", "f32"), ("bf16", "f32", "f32"), ("f32", "f32", "bf16")])
def test_types_of_the_gradients(types_of):
    g, ids, inputs, outputs = attention_graph(150, 4, 2, 40, grad=True, grad_types=types_of)
    feeds = attention_feeds(g, inputs, 40)
    got, _ = run_gpu(g.desc, inputs, outputs, feeds)
    want, bounds = interp.run_function(g.desc, inputs, outputs, feeds), attention_bounds(g, inputs, outputs, feeds)
    for n, dt, a, b in zip(("dq", "dk", "dv"), types_of, got[1:], want[1:]):
        assert within(a, b, bounds[n], dt) <= 1, n
    h, hids, inputs, outputs = head_graph(70, 3, 24, grad=True, grad_types=types_of[:2])
    feeds = head_feeds(h, inputs, 41)
    got, _ = run_gpu(h.desc, inputs, outputs, feeds)
    want, bounds = interp.run_function(h.desc, inputs, outputs, feeds), head_bounds(h, inputs, outputs, feeds)
    for n, dt, a, b in zip(("dx", "dgain"), types_of, got[1:], want[1:]):
        assert within(a, b, bounds[n], dt) <= 1, n


@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
@pytest.mark.parametrize("where", ["q", "k", "v", "dy"])
def test_values_that_are_not_finite_stay_among_the_rows_that_meet_them(bad, where):
    """Causal with a window of 20: row d of q or dy is met by itself and reaches the keys d - 19 .. d, row d of k or v is met by the
    rows d .. d + 19 and reaches their keys.  Other rows, of the same tile too, are as they were."""
    d, w, rows = 150, 20, 300
    g, ids, inputs, outputs = attention_graph(rows, 2, 1, 64, window=w, grad=True)
    feeds = attention_feeds(g, inputs, 42)
    clean, bounds = interp.run_function(g.desc, inputs, outputs, feeds), attention_bounds(g, inputs, outputs, feeds)
    feeds[{"q": 0, "k": 1, "v": 2, "dy": 3}[where]][d] = bad
    got, _ = run_gpu(g.desc, inputs, outputs, feeds)
    by_rows, by_keys = np.zeros(rows, bool), np.zeros(rows, bool)
    by_rows[d:d + (1 if where in ("q", "dy") else w)] = True
    by_keys[d - w + 1:d + (1 if where in ("q", "dy") else w)] = True
    for n, a, b in zip(("y", "dq", "dk", "dv"), got, clean):
        fine = ~(by_rows if n in ("y", "dq") else by_keys)
        if n == "y" and where == "dy":
            fine[:] = True
        assert within(a[fine], b[fine], bounds[n][fine], "bf16") <= 1, n
    if np.isnan(bad) and where != "dy":
        assert np.isnan(got[0][by_rows]).all(axis=1).any()


# few rows and heads: a CTA's keys (or queries) are split into parts that a launch of its own puts together
@pytest.mark.parametrize("rows,heads,kv,width,causal,window,sequences,starts", [
    (3001, 1, 1, 32, 1, 0, 1, None), (1500, 2, 1, 128, 0, 0, 1, None), (1024, 3, 1, 64, 1, 0, 2, None), (2500, 1, 1, 96, 1, 700, 1, None), (1999, 4, 4, 40, 1, 0, 1, None),
    (1400, 8, 2, 64, 1, 0, 1, [0, 0, 1, 130, 1290, 1290]), (1300, 2, 2, 128, 0, 0, 1, [40, 50, 1200, 1201])])
def test_work_that_is_split(rows, heads, kv, width, causal, window, sequences, starts):
    g, ids, inputs, outputs = attention_graph(rows, heads, kv, width, causal, window, sequences=sequences, starts=len(starts) - 1 if starts else 0, grad=True)
    feeds = attention_feeds(g, inputs, rows, starts)
    got, f = run_gpu(g.desc, inputs, outputs, feeds)
    want, bounds = interp.run_function(g.desc, inputs, outputs, feeds), attention_bounds(g, inputs, outputs, feeds)
    for n, a, b in zip(("y", "dq", "dk", "dv"), got, want):
        assert within(a, b, bounds[n], "bf16") <= 1, n
    if starts:
        for a in got:
            assert (a[:starts[0]] == 0).all() and (a[starts[-1]:] == 0).all()
    again, _ = run_gpu(g.desc, inputs, outputs, feeds)
    for a, b in zip(got, again):
        assert np.array_equal(a, b)
    some, _ = run_gpu(g.desc, inputs, outputs[2:3], feeds)
    assert np.array_equal(some[0], got[2])


def test_values_that_are_not_finite_in_work_that_is_split():
    rows, d, w = 2000, 900, 300
    g, ids, inputs, outputs = attention_graph(rows, 1, 1, 64, window=w, grad=True)
    feeds = attention_feeds(g, inputs, 51)
    clean, bounds = interp.run_function(g.desc, inputs, outputs, feeds), attention_bounds(g, inputs, outputs, feeds)
    feeds[1][d], feeds[2][d] = np.nan, np.inf
    got, _ = run_gpu(g.desc, inputs, outputs, feeds)
    for n, a, b in zip(("y", "dq", "dk", "dv"), got, clean):
        fine = np.ones(rows, bool)
        fine[(d if n in ("y", "dq") else d - w + 1):d + w] = False
        assert within(a[fine], b[fine], bounds[n][fine], "bf16") <= 1, n
        assert np.isnan(a[~fine]).any(axis=1).all() or n in ("dk", "dv")


def test_a_sequence_of_nan_beside_others_in_a_tile():
    starts = [0, 30, 77, 128, 140]
    g, ids, inputs, outputs = attention_graph(160, 4, 2, 72, starts=4, grad=True)
    feeds = attention_feeds(g, inputs, 43, starts)
    clean, bounds = interp.run_function(g.desc, inputs, outputs, feeds), attention_bounds(g, inputs, outputs, feeds)
    for k in (0, 1, 2, 4):
        feeds[k][30:77] = np.nan
        feeds[k][140:] = np.nan                   # rows of no sequence
    got, _ = run_gpu(g.desc, inputs, outputs, feeds)
    fine = np.ones(160, bool)
    fine[30:77] = False
    for n, a, b in zip(("y", "dq", "dk", "dv"), got, clean):
        assert within(a[fine], b[fine], bounds[n][fine], "bf16") <= 1, n
        assert (a[140:] == 0).all() and np.isnan(a[30:77]).any(axis=1).all()


@pytest.mark.parametrize("kind", ["forward", "gradients", "chunk"])
def test_waits_that_run_out_and_the_run_behind_them(kind, monkeypatch):
    """The first copy's signal never comes: with the wait budget shortened to about a millisecond the kernels record DRAGON_ERR_TIMEOUT,
    let copies and products in flight land, free their tensor memory and return; the same function is right again afterwards."""
    import torch
    if kind == "chunk":
        lengths, page, pool, starts = [300, 90], 16, 27, [0, 200, 260]
        g, ids, inputs, outputs = paged_graph(260, 2, 4, 2, 64, page, 20, pool, starts=True, write=False)
        feeds = paged_feeds(g, inputs, 44, lengths, page, pool, starts)
        bounds = [paged_bounds(g, inputs, outputs, feeds)]
    else:
        g, ids, inputs, outputs = attention_graph(700, 4, 2, 128, grad=kind == "gradients")
        feeds = attention_feeds(g, inputs, 44)
        bounds = list(attention_bounds(g, inputs, outputs, feeds).values())
    f = B.Graph.from_desc(g.desc).function(inputs, outputs)
    dev = [to_gpu(a, g.desc["tensors"][t]["dtype"]) for a, t in zip(feeds, inputs)]
    outs = [torch.zeros(g.shape(t), dtype=torch.bfloat16, device="cuda") for t in outputs]
    monkeypatch.setenv("DRAGON_ATTENTION_WAIT_BUDGET", "2000000")
    monkeypatch.setenv("DRAGON_ATTENTION_DROP_FIRST_LOAD", "1")
    f.run_torch(dev, outs)
    assert f.status() == B.ERR_TIMEOUT
    monkeypatch.delenv("DRAGON_ATTENTION_WAIT_BUDGET")
    monkeypatch.delenv("DRAGON_ATTENTION_DROP_FIRST_LOAD")
    f.run_torch(dev, outs)
    assert f.status() == 0
    want = interp.run_function(g.desc, inputs, outputs, feeds)
    for o, w, b in zip(outs, want, bounds):
        assert within(o.double().cpu().numpy(), w, b, "bf16") <= 1


def test_steps_of_one_launch_keep_their_own_numbers():
    """Neighbouring norms run as one launch: each with its own eps, its own type in front of the rotation, its own pairing."""
    rng = np.random.default_rng(45)
    g = wl.GraphDesc()
    pos = g.tensor("pos", [60], "i32")
    inputs, outputs, feeds = [pos], [], [rng.integers(0, 4000, 60).astype(np.int32)]
    for k, (eps, u, y, dims, pairing, heads, width) in enumerate([(1e-6, "f32", "bf16", 32, 0, 3, 32), (2.0, "f32", "bf16", 32, 0, 2, 32), (1e-6, "bf16", "bf16", 20, 0, 2, 32),
                                                                   (0.5, "f32", "f32", 32, 1, 1, 32), (1e-3, "f32", "bf16", 8, 0, 5, 8)]):
        x, gain = g.tensor("x%d" % k, [60, heads * width], "bf16"), g.tensor("gain%d" % k, [width])
        n = g.op("HeadNorm", [x, gain], "u%d" % k, g.shape(x), u, attrs=[eps])
        outputs.append(g.op("Rotate", [n, pos], "y%d" % k, g.shape(x), y, attrs=[heads, dims, pairing]))
        inputs += [x, gain]
        feeds += [as_type(rng.standard_normal(g.shape(x)), "bf16"), as_type(1 + 0.2 * rng.standard_normal(width), "f32")]
    got, f = run_gpu(g.desc, inputs, outputs, feeds)
    for t, a, b in zip(outputs, got, interp.run_function(g.desc, inputs, outputs, feeds)):
        dt = g.desc["tensors"][t]["dtype"]
        # (values of magnitude 4 at most after the norm and the turn; a value in bf16 in front of the turn may fall to the other side)
        assert np.abs(a - b).max() <= 8 * (2.0 ** -8 if dt == "bf16" or g.desc["tensors"][t]["name"] == "y2" else 2.0 ** -18)


@pytest.mark.parametrize("kv", [1, 2])
def test_queries_keys_and_values_out_of_one_tensor(kv):
    """One tensor as all three: its gradient is the sum of the three."""
    g = wl.GraphDesc()
    x, dy = g.tensor("x", [140, 64], "bf16"), g.tensor("dy", [140, 64], "bf16")
    y = g.op("Attention", [x, x, x], "y", [140, 64], "bf16", attrs=[kv, kv])
    outputs = [y] + g.grad([g.op("Mul", [y, dy], "along")], [x])
    rng = np.random.default_rng(46)
    feeds = [as_type(rng.standard_normal((140, 64)), "bf16") for _ in range(2)]
    got, _ = run_gpu(g.desc, [x, dy], outputs, feeds)
    want = interp.run_function(g.desc, [x, dy], outputs, feeds)
    h, ids, inputs, outs = attention_graph(140, kv, kv, 64 // kv, grad=True)
    b = attention_bounds(h, inputs, outs, [feeds[0]] * 3 + [feeds[1]])
    parts = interp.run_function(h.desc, inputs, outs, [feeds[0]] * 3 + [feeds[1]])
    assert within(got[0], want[0], b["y"], "bf16") <= 1
    # the three may be rounded to bf16 before they are added
    room = b["dq"] + b["dk"] + b["dv"] + 2.0 ** -8 * sum(np.abs(p) for p in parts[1:])
    assert within(got[1], want[1], room, "f32") <= 1


def test_attention_of_attention():
    """Two of them one after another with their gradients, in one function: workspaces and row sums of their own."""
    g = wl.GraphDesc()
    q, k, v, dy = (g.tensor(n, [200, 64], "bf16") for n in ("q", "k", "v", "dy"))
    a = g.op("Attention", [q, k, v], "a", [200, 64], "bf16", attrs=[2, 2])
    y = g.op("Attention", [a, k, v], "y", [200, 64], "bf16", attrs=[2, 2, 0])
    outputs = [a, y] + g.grad([g.op("Mul", [y, dy], "along")], [q, k, v])
    feeds = [as_type(np.random.default_rng(47 + i).standard_normal((200, 64)), "bf16") for i in range(4)]
    got, _ = run_gpu(g.desc, [q, k, v, dy], outputs, feeds)
    for a, b in zip(got, interp.run_function(g.desc, [q, k, v, dy], outputs, feeds)):
        # ten roundings of 2^-8 one after another, in each of two evaluations
        assert np.linalg.norm(a - b) <= 20 * 2.0 ** -8 * np.linalg.norm(b)


def test_host_buffers_and_named_tensors():
    import torch
    cases = [attention_graph(130, 4, 2, 32, grad=True), head_graph(40, 3, 24, grad=True), paged_graph(5, 5, 4, 2, 64, 16, 4, 22)]
    for g, ids, inputs, outputs in cases:
        if "kc" in ids:
            feeds = paged_feeds(g, inputs, 48, [1, 64, 30, 17, 50], 16, 22)
        else:
            feeds = (attention_feeds if "q" in ids else head_feeds)(g, inputs, 48)
        plain, f = run_gpu(g.desc, inputs, outputs, feeds)
        host = [to_gpu(a, g.desc["tensors"][t]["dtype"]).cpu().pin_memory() for a, t in zip(feeds, inputs)]
        outs = [torch.empty(g.shape(t), dtype=torch_type(g.desc["tensors"][t]["dtype"])).pin_memory() for t in outputs]
        staging = torch.empty(f.staging_bytes() + 256, dtype=torch.uint8, device="cuda")
        f.run_host([h.data_ptr() for h in host], [o.data_ptr() for o in outs], (staging.data_ptr() + 255) & ~255, f.staging_bytes(), torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        for o, p in zip(outs, plain):
            assert np.array_equal(o.double().numpy(), p)


def test_a_cache_in_32_bits_and_starts_out_of_order():
    """CacheWrite moves f32 rows too; starts out of order are cut and reported, and rows behind a sequence's place in the table too."""
    import torch
    rng = np.random.default_rng(49)
    g = wl.GraphDesc()
    c, r, p, n, s = g.tensor("c", [64, 24]), g.tensor("r", [9, 24]), g.tensor("pages", [3, 2], "i32"), g.tensor("lengths", [3], "i32"), g.tensor("starts", [4], "i32")
    o = g.op("CacheWrite", [c, r, p, n, s], "o", [64, 24], attrs=[16])
    feeds = [as_type(rng.standard_normal((64, 24)), "f32"), as_type(rng.standard_normal((9, 24)), "f32"), np.array([[2, 0], [1, 9], [3, 3]], np.int32),
             np.array([20, 4, 3], np.int32), np.array([0, 5, 9, 9], np.int32)]
    (got,), _ = run_gpu(g.desc, [c, r, p, n, s], [o], feeds)
    want = interp.run_function(g.desc, [c, r, p, n, s], [o], feeds)[0]
    assert np.array_equal(got, want) and (got != feeds[0]).any()
    f = B.Graph.from_desc(g.desc).function([c, r, p, n, s], [o])
    for starts, lengths in (([0, 7, 3, 9], [20, 4, 3]), ([-4, 5, 9, 9], [20, 4, 3]), ([0, 5, 9, 11], [20, 4, 3]), ([0, 5, 9, 9], [40, 4, 3]), ([0, 5, 9, 9], [20, 18, 3])):
        dev = [to_gpu(a, t) for a, t in zip(feeds[:3] + [np.array(lengths), np.array(starts)], ("f32", "f32", "i32", "i32", "i32"))]
        out = torch.empty(64, 24, device="cuda")
        f.run_torch(dev, [out])
        assert f.status() == B.ERR_INVALID_ARG and bool(torch.isfinite(out).all())


def test_rows_beyond_32_bits():
    """Tensors of more than 2^31 elements: the last sequences (and the first) are what they are alone, up to roundings."""
    import torch
    rows, heads, kv, width, each = 263168, 64, 1, 128, 257           # 2^31 elements are 262144 rows
    count = rows // each
    assert count * each == rows
    gen = torch.Generator(device="cuda").manual_seed(3)

    def drawn(cols):
        t = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")
        for part in t.split(32768):
            part.copy_(torch.randn(part.shape, generator=gen, device="cuda"))
        return t

    def graph(rows, sequences):
        g = wl.GraphDesc()
        x, gain, pos = g.tensor("x", [rows, heads * width], "bf16"), g.tensor("gain", [width]), g.tensor("pos", [rows], "i32")
        k, v, dy = g.tensor("k", [rows, kv * width], "bf16"), g.tensor("v", [rows, kv * width], "bf16"), g.tensor("dy", [rows, heads * width], "bf16")
        q = g.op("Rotate", [g.op("HeadNorm", [x, gain], "u", g.shape(x)), pos], "q", g.shape(x), "bf16", attrs=[heads])
        y = g.op("Attention", [q, k, v], "y", g.shape(x), "bf16", attrs=[heads, kv, 1, 0, 0.0, sequences])
        return g, [x, gain, pos, k, v, dy], [y] + g.grad([g.op("Mul", [y, dy], "along")], [x, k, v], ["bf16"] * 3)

    feeds = [drawn(heads * width), torch.ones(width, device="cuda"), torch.arange(rows, dtype=torch.int32, device="cuda") % each,
             drawn(width), drawn(width), drawn(heads * width)]
    g, inputs, outputs = graph(rows, count)
    f = B.Graph.from_desc(g.desc).function(inputs, outputs)
    outs = [torch.full(g.shape(t), float("nan"), dtype=torch.bfloat16, device="cuda") for t in outputs]
    f.run_torch(feeds, outs)
    assert f.status() == 0
    small, s_in, s_out = graph(2 * each, 2)
    alone = B.Graph.from_desc(small.desc).function(s_in, s_out)
    for a in (0, rows - 2 * each):
        some = [t if t.shape[0] == width else t[a:a + 2 * each].clone() for t in feeds]
        parts = [torch.empty(small.shape(t), dtype=torch.bfloat16, device="cuda") for t in s_out]
        alone.run_torch(some, parts)
        assert alone.status() == 0
        # alone there is little work, and it is split: probabilities of a part are rounded relative to its own maximum, so bits differ.
        # Probabilities, scores' gradient, the result they go through and the result are rounded, each by 2^-8 at most, in both
        for o, p in zip(outs, parts):
            for k in range(2):
                x, y = (t[k * each:(k + 1) * each].float() for t in (o[a:a + 2 * each], p))
                assert float((x - y).norm()) <= 8 * 2.0 ** -8 * float(y.norm())
    for o in outs:
        assert all(bool(torch.isfinite(part).all()) for part in o.split(32768))


@pytest.mark.parametrize("new", [1, 70])
def test_a_cache_beyond_32_bits(new):
    """Two caches of more than 2^31 elements, written in place; the sequences' pages are the last ones, the first and some between."""
    import torch
    heads, kv, width, page = 32, 16, 128, 32
    pool = 2 ** 31 // (kv * width * page) + 40
    numbers = [pool - 1, 0, pool - 2, pool // 2, pool - 30, 1, pool - 39, 17]
    lengths, most = [100, 128], 4
    small, ids, inputs, outputs = paged_graph(2 * new, 2, heads, kv, width, page, most, 8)
    feeds = paged_feeds(small, inputs, 50, lengths, page, 8)
    want = interp.run_function(small.desc, inputs, outputs, feeds)
    bound = paged_bounds(small, inputs, outputs, feeds)
    g, ids, inputs, outputs = paged_graph(2 * new, 2, heads, kv, width, page, most, pool)
    names = [g.desc["tensors"][t]["name"] for t in inputs]
    dev = []
    for n, a, t in zip(names, feeds, inputs):
        if n in ("kc", "vc"):
            c = torch.zeros(pool * page, kv * width, dtype=torch.bfloat16, device="cuda")
            for j, at in enumerate(numbers):
                c[at * page:(at + 1) * page] = to_gpu(a[j * page:(j + 1) * page], "bf16")
            dev.append(c)
        elif n == "pages":
            dev.append(to_gpu(np.array(numbers, np.int64)[np.clip(a, 0, 7)], "i32"))
        else:
            dev.append(to_gpu(a, g.desc["tensors"][t]["dtype"]))
    f = B.Graph.from_desc(g.desc).function(inputs, outputs)
    y = torch.empty(g.shape(outputs[0]), dtype=torch.bfloat16, device="cuda")
    kc, vc = dev[names.index("kc")], dev[names.index("vc")]
    f.run_torch(dev, [y, kc, vc])
    assert f.status() == 0
    assert within(y.double().cpu().numpy(), want[0], bound, "bf16") <= 1
    for c, w in ((kc, want[1]), (vc, want[2])):
        for j, at in enumerate(numbers):
            assert np.array_equal(c[at * page:(at + 1) * page].double().cpu().numpy(), w[j * page:(j + 1) * page])


def test_everything_nan_ends_soon():
    """A training run that has come apart: every row is computed by itself, and ends at its first key.  (Every row over all of its keys would
    take some seconds here.)"""
    import torch
    g, ids, inputs, outputs = attention_graph(32768, 8, 2, 128, grad=True)
    dev = [torch.full(g.shape(t), float("nan"), dtype=torch.bfloat16, device="cuda") for t in inputs]
    outs = [torch.zeros(g.shape(t), dtype=torch.bfloat16, device="cuda") for t in outputs]
    f = B.Graph.from_desc(g.desc).function(inputs, outputs)
    f.run_torch(dev, outs)
    start, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    start.record()
    f.run_torch(dev, outs)
    end.record()
    torch.cuda.synchronize()
    assert f.status() == 0 and all(bool(torch.isnan(o).all()) for o in outs)
    assert start.elapsed_time(end) < 200
