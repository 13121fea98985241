"""The attention operators on the GPU against the fp64 oracle, element by element within bounds derived from their roundings."""
import numpy as np
import pytest

from attention_cases import (attention_bounds, attention_feeds, attention_graph, head_bounds, head_feeds, head_graph, paged_bounds, paged_feeds, paged_graph,
                             within)
from lm_cases import run_gpu, to_gpu, torch_type
from oracle import interp
from paper_1707_08265_b200 import binding as B

pytestmark = pytest.mark.gpu


def types(g, outputs):
    return [g.desc["tensors"][t]["dtype"] for t in outputs]


@pytest.mark.parametrize("rows,heads,width,dims,interleaved,norm,numbers", [
    (1, 1, 8, None, 0, True, ()), (5, 3, 16, None, 1, True, ()), (33, 2, 32, 20, 0, True, ()), (70, 5, 40, 24, 1, False, ()),
    (64, 8, 64, None, 0, False, (500000.0, 8.0, 1.0, 4.0, 8192.0)), (19, 4, 72, 72, 0, True, (10000.0, 4.0)), (130, 6, 80, 48, 0, True, ()),
    (7, 12, 96, None, 1, True, (1e6, 2.0, 1.0, 1.0, 100.0, 1.25)), (600, 32, 128, None, 0, True, ()), (9, 3, 256, None, 0, True, ()),
    (9, 3, 248, 2, 0, True, ()), (3000, 5, 128, 64, 0, True, ())])
@pytest.mark.parametrize("x,u,y,gain", [("bf16", "f32", "bf16", "f32"), ("f32", "f32", "f32", "bf16"), ("f32", "bf16", "bf16", "f32")])
def test_norm_and_rotation(rows, heads, width, dims, interleaved, norm, numbers, x, u, y, gain):
    g, ids, inputs, outputs = head_graph(rows, heads, width, dims, interleaved, norm, numbers, x, u, y, gain, grad=True,
                                         grad_types=(["bf16"] if x == "bf16" else ["f32"]) + (["f32"] if norm else []))
    feeds = head_feeds(g, inputs, rows + width)
    got, _ = run_gpu(g.desc, inputs, outputs, feeds)
    want = interp.run_function(g.desc, inputs, outputs, feeds)
    bounds = head_bounds(g, inputs, outputs, feeds)
    for n, a, b, t in zip(["y", "dx", "dgain"], got, want, types(g, outputs)):
        assert within(a, b, bounds[n], t) <= 1, n


@pytest.mark.parametrize("rotate", [False, True])
def test_norm_fetched_and_alone(rotate):
    g, ids, inputs, outputs = head_graph(37, 4, 64, u="bf16", fetch_u=rotate, rotate=rotate)
    feeds = head_feeds(g, inputs, 2)
    got, f = run_gpu(g.desc, inputs, outputs, feeds)
    bounds = head_bounds(g, inputs, outputs, feeds)
    for n, a, b in zip(["u", "y"] if rotate else ["u"], got, interp.run_function(g.desc, inputs, outputs, feeds)):
        assert within(a, b, bounds[n], "bf16") <= 1, n
    assert f.num_launches() == 1


def test_far_positions():
    """The angle is exact at every int32 position."""
    g, ids, inputs, outputs = head_graph(8, 2, 128, norm=False, x="f32", y="f32")
    feeds = head_feeds(g, inputs, 8)
    feeds[1] = np.array([0, 1, -1, 2 ** 31 - 1, -2 ** 31, 10 ** 9, 123456789, -5], np.int32)
    got, _ = run_gpu(g.desc, inputs, outputs, feeds)
    want = interp.run_function(g.desc, inputs, outputs, feeds)
    # the oracle's own product of position and frequency is off by 2^-64 of an angle of 2^31 at most
    assert within(got[0], want[0], head_bounds(g, inputs, outputs, feeds)["y"], "f32") <= 1


ATTENTION = [
    # rows, heads, kv, width, causal, window, sequences, starts
    (1, 1, 1, 8, 1, 0, 1, None), (2, 2, 1, 16, 0, 0, 1, None), (127, 2, 2, 64, 1, 0, 1, None), (128, 4, 1, 128, 1, 0, 1, None), (129, 3, 3, 72, 0, 0, 1, None),
    (255, 2, 1, 128, 1, 0, 1, None), (257, 2, 2, 96, 1, 0, 1, None), (384, 2, 1, 40, 1, 100, 1, None), (600, 4, 2, 64, 1, 1, 1, None), (600, 2, 1, 128, 1, 129, 1, None),
    (640, 2, 1, 128, 0, 0, 5, None), (513, 2, 2, 80, 1, 0, 3, None), (700, 4, 2, 128, 1, 0, 1, [0, 0, 1, 130, 130, 400, 656, 700]),
    (500, 2, 2, 64, 0, 0, 1, [3, 3, 131, 390, 480]), (300, 3, 1, 32, 1, 17, 1, [0, 64, 300]), (90, 1, 1, 128, 1, 0, 1, [0, 0, 0]), (1025, 8, 2, 128, 1, 0, 1, None),
]


@pytest.mark.parametrize("rows,heads,kv,width,causal,window,sequences,starts", ATTENTION)
def test_attention_and_gradients(rows, heads, kv, width, causal, window, sequences, starts):
    g, ids, inputs, outputs = attention_graph(rows, heads, kv, width, causal, window, sequences=sequences, starts=len(starts) - 1 if starts else 0, grad=True)
    feeds = attention_feeds(g, inputs, rows + width, starts)
    got, _ = run_gpu(g.desc, inputs, outputs, feeds)
    want = interp.run_function(g.desc, inputs, outputs, feeds)
    bounds = attention_bounds(g, inputs, outputs, feeds)
    for n, a, b, t in zip(["y", "dq", "dk", "dv"], got, want, types(g, outputs)):
        assert within(a, b, bounds[n], t) <= 1, n


@pytest.mark.parametrize("types_of", [("f32", "f32", "f32", "f32", "f32"), ("bf16", "bf16", "bf16", "f32", "bf16"), ("f32", "bf16", "f32", "bf16", "f32")])
def test_attention_types(types_of):
    q, k, v, y, d = types_of
    g, ids, inputs, outputs = attention_graph(200, 4, 2, 64, q=q, k=k, v=v, y=y, dy=d, grad=True, grad_types=["f32", "bf16", "f32"])
    feeds = attention_feeds(g, inputs, 9)
    got, _ = run_gpu(g.desc, inputs, outputs, feeds)
    want = interp.run_function(g.desc, inputs, outputs, feeds)
    bounds = attention_bounds(g, inputs, outputs, feeds)
    for n, a, b, t in zip(["y", "dq", "dk", "dv"], got, want, types(g, outputs)):
        assert within(a, b, bounds[n], t) <= 1, n


@pytest.mark.parametrize("scale", [0.01, 1.0, 3.0])
def test_attention_scales(scale):
    """Flat rows, and rows whose scores differ by hundreds, with the largest at either end."""
    g, ids, inputs, outputs = attention_graph(300, 2, 1, 64, scale=scale, grad=True)
    feeds = attention_feeds(g, inputs, 10)
    feeds[1] = interp.round_bf16(feeds[1] * np.linspace(0.1, 3, 300)[:, None])
    got, _ = run_gpu(g.desc, inputs, outputs, feeds)
    want = interp.run_function(g.desc, inputs, outputs, feeds)
    bounds = attention_bounds(g, inputs, outputs, feeds)
    for n, a, b in zip(["y", "dq", "dk", "dv"], got, want):
        assert within(a, b, bounds[n], "bf16") <= 1, n


@pytest.mark.parametrize("wanted", [[0], [1], [2], [0, 2], [1, 2]])
def test_some_of_the_gradients(wanted):
    g, ids, inputs, outputs = attention_graph(333, 4, 2, 64, grad=True)
    feeds = attention_feeds(g, inputs, 11)
    full, _ = run_gpu(g.desc, inputs, outputs, feeds)
    some, _ = run_gpu(g.desc, inputs, [outputs[1 + w] for w in wanted], feeds)
    for w, a in zip(wanted, some):
        assert np.array_equal(a, full[1 + w])


def test_infinities_and_nan_in_keys_that_nobody_sees():
    """A causal row is untouched by what stands behind it, a window by what lies in front of it.  (A row whose tile held something
    not finite is computed a second time, from fp32 probabilities: it is another rounding of the same formula, so both are held
    to the formula's bound and not to each other's bits.)"""
    g, ids, inputs, outputs = attention_graph(300, 2, 1, 64, window=40)
    feeds = attention_feeds(g, inputs, 12)
    clean = interp.run_function(g.desc, inputs, outputs, feeds)
    bound = attention_bounds(g, inputs, outputs, feeds)["y"]
    for bad in (np.nan, np.inf):
        dirty = [f.copy() for f in feeds]
        dirty[1][150], dirty[2][150] = bad, bad
        got, _ = run_gpu(g.desc, inputs, outputs, dirty)
        seen = np.zeros(300, bool)
        seen[150:190] = True
        assert within(got[0][~seen], clean[0][~seen], bound[~seen], "bf16") <= 1
        assert not np.isfinite(got[0][seen]).all(axis=1).any() or bad == np.inf


def test_starts_out_of_order_are_reported():
    g, ids, inputs, outputs = attention_graph(200, 2, 1, 32, starts=3, grad=True)
    feeds = attention_feeds(g, inputs, 13, [0, 150, 90, 999])
    f = B.Graph.from_desc(g.desc).function(inputs, outputs)
    import torch
    dev = [to_gpu(a, g.desc["tensors"][t]["dtype"]) for a, t in zip(feeds, inputs)]
    outs = [torch.zeros(g.shape(t), dtype=torch_type(g.desc["tensors"][t]["dtype"]), device="cuda") for t in outputs]
    f.run_torch(dev, outs)
    assert f.status() == B.ERR_INVALID_ARG
    dev[3].copy_(torch.tensor([0, 90, 150, 200], dtype=torch.int32))
    f.run_torch(dev, outs)
    assert f.status() == 0


PAGED = [
    # heads, kv, width, page, window, new rows, lengths
    (1, 1, 8, 16, 0, [1], [1]), (4, 2, 64, 16, 0, [1, 1, 1], [1, 200, 77]), (8, 1, 128, 32, 0, [1] * 5, [1000, 17, 33, 64, 5]),
    (6, 6, 96, 64, 0, [1, 1], [300, 128]), (3, 1, 72, 16, 50, [1, 1], [300, 20]), (32, 8, 128, 16, 0, [1], [3000]), (16, 1, 64, 128, 0, [1, 1], [500, 1]),
    (4, 2, 128, 16, 0, [5, 1, 0, 130, 300], [5, 90, 40, 400, 300]), (2, 2, 64, 256, 0, [7, 7], [600, 7]), (4, 1, 80, 32, 100, [40, 1, 200], [40, 300, 500]),
    (8, 2, 128, 64, 0, [64, 64], [64, 700]), (2, 1, 40, 16, 1, [3, 2], [20, 9]), (4, 4, 128, 16, 0, [2, 3], [1, 3]), (4, 4, 32, 16, 0, [1, 1, 1], [0, 5, -3]),
    (20, 2, 64, 16, 0, [3, 3], [100, 259]), (5, 5, 128, 16, 0, [17, 16, 33], [1000, 400, 50]), (64, 1, 128, 16, 0, [1, 2], [140, 700]),
]


@pytest.mark.parametrize("heads,kv,width,page,window,new,lengths", PAGED)
@pytest.mark.parametrize("y", ["bf16", "f32"])
def test_paged_attention(heads, kv, width, page, window, new, lengths, y):
    starts = None if len(set(new)) == 1 else np.concatenate([[0], np.cumsum(new)])
    rows = sum(new) + (4 if starts is not None else 0)         # rows behind the last sequence
    most = max(1, max(-(-n // page) for n in lengths)) + 1
    pool = sum(-(-max(n, 0) // page) for n in lengths) + 2
    g, ids, inputs, outputs = paged_graph(rows, len(new), heads, kv, width, page, most, pool, window, starts=starts is not None, y=y)
    feeds = paged_feeds(g, inputs, heads + width, lengths, page, pool, starts)
    got, f = run_gpu(g.desc, inputs, outputs, feeds)
    want = interp.run_function(g.desc, inputs, outputs, feeds)
    assert within(got[0], want[0], paged_bounds(g, inputs, outputs, feeds), y) <= 1
    assert np.array_equal(got[1], want[1]) and np.array_equal(got[2], want[2])
    if starts is not None:
        assert (got[0][-4:] == 0).all()


@pytest.mark.parametrize("new", [1, 40])
def test_bad_pages_are_reported(new):
    """Numbers of no page are neither read nor written; other sequences are as they were."""
    import torch
    lengths, page, pool = [70, 90], 16, 14
    g, ids, inputs, outputs = paged_graph(2 * new, 2, 4, 2, 64, page, 6, pool)
    feeds = paged_feeds(g, inputs, 3, lengths, page, pool)
    names = [g.desc["tensors"][t]["name"] for t in inputs]
    want = interp.run_function(g.desc, inputs, outputs, feeds)
    for at, bad in (((0, 4), pool), ((0, 0), -1), ((0, 2), 2 ** 31 - 1), ((0, 1), -2 ** 31)):
        broken = [a.copy() for a in feeds]
        broken[names.index("pages")][at] = bad
        f = B.Graph.from_desc(g.desc).function(inputs, outputs)
        dev = [to_gpu(a, g.desc["tensors"][t]["dtype"]) for a, t in zip(broken, inputs)]
        outs = [torch.zeros(g.shape(t), dtype=torch.bfloat16, device="cuda") for t in outputs]
        f.run_torch(dev, outs)
        assert f.status() == B.ERR_INVALID_ARG
        y = outs[0].double().cpu().numpy()
        assert np.isfinite(y).all()
        assert within(y[new:], want[0][new:], paged_bounds(g, inputs, outputs, feeds)[new:], "bf16") <= 1
    too_long = [a.copy() for a in feeds]
    too_long[names.index("lengths")][0] = 2 ** 31 - 1
    dev = [to_gpu(a, g.desc["tensors"][t]["dtype"]) for a, t in zip(too_long, inputs)]
    f.run_torch(dev, outs)
    assert f.status() == B.ERR_INVALID_ARG
    y = outs[0].double().cpu().numpy()
    assert within(y[new:], want[0][new:], paged_bounds(g, inputs, outputs, feeds)[new:], "bf16") <= 1


def test_cache_written_in_place_and_copied():
    import torch
    lengths, page, pool = [33, 50, 16], 16, 12
    g, ids, inputs, outputs = paged_graph(3, 3, 4, 2, 64, page, 4, pool)
    feeds = paged_feeds(g, inputs, 4, lengths, page, pool)
    f = B.Graph.from_desc(g.desc).function(inputs, outputs)
    dev = [to_gpu(a, g.desc["tensors"][t]["dtype"]) for a, t in zip(feeds, inputs)]
    names = [g.desc["tensors"][t]["name"] for t in inputs]
    copies = [torch.empty(g.shape(t), dtype=torch.bfloat16, device="cuda") for t in outputs]
    f.run_torch(dev, copies)
    kc, vc = dev[names.index("kc")], dev[names.index("vc")]
    y = torch.empty_like(copies[0])
    f.run_torch(dev, [y, kc, vc])
    torch.cuda.synchronize()
    assert f.status() == 0
    for a, b in zip([y, kc, vc], copies):
        assert torch.equal(a, b)


def test_one_page_shared_by_two_sequences():
    """A common beginning is stored once: both sequences read its page."""
    lengths, page, pool = [20, 31], 16, 6
    g, ids, inputs, outputs = paged_graph(2, 2, 4, 2, 64, page, 2, pool)
    feeds = paged_feeds(g, inputs, 5, lengths, page, pool)
    names = [g.desc["tensors"][t]["name"] for t in inputs]
    feeds[names.index("pages")][1, 0] = feeds[names.index("pages")][0, 0]
    got, _ = run_gpu(g.desc, inputs, outputs, feeds)
    want = interp.run_function(g.desc, inputs, outputs, feeds)
    assert within(got[0], want[0], paged_bounds(g, inputs, outputs, feeds), "bf16") <= 1


@pytest.mark.parametrize("heads,kv,width,length", [(32, 8, 128, 40000), (2, 2, 64, 20011), (8, 1, 128, 33333)])
def test_decoding_a_long_context(heads, kv, width, length):
    page = 64
    pool = -(-length // page) + 1
    g, ids, inputs, outputs = paged_graph(1, 1, heads, kv, width, page, pool, pool)
    feeds = paged_feeds(g, inputs, 6, [length], page, pool)
    got, _ = run_gpu(g.desc, inputs, outputs[:1], feeds)
    want = interp.run_function(g.desc, inputs, outputs[:1], feeds)
    assert within(got[0], want[0], paged_bounds(g, inputs, outputs, feeds), "bf16") <= 1


def test_captured_and_replayed_on_another_stream():
    """A step captured into a graph and replayed after its inputs have changed in place, and an eager run beside it."""
    import torch
    g, ids, inputs, outputs = attention_graph(700, 4, 2, 64, starts=3, grad=True)
    first = attention_feeds(g, inputs, 20, [0, 300, 301, 700])
    second = attention_feeds(g, inputs, 21, [0, 1, 650, 690])
    b = B.Graph.from_desc(g.desc)
    f, eager = b.function(inputs, outputs), b.function(inputs, outputs)
    dt = [g.desc["tensors"][t]["dtype"] for t in inputs]
    dev = [to_gpu(a, t) for a, t in zip(first, dt)]
    outs = [torch.empty(g.shape(t), dtype=torch.bfloat16, device="cuda") for t in outputs]
    want = [torch.empty_like(o) for o in outs]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        f.run_torch(dev, outs)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            f.run_torch(dev, outs)
    torch.cuda.current_stream().wait_stream(side)
    for d, a, t in zip(dev, second, dt):
        d.copy_(to_gpu(a, t))
    for o in outs:
        o.fill_(float("nan"))
    graph.replay()
    eager.run_torch(dev, want)
    torch.cuda.synchronize()
    assert eager.status() == 0
    for a, c in zip(outs, want):
        assert torch.equal(a, c)


def test_two_streams_at_once():
    import torch
    g, ids, inputs, outputs = attention_graph(500, 4, 4, 128, grad=True)
    b = B.Graph.from_desc(g.desc)
    streams, runs = [torch.cuda.Stream() for _ in range(2)], []
    for k, s in enumerate(streams):
        feeds = attention_feeds(g, inputs, 30 + k)
        f = b.function(inputs, outputs)
        dev = [to_gpu(a, g.desc["tensors"][t]["dtype"]) for a, t in zip(feeds, inputs)]
        alone = [torch.empty(g.shape(t), dtype=torch.bfloat16, device="cuda") for t in outputs]
        f.run_torch(dev, alone)
        runs.append((f, dev, alone, [torch.empty_like(o) for o in alone], s))
    torch.cuda.synchronize()
    for _ in range(5):
        for f, dev, alone, outs, s in runs:
            f.run_torch(dev, outs, s)
    torch.cuda.synchronize()
    for f, dev, alone, outs, s in runs:
        for a, c in zip(outs, alone):
            assert torch.equal(a, c)
