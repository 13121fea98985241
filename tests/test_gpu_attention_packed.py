"""Attention and PagedAttention over many packed sequences."""
import numpy as np
import pytest

from attention_cases import attention_bounds, attention_feeds, attention_graph, paged_bounds, paged_feeds, paged_graph, within
from lm_cases import run_gpu, to_gpu
from oracle import interp
from paper_1707_08265_b200 import binding as B

pytestmark = pytest.mark.gpu


def packed(sequences, longest, seed, first=0):
    """starts of sequences of 0 to `longest` rows (every fourth one empty), beginning at row `first`."""
    rng = np.random.default_rng(seed)
    n = rng.integers(0, longest + 1, sequences) * (rng.integers(0, 4, sequences) > 0)
    return first + np.concatenate([[0], np.cumsum(n)])


@pytest.mark.parametrize("sequences,longest,heads,kv,width,causal,window,first,behind", [
    (32, 40, 2, 1, 16, 1, 0, 0, 0), (33, 40, 4, 4, 64, 0, 0, 0, 5), (64, 300, 2, 1, 128, 1, 50, 7, 0), (100, 9, 3, 1, 72, 1, 0, 300, 300), (1024, 5, 2, 2, 32, 1, 0, 1, 0),
    (1025, 4, 2, 1, 64, 1, 0, 0, 130), (1100, 3, 1, 1, 128, 0, 0, 129, 1), (40, 0, 2, 2, 64, 1, 0, 0, 10)])
def test_many_sequences(sequences, longest, heads, kv, width, causal, window, first, behind):
    starts = packed(sequences, longest, sequences + width, first)
    rows = int(starts[-1]) + behind
    g, ids, inputs, outputs = attention_graph(rows, heads, kv, width, causal, window, starts=sequences, grad=True)
    feeds = attention_feeds(g, inputs, rows, starts)
    got, _ = run_gpu(g.desc, inputs, outputs, feeds)
    want, bounds = interp.run_function(g.desc, inputs, outputs, feeds), attention_bounds(g, inputs, outputs, feeds)
    for n, a, b in zip(("y", "dq", "dk", "dv"), got, want):
        assert within(a, b, bounds[n], "bf16") <= 1, n
        assert (a[:first] == 0).all() and (a[starts[-1]:] == 0).all()


@pytest.mark.parametrize("sequences,longest,heads,kv,width,first", [(40, 30, 4, 2, 64, 3), (200, 20, 6, 2, 128, 0), (1100, 4, 2, 1, 32, 140)])
def test_many_sequences_over_a_cache(sequences, longest, heads, kv, width, first):
    rng = np.random.default_rng(sequences)
    starts = packed(sequences, longest, sequences, first)
    lengths = np.diff(starts) + rng.integers(0, 90, sequences)
    pool, most = int((-(-lengths // 16)).sum()) + 1, int(-(-lengths.max() // 16))
    g, ids, inputs, outputs = paged_graph(int(starts[-1]) + 6, sequences, heads, kv, width, 16, most, pool, starts=True)
    feeds = paged_feeds(g, inputs, 60, lengths, 16, pool, starts)
    got, _ = run_gpu(g.desc, inputs, outputs, feeds)
    want = interp.run_function(g.desc, inputs, outputs, feeds)
    assert within(got[0], want[0], paged_bounds(g, inputs, outputs, feeds), "bf16") <= 1
    assert np.array_equal(got[1], want[1]) and np.array_equal(got[2], want[2])
    assert (got[0][:first] == 0).all() and (got[0][starts[-1]:] == 0).all()


def test_as_many_sequences_as_rows():
    """A row that sees itself alone: y is v and dv is dy.  A CTA's start does not grow with the number of sequences: two kernels of some 132000
    and some 264000 CTAs end in some 13 ms (a walk over all sequences in each CTA would take sixteen times as long as the 46 ms of a quarter of them)."""
    import torch
    rows = 65536
    g, ids, inputs, outputs = attention_graph(rows, 2, 2, 64, starts=rows, grad=True)
    gen = torch.Generator(device="cuda").manual_seed(5)
    dev = [torch.arange(rows + 1, dtype=torch.int32, device="cuda") if g.desc["tensors"][t]["dtype"] == "i32" else
           torch.randn(g.shape(t), generator=gen, device="cuda").to(torch.bfloat16) for t in inputs]
    outs = [torch.full(g.shape(t), float("nan"), dtype=torch.bfloat16, device="cuda") for t in outputs]
    f = B.Graph.from_desc(g.desc).function(inputs, outputs)
    f.run_torch(dev, outs)
    start, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    start.record()
    f.run_torch(dev, outs)
    end.record()
    torch.cuda.synchronize()
    assert f.status() == 0
    assert torch.equal(outs[0], dev[2]) and torch.equal(outs[3], dev[4])
    # ds = dp - delta is what two fp32 sums of 64 products differ by: 128 * 2^-24 of the sum of their magnitudes, 0.125 of it here
    size = (dev[2].float().abs() * dev[4].float().abs()).view(rows, 2, 64).sum(-1, keepdim=True)
    for d, x in ((outs[1], dev[1]), (outs[2], dev[0])):
        assert bool((d.float().view(rows, 2, 64).abs() <= 128 * 2.0 ** -24 * 0.125 * size * x.float().view(rows, 2, 64).abs() * (1 + 2.0 ** -6) + 1e-30).all())
    assert start.elapsed_time(end) < 40


@pytest.mark.parametrize("sequences", [40, 200])
def test_many_starts_out_of_order_are_reported(sequences):
    """No access leaves the tensors whatever stands in starts, and the next run with good ones is right."""
    import torch
    rows, rng = 700, np.random.default_rng(sequences)
    good = np.sort(rng.integers(0, rows + 1, sequences + 1))
    g, ids, inputs, outputs = attention_graph(rows, 4, 2, 64, starts=sequences, grad=True)
    feeds = attention_feeds(g, inputs, sequences, good)
    f = B.Graph.from_desc(g.desc).function(inputs, outputs)
    dev = [to_gpu(a, g.desc["tensors"][t]["dtype"]) for a, t in zip(feeds, inputs)]
    raw = [torch.full((rows * g.shape(t)[1] + 64,), 7.0, dtype=torch.bfloat16, device="cuda") for t in outputs]
    outs = [b[:-64].view(rows, -1) for b in raw]
    for bad in (rng.permutation(good), good[::-1].copy(), rng.integers(-2 ** 31, 2 ** 31, sequences + 1), np.where(np.arange(sequences + 1) % 2, 0, rows)):
        dev[3].copy_(torch.from_numpy(bad.astype(np.int32)))
        f.run_torch(dev, outs)
        assert f.status() == B.ERR_INVALID_ARG and all(bool((b[-64:] == 7).all()) for b in raw)
    dev[3].copy_(torch.from_numpy(good.astype(np.int32)))
    f.run_torch(dev, outs)
    assert f.status() == 0
    want, bounds = interp.run_function(g.desc, inputs, outputs, feeds), attention_bounds(g, inputs, outputs, feeds)
    for n, a, b in zip(("y", "dq", "dk", "dv"), outs, want):
        assert within(a.double().cpu().numpy(), b, bounds[n], "bf16") <= 1, n
