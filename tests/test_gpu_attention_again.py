"""Rows that are computed a second time by themselves (a tile held something not finite): what they give, and that they end."""
import numpy as np
import pytest

from attention_cases import attention_bounds, attention_feeds, attention_graph, paged_bounds, paged_feeds, paged_graph, within
from lm_cases import run_gpu
from oracle import interp
from paper_1707_08265_b200 import binding as B

pytestmark = pytest.mark.gpu


def spoil(a, bad, seed, some=3):
    """A few single elements."""
    rng = np.random.default_rng(seed)
    a[rng.integers(0, a.shape[0], some), rng.integers(0, a.shape[1], some)] = bad


def compare(name, got, want, clean, bound, dtype="bf16"):
    """Not finite where the formula is not; everything else is as it was without what is not finite."""
    fine = np.isfinite(want)
    assert not np.isfinite(got[~fine]).any(), name
    assert within(got[fine], clean[fine], bound[fine], dtype) <= 1, name


def over_seen(p, x, seen):
    """Rows of p times x, over what each row sees and nothing else (a product of whole matrices takes 0 times the rest)."""
    out = np.zeros((p.shape[0], x.shape[1]))
    for i in range(p.shape[0]):
        out[i] = p[i, seen[i]] @ x[seen[i]]
    return out


def attention(q, k, v, dy, heads, kv, causal, window, starts):
    """y, dq, dk, dv by their formulas, row by row."""
    out = [np.zeros_like(t) for t in (q, q, k, v)]
    width, group = q.shape[1] // heads, heads // kv
    for a, b in zip(starts[:-1], starts[1:]):
        i = np.arange(b - a)
        seen = np.ones((b - a, b - a), bool)
        if causal:
            seen &= i[:, None] >= i
        if window:
            seen &= i[:, None] - i < window
        for h in range(heads if b > a else 0):
            mine, theirs = slice(h * width, (h + 1) * width), slice(h // group * width, (h // group + 1) * width)
            Q, K, V, D = q[a:b, mine], k[a:b, theirs], v[a:b, theirs], dy[a:b, mine]
            x = np.where(seen, Q @ K.T / np.sqrt(width), -np.inf)
            e = np.exp(x - x.max(axis=1, keepdims=True))
            p = e / e.sum(axis=1, keepdims=True)
            y = over_seen(p, V, seen)
            ds = p * (D @ V.T - (D * y).sum(axis=1, keepdims=True)) / np.sqrt(width)
            out[0][a:b, mine] = y
            out[1][a:b, mine] = over_seen(ds, K, seen)
            out[2][a:b, theirs] += over_seen(ds.T, Q, seen.T)
            out[3][a:b, theirs] += over_seen(p.T, D, seen.T)
    return out


# (a NaN in q or k takes its rows with it; an infinity in v or dy stays in its column until the gradient spreads it)
@pytest.mark.parametrize("rows,heads,kv,width,causal,window,starts", [
    (333, 4, 2, 72, 1, 0, None), (300, 2, 1, 64, 1, 60, None), (260, 3, 1, 128, 0, 0, None), (290, 6, 2, 40, 1, 0, [3, 130, 131, 131, 280]), (1500, 1, 1, 64, 1, 0, None),
    (200, 2, 2, 8, 1, 33, None)])
@pytest.mark.parametrize("where,bad", [("q", np.nan), ("k", np.nan), ("v", np.inf), ("v", -np.inf), ("dy", np.inf), ("dy", np.nan)])
def test_what_is_not_finite_goes_where_the_formula_takes_it(rows, heads, kv, width, causal, window, starts, where, bad):
    g, ids, inputs, outputs = attention_graph(rows, heads, kv, width, causal, window, starts=len(starts) - 1 if starts else 0, grad=True)
    feeds = attention_feeds(g, inputs, rows, starts)
    clean, bounds = interp.run_function(g.desc, inputs, outputs, feeds), attention_bounds(g, inputs, outputs, feeds)
    names = [g.desc["tensors"][t]["name"] for t in inputs]
    spoil(feeds[names.index(where)], bad, rows + width)
    got, _ = run_gpu(g.desc, inputs, outputs, feeds)
    with np.errstate(invalid="ignore"):
        want = attention(*(feeds[names.index(n)] for n in ("q", "k", "v", "dy")), heads, kv, causal, window, starts or [0, rows])
    for n, a, w, c in zip(("y", "dq", "dk", "dv"), got, want, clean):
        compare(n, a, w, c, bounds[n])


@pytest.mark.parametrize("heads,kv,width,page,window,new,lengths", [
    (4, 2, 72, 16, 0, [1, 1], [300, 77]), (8, 1, 128, 32, 0, [1], [3000]), (2, 1, 64, 16, 50, [40, 40], [60, 500]), (4, 2, 64, 64, 0, [90, 90], [90, 2500])])
@pytest.mark.parametrize("where,bad", [("q", np.nan), ("kc", np.nan), ("vc", np.inf)])
def test_what_is_not_finite_in_a_cache(heads, kv, width, page, window, new, lengths, where, bad):
    pool, most = sum(-(-n // page) for n in lengths) + 1, -(-max(lengths) // page)
    g, ids, inputs, outputs = paged_graph(sum(new), len(new), heads, kv, width, page, most, pool, window, write=False)
    feeds = paged_feeds(g, inputs, heads + width, lengths, page, pool)
    clean, bound = interp.run_function(g.desc, inputs, outputs, feeds), paged_bounds(g, inputs, outputs, feeds)
    names = [g.desc["tensors"][t]["name"] for t in inputs]
    spoil(feeds[names.index(where)], bad, width)
    got, _ = run_gpu(g.desc, inputs, outputs, feeds)
    with np.errstate(invalid="ignore"):
        want = interp.run_function(g.desc, inputs, outputs, feeds)
    compare("y", got[0], want[0], clean[0], bound)


@pytest.mark.parametrize("where", ["v", "dy"])
def test_one_infinity_in_a_long_sequence_ends_soon(where):
    """Nearly every row or key is computed a second time then, over all that it sees: 32 at a time, not one by one (1374 ms)."""
    import torch
    g, ids, inputs, outputs = attention_graph(16384, 8, 2, 128, grad=True)
    gen = torch.Generator(device="cuda").manual_seed(8)
    dev = [torch.randn(g.shape(t), generator=gen, device="cuda").to(torch.bfloat16) for t in inputs]
    dev[inputs.index(ids[where])][0 if where == "v" else -1, 0] = float("inf")
    outs = [torch.zeros(g.shape(t), dtype=torch.bfloat16, device="cuda") for t in outputs]
    f = B.Graph.from_desc(g.desc).function(inputs, outputs)
    f.run_torch(dev, outs)
    start, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    start.record()
    f.run_torch(dev, outs)
    end.record()
    torch.cuda.synchronize()
    assert f.status() == 0 and not bool(torch.isfinite(outs[2]).all())
    assert start.elapsed_time(end) < 300
