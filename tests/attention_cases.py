"""Shared by the tests of the attention operators: graphs, seeded inputs, and error bounds derived from the roundings."""
import numpy as np

from lm_cases import U16, U32, as_type
from oracle import interp
from paper_1707_08265_b200 import workloads as wl

HALF = {"f32": U32, "bf16": U16}


def head_graph(rows, heads, width, dims=None, interleaved=0, norm=True, numbers=(), x="bf16", u="f32", y="bf16", gain="f32", grad=False, dy=None,
               grad_types=None, fetch_u=False, rotate=True):
    g = wl.GraphDesc()
    shape = [rows, heads * width]
    ids = {"x": g.tensor("x", shape, x)}
    inputs, last = [ids["x"]], ids["x"]
    if norm:
        ids["gain"] = g.tensor("gain", [width], gain)
        inputs.append(ids["gain"])
        ids["u"] = last = g.op("HeadNorm", [last, ids["gain"]], "u", shape, u if rotate else y, attrs=[1e-5])
    if rotate:
        ids["pos"] = g.tensor("pos", [rows], "i32")
        inputs.append(ids["pos"])
        last = g.op("Rotate", [last, ids["pos"]], "y", shape, y, attrs=[heads, dims or width, interleaved] + list(numbers))
    ids["y"] = last
    outputs = ([ids["u"]] if fetch_u else []) + [last]
    if grad:
        ids["dy"] = g.tensor("dy", shape, dy or y)
        obj = g.op("Mul", [last, ids["dy"]], "along")
        wrts = [ids["x"]] + ([ids["gain"]] if norm else [])
        outputs += g.grad([obj], wrts, grad_types)
        inputs.append(ids["dy"])
    return g, ids, inputs, outputs


def head_feeds(g, inputs, seed, far=5000):
    rng = np.random.default_rng(seed)
    out = []
    for t in inputs:
        info = g.desc["tensors"][t]
        if info["dtype"] == "i32":
            out.append(rng.integers(-far, far, info["shape"]).astype(np.int32))
        else:
            out.append(as_type(rng.standard_normal(info["shape"]) * (0.3 if info["name"] == "gain" else 1.5) + (info["name"] == "gain"), info["dtype"]))
    return out


def head_bounds(g, inputs, outputs, feeds):
    """fp32 evaluation: the head's sum of squares is off by (width / 8 + 8) 2^-24, the root by 2 more, each product by one, an angle
    by 2^-25 turns (pi 2^-24 radians) and its sine and cosine by two units, 4 * 2^-24; then half a step of the result's type.
    A sum over rows and heads is off by its length times 2^-24 of its magnitudes at most."""
    desc, val = g.desc, {t: f for t, f in zip(inputs, feeds)}
    ops = {op["type"]: op for op in desc["ops"]}
    by = {desc["tensors"][t]["name"]: f for t, f in zip(inputs, feeds)}
    x = by["x"]
    width = by["gain"].shape[0] if "gain" in by else None
    if width:
        h = x.reshape(x.shape[0], -1, width)
        inv = 1 / np.sqrt((h ** 2).mean(-1, keepdims=True) + 1e-5)
        u = h * inv * by["gain"]
        eu = np.abs(u) * (width / 8 + 14) * U32
        if desc["tensors"][ops["HeadNorm"]["out"][0]]["dtype"] == "bf16" and "Rotate" in ops:
            eu = eu + 2 * np.abs(u) * U16          # rounded in front of the rotation, and here and in the oracle perhaps to different sides
        u, eu = u.reshape(x.shape), eu.reshape(x.shape)
    else:
        u, eu = x, np.zeros_like(x)

    def turned(m, e):          # bound of the rotation of values of magnitude m with errors e
        if "Rotate" not in ops:
            return e
        op = ops["Rotate"]
        c, s, first, second = interp.rotation(op, x.shape[1], by["pos"])
        amp = abs(interp._numbers(op, [1, 0, 0, 1e4, 1, 0, 0, 0, 1.0])[8])
        m, e = (a.reshape(x.shape[0], int(op["attrs"][0]), -1) for a in (m, e))
        out = e.copy()
        both = amp * (m[..., first] + m[..., second]) * 10 * U32
        out[..., first] = out[..., second] = amp * (e[..., first] + e[..., second]) + both
        return out.reshape(x.shape)

    bounds = {"y": turned(np.abs(u), eu), "u": eu}
    if "dy" in by:
        d = np.abs(by["dy"])
        ed = turned(d, np.zeros_like(d))
        amp = abs(interp._numbers(ops["Rotate"], [1, 0, 0, 1e4, 1, 0, 0, 0, 1.0])[8]) if "Rotate" in ops else 1.0
        md = (turned(d, d) - ed + d) if "Rotate" in ops else d           # magnitude of the turned gradient (both parts of a pair)
        md = np.maximum(md, amp * d)
        if width:
            shape = h.shape
            md, ed = md.reshape(shape), ed.reshape(shape)
            gain = np.abs(by["gain"])
            n = h.shape[0] * h.shape[1]
            rel = (width / 8 + 24) * U32
            t, et = md * gain, ed * gain
            mean = (t * np.abs(h)).mean(-1, keepdims=True)
            emean = (et * np.abs(h)).mean(-1, keepdims=True)
            bounds["dx"] = (inv * (et + rel * t) + np.abs(h) * inv ** 3 * (emean + 3 * rel * mean)).reshape(x.shape)
            bounds["dgain"] = ((ed + md * (rel + n * U32)) * np.abs(h) * inv).sum((0, 1))
        else:
            bounds["dx"] = ed
    return bounds


def attention_graph(rows, heads, kv_heads, width, causal=1, window=0, scale=0.0, sequences=1, starts=0, q="bf16", k="bf16", v="bf16", y="bf16", grad=False,
                    dy=None, grad_types=("bf16", "bf16", "bf16")):
    """starts: the number of packed sequences, 0 for none."""
    g = wl.GraphDesc()
    ids = {"q": g.tensor("q", [rows, heads * width], q), "k": g.tensor("k", [rows, kv_heads * width], k), "v": g.tensor("v", [rows, kv_heads * width], v)}
    ins = [ids["q"], ids["k"], ids["v"]]
    if starts:
        ids["starts"] = g.tensor("starts", [starts + 1], "i32")
        ins.append(ids["starts"])
    ids["y"] = g.op("Attention", ins, "y", [rows, heads * width], y, attrs=[heads, kv_heads, causal, window, scale, sequences])
    inputs, outputs = list(ins), [ids["y"]]
    if grad:
        ids["dy"] = g.tensor("dy", [rows, heads * width], dy or y)
        obj = g.op("Mul", [ids["y"], ids["dy"]], "along")
        outputs += g.grad([obj], ins[:3], grad_types)
        inputs.append(ids["dy"])
    return g, ids, inputs, outputs


def attention_feeds(g, inputs, seed, starts=None, scale=1.0):
    rng = np.random.default_rng(seed)
    out = []
    for t in inputs:
        info = g.desc["tensors"][t]
        out.append(np.asarray(starts, np.int32) if info["dtype"] == "i32" else as_type(rng.standard_normal(info["shape"]) * (scale if info["name"] in "qk" else 1.0), info["dtype"]))
    return out


def attention_bounds(g, inputs, outputs, feeds):
    """Bounds of y, dq, dk, dv.  A score is off by (width + 4) 2^-24 of the sum of its products' magnitudes (fp32 sums in any
    order; twice that, for the maximum's and the sum's own score), so a probability by that much of itself plus 16 units of
    2^-24 for the exponentials and their sum; it is rounded to bf16 for its product (2^-8 of itself), and so is ds.  delta is
    taken from y as it is stored.  Then half a step of the result's type."""
    desc = g.desc
    by = {desc["tensors"][t]["name"]: f for t, f in zip(inputs, feeds)}
    op = next(o for o in desc["ops"] if o["type"] == "Attention")
    q, k, v = (interp.round_bf16(by[n]) for n in ("q", "k", "v"))
    ins = [q, k, v] + ([by["starts"]] if "starts" in by else [])
    B = {"y": np.zeros_like(q), "dq": np.zeros_like(q), "dk": np.zeros_like(k), "dv": np.zeros_like(v)}
    uy = HALF[desc["tensors"][op["out"][0]]["dtype"]]
    for rows, mine, theirs, p, scale in interp.attention_parts(op, ins):
        if rows.stop <= rows.start:
            continue
        width = mine.stop - mine.start
        es = 2 * scale * (width + 4) * U32 * (np.abs(q[rows, mine]) @ np.abs(k[rows, theirs]).T).max() + 16 * U32
        ep = p * (es + U16)
        n = p.shape[0]
        B["y"][rows, mine] = ep @ np.abs(v[rows, theirs]) + (p @ np.abs(v[rows, theirs])) * n * U32
        if "dy" in by:
            do, y = interp.round_bf16(by["dy"])[rows, mine], p @ v[rows, theirs]
            dp = do @ v[rows, theirs].T
            mdp = np.abs(do) @ np.abs(v[rows, theirs]).T
            delta = (np.abs(y) * np.abs(do)).sum(1, keepdims=True)
            ds = p * np.abs(dp - (y * do).sum(1, keepdims=True))
            edelta = uy * delta + (np.abs(do) * B["y"][rows, mine]).sum(1, keepdims=True) + width * U32 * delta
            eds = ds * (es + 2 * U16) + p * (edelta + (width + 8) * U32 * mdp)
            B["dq"][rows, mine] = scale * ((eds + n * U32 * ds) @ np.abs(k[rows, theirs]))
            B["dk"][rows, theirs] += scale * ((eds + n * U32 * ds).T @ np.abs(q[rows, mine]))
            B["dv"][rows, theirs] += (ep + n * U32 * p).T @ np.abs(do)
    return B


def within(got, want, bound, dtype):
    """Largest excess of |got - want| over the bound plus half a step of the type (a result that rounds to the other side of a
    midpoint is another half step off), as a share of it."""
    room = bound * (1 + 2 * HALF[dtype]) + 2 * HALF[dtype] * np.abs(want) + 1e-30
    assert np.isfinite(got).all()
    return float(np.max(np.abs(got - want) / room)) if got.size else 0.0


def paged_graph(rows, sequences, heads, kv_heads, width, page, most, pool, window=0, scale=0.0, starts=False, write=True, q="bf16", y="bf16"):
    g = wl.GraphDesc()
    ids = {"q": g.tensor("q", [rows, heads * width], q)}
    cols = kv_heads * width
    for n in ("kc", "vc"):
        ids[n] = g.tensor(n, [pool * page, cols], "bf16")
    ids["pages"], ids["lengths"] = g.tensor("pages", [sequences, most], "i32"), g.tensor("lengths", [sequences], "i32")
    table = [ids["pages"], ids["lengths"]]
    if starts:
        ids["starts"] = g.tensor("starts", [sequences + 1], "i32")
        table.append(ids["starts"])
    inputs, kc, vc, outputs = [ids["q"], ids["kc"], ids["vc"]] + table, ids["kc"], ids["vc"], []
    if write:
        ids["k"], ids["v"] = g.tensor("k", [rows, cols], "bf16"), g.tensor("v", [rows, cols], "bf16")
        inputs += [ids["k"], ids["v"]]
        kc = g.op("CacheWrite", [kc, ids["k"]] + table, "kc2", [pool * page, cols], "bf16", attrs=[page])
        vc = g.op("CacheWrite", [vc, ids["v"]] + table, "vc2", [pool * page, cols], "bf16", attrs=[page])
        outputs = [kc, vc]
    ids["y"] = g.op("PagedAttention", [ids["q"], kc, vc] + table, "y", [rows, heads * width], y, attrs=[heads, kv_heads, page, window, scale])
    return g, ids, inputs, [ids["y"]] + outputs


def paged_feeds(g, inputs, seed, lengths, page, pool, starts=None):
    """Every sequence has pages of its own, handed out in a random order; entries behind its last page hold numbers of no page."""
    rng = np.random.default_rng(seed)
    order = list(rng.permutation(pool))
    out = []
    for t in inputs:
        info = g.desc["tensors"][t]
        if info["name"] == "pages":
            a = np.full(info["shape"], -7, np.int32)
            for s, n in enumerate(lengths):
                for j in range(min(-(-max(n, 0) // page), info["shape"][1])):
                    a[s, j] = order.pop()
            out.append(a)
        elif info["name"] in ("lengths", "starts"):
            out.append(np.asarray(lengths if info["name"] == "lengths" else starts, np.int32))
        else:
            out.append(as_type(rng.standard_normal(info["shape"]), info["dtype"]))
    return out


def paged_bounds(g, inputs, outputs, feeds):
    """The bound of y as in attention_bounds."""
    desc = g.desc
    by = {desc["tensors"][t]["name"]: f for t, f in zip(inputs, feeds)}
    op = next(o for o in desc["ops"] if o["type"] == "PagedAttention")
    writes = [o for o in desc["ops"] if o["type"] == "CacheWrite"]
    table = [by["pages"], by["lengths"]] + ([by["starts"]] if "starts" in by else [])
    kc, vc = by["kc"], by["vc"]
    if writes:
        kc, vc = (interp._forward(writes[0], [c, r] + table, np.float64) for c, r in ((kc, by["k"]), (vc, by["v"])))
    q = interp.round_bf16(by["q"])
    B = np.zeros_like(q)
    for r, mine, theirs, at, p in interp.paged_parts(op, [q, kc, vc] + table):
        width = mine.stop - mine.start
        scale = interp._numbers(op, [1, 0, 16, 0, 0.0])[4] or 1 / np.sqrt(width)
        es = 2 * scale * (width + 4) * U32 * (np.abs(kc[at, theirs]) @ np.abs(q[r, mine])).max() + 16 * U32
        B[r, mine] = (p * (es + U16 + len(p) * U32)) @ np.abs(vc[at, theirs])
    return B
