"""Measured cases of the attention operators: what one pass computes, in plain torch and through the library.

Operators (operator types of the graph, see include/dragon.h):
  HeadNorm, Rotate         every head of a row over its root mean square, and its rotation by the row's position, with gradients
  Attention                softmax(scale q k^T) v over packed sequences: causal, windowed or over all rows, heads of queries that
                           share heads of keys, with the gradients of q, k and v
  CacheWrite               rows of new tokens written to their places in a cache of pages, in place
  PagedAttention           attention of the new rows of every sequence over its pages

``own`` false: elementary torch operations in 32 bits (64 for the angles of far positions).  ``own`` true: the library's
functions, compiled once per shape as a user's program keeps them, run on the state's buffers.
"""
import functools
import math
import random

import torch

own = False

EPS = 1e-6
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


# ---- cases ------------------------------------------------------------------------------------------------

def listed():
    return [
        # one decoding step's queries and keys of 16 sequences, far into a long context
        {"name": "rotate_token", "op": "rotate", "rows": 16, "heads": 32, "kv_heads": 8, "dim": 128, "rotated": 128, "interleaved": False, "scaled": True,
         "norm": True, "dtype": "bf16", "train": False},
        # a training step's queries and keys, forward and gradients, at the benchmark MLP's activation size
        {"name": "rotate_train", "op": "rotate", "rows": 8192, "heads": 32, "kv_heads": 8, "dim": 128, "rotated": 128, "interleaved": False, "scaled": False,
         "norm": True, "dtype": "bf16", "train": True},
        # a ragged prompt in 32 bits, neighbouring pairs, only part of every head rotated, no norm
        {"name": "rotate_ragged", "op": "rotate", "rows": 4099, "heads": 13, "kv_heads": 13, "dim": 80, "rotated": 48, "interleaved": True, "scaled": False,
         "norm": False, "dtype": "f32", "train": False},
        # short packed documents in training
        {"name": "attend_packed", "op": "attend", "seqs": 9, "length": 300, "ragged": True, "heads": 8, "kv_heads": 2, "dim": 64, "causal": True, "window": 0, "train": True},
        # an ordinary training step: four sequences, query heads that share key heads
        {"name": "attend_train", "op": "attend", "seqs": 4, "length": 2048, "ragged": False, "heads": 32, "kv_heads": 8, "dim": 128, "causal": True, "window": 0, "train": True},
        # one long sequence in training
        {"name": "attend_long", "op": "attend", "seqs": 1, "length": 16384, "ragged": False, "heads": 8, "kv_heads": 2, "dim": 128, "causal": True, "window": 0, "train": True},
        # a long prompt under a window, odd length, a head width that is no power of two
        {"name": "attend_window", "op": "attend", "seqs": 1, "length": 12001, "ragged": False, "heads": 6, "kv_heads": 6, "dim": 96, "causal": True, "window": 1024, "train": False},
        # every row sees every row of its sequence (an encoder's batch)
        {"name": "attend_full", "op": "attend", "seqs": 16, "length": 1000, "ragged": True, "heads": 16, "kv_heads": 16, "dim": 64, "causal": False, "window": 0, "train": False},
        # decoding a few short sequences: the launches are what counts
        {"name": "serve_small", "op": "serve", "seqs": 3, "new": 1, "ragged": False, "context": 200, "heads": 16, "kv_heads": 4, "dim": 64, "page": 16, "window": 0},
        # decoding a full batch: the cache's bytes are what counts
        {"name": "serve_batch", "op": "serve", "seqs": 64, "new": 1, "ragged": False, "context": 4000, "heads": 32, "kv_heads": 8, "dim": 128, "page": 16, "window": 0},
        # decoding one sequence of a very long context: the work has to be split along it
        {"name": "serve_one", "op": "serve", "seqs": 1, "new": 1, "ragged": False, "context": 100000, "heads": 32, "kv_heads": 8, "dim": 128, "page": 64, "window": 0},
        # a chunk of a prompt for some sequences beside single tokens for the others
        {"name": "serve_chunk", "op": "serve", "seqs": 6, "new": 1500, "ragged": True, "context": 8000, "heads": 16, "kv_heads": 4, "dim": 128, "page": 32, "window": 0},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rotate", "rotate", "attend", "attend", "attend", "serve", "serve", "serve"])
    if op == "rotate":
        kv = _log(rng, 1, 16)
        heads, dim = kv * rng.choice([1, 1, 2, 4]), rng.choice([32, 40, 64, 80, 96, 128, 128, 256])
        rotated = dim if rng.random() < 0.6 else max(2, rng.randint(1, dim // 2) * 2)
        return {"op": op, "rows": max(1, min(_log(rng, 1, 16384), 33554432 // (heads * dim))), "heads": heads, "kv_heads": kv, "dim": dim, "rotated": rotated,
                "interleaved": rng.random() < 0.4, "scaled": rng.random() < 0.4, "norm": rng.random() < 0.6, "dtype": rng.choice(["bf16", "bf16", "f32"]),
                "train": rng.random() < 0.5}
    kv, group, dim = _log(rng, 1, 8), rng.choice([1, 1, 2, 3, 4, 8]), rng.choice([32, 64, 64, 72, 80, 96, 128, 128, 128])
    if op == "attend":
        causal = rng.random() < 0.75
        window = _log(rng, 16, 4096) if causal and rng.random() < 0.35 else 0
        length = _log(rng, 1, 16384)
        length = min(length, int(math.sqrt(2.0 ** 31 / (kv * group))))
        seqs = max(1, min(_log(rng, 1, 32), 2 ** 31 // (length * length * kv * group), 65536 // length))
        return {"op": op, "seqs": seqs, "length": length, "ragged": rng.random() < 0.4, "heads": kv * group, "kv_heads": kv, "dim": dim,
                "causal": causal, "window": window, "train": rng.random() < 0.6}
    context, new = _log(rng, 1, 100000), 1 if rng.random() < 0.5 else _log(rng, 2, 2000)
    context = min(context, 2 ** 29 // (new * kv * group))
    seqs = max(1, min(_log(rng, 1, 128), 2 ** 28 // ((context + new) * kv * dim), 2 ** 31 // (new * (context + new) * kv * group)))
    return {"op": op, "seqs": seqs, "new": new, "ragged": new > 1 and rng.random() < 0.5, "context": context, "heads": kv * group, "kv_heads": kv, "dim": dim,
            "page": rng.choice([16, 16, 32, 64, 128, 256]), "window": _log(rng, 16, 8192) if rng.random() < 0.2 else 0}


def _lengths(c):
    """Rows of every sequence of an attention case."""
    if not c["ragged"]:
        return [c["length"]] * c["seqs"]
    rng = random.Random(c["length"] * 131 + c["seqs"])
    return [rng.randint(1, c["length"]) for _ in range(c["seqs"] - 1)] + [c["length"]]


def _rows_and_totals(c):
    """New rows and total length of every sequence of a serving case; ragged ones: half of the sequences have a single new row."""
    rng = random.Random(c["context"] * 131 + c["seqs"])
    new = [c["new"]] * c["seqs"]
    if c["ragged"]:
        new = [1 if s % 2 else max(1, rng.randint(c["new"] // 2, c["new"])) for s in range(c["seqs"])]
    before = [rng.randint(c["context"] // 2, c["context"]) for _ in range(c["seqs"])]
    return new, [a + b for a, b in zip(new, before)]


# ---- inputs -----------------------------------------------------------------------------------------------

def _starts(lengths):
    out = [0]
    for n in lengths:
        out.append(out[-1] + n)
    return out


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, dtype=torch.float32, scale=1.0, shift=0.0):
        return torch.empty(shape, device="cuda").normal_(shift, scale, generator=gen).to(dtype)

    def ints(values, *shape):
        return torch.tensor(values, dtype=torch.int32).reshape(shape or (len(values),)).cuda()

    c, s, op = dict(case), {"case": dict(case)}, case["op"]
    H, G, D = c["heads"], c["kv_heads"], c["dim"]
    if op == "rotate":
        R, dt = c["rows"], DT[c["dtype"]]
        far = 131072 if c["scaled"] else 8192                    # sequences packed one after another, each with positions of its own
        s["pos"] = ((torch.arange(R, device="cuda") * (1 if R > 64 else 977) + torch.randint(0, far, (1,), device="cuda", generator=gen)) % far).to(torch.int32)
        for n, heads in (("q", H), ("k", G)):
            s[n] = normal(R, heads * D, dtype=dt, scale=1.5)
            s["y" + n] = torch.empty_like(s[n])
            if c["norm"]:
                s["gain" + n] = normal(D, scale=0.2, shift=1.0)
            if c["train"]:
                s["dy" + n] = normal(R, heads * D, dtype=dt)
                s["d" + n] = torch.empty_like(s[n])
                if c["norm"]:
                    s["dgain" + n] = torch.empty(D, device="cuda")
    elif op == "attend":
        lengths = _lengths(c)
        T = sum(lengths)
        s["starts"] = ints(_starts(lengths)) if c["ragged"] else None
        for n, heads in (("q", H), ("k", G), ("v", G)):          # queries and keys as large as a norm leaves them
            s[n] = normal(T, heads * D, dtype=torch.bfloat16)
        s["y"] = torch.empty_like(s["q"])
        if c["train"]:
            s["dy"] = normal(T, H * D, dtype=torch.bfloat16)
            for n in ("q", "k", "v"):
                s["d" + n] = torch.empty_like(s[n])
    elif op == "serve":
        new, total = _rows_and_totals(c)
        page = c["page"]
        per = [-(-n // page) for n in total]
        P, pool = max(per), sum(per) + 3
        order = torch.randperm(pool, device="cuda", generator=gen).to(torch.int32)      # pages as a running server has handed them out
        at = torch.arange(P, device="cuda")[None] + torch.tensor(_starts(per)[:-1]).cuda()[:, None]
        s["pages"] = torch.where(torch.arange(P, device="cuda")[None] < torch.tensor(per).cuda()[:, None], order[at.clamp(max=pool - 1)], 0).to(torch.int32).contiguous()
        s["lengths"] = ints(total)
        s["starts"] = ints(_starts(new)) if c["ragged"] else None
        T = sum(new)
        s["q"], s["k"], s["v"] = (normal(T, h * D, dtype=torch.bfloat16) for h in (H, G, G))
        s["kc"], s["vc"] = (normal(pool * page, G * D, dtype=torch.bfloat16) for _ in range(2))
        s["y"] = torch.empty_like(s["q"])
    else:
        raise ValueError(op)
    return s


# ---- the plain forms --------------------------------------------------------------------------------------

def _frequencies(c, device):
    """Radians per position of every rotated pair, in 64 bits; scaled: slow pairs by 1/8, fast ones kept, a ramp between them."""
    n = c["rotated"]
    f = 500000.0 ** (-torch.arange(0, n, 2, device=device, dtype=torch.float64) / n)
    if not c["scaled"]:
        return f
    keep = ((f * (8192 / (2 * math.pi)) - 1.0) / (4.0 - 1.0)).clamp(0, 1)
    return f * (keep + (1 - keep) / 8)


def _turn(x, cos, sin, c):
    """x [rows, heads, dim] rotated."""
    n = c["rotated"]
    a, b = (x[..., 0:n:2], x[..., 1:n:2]) if c["interleaved"] else (x[..., :n // 2], x[..., n // 2:n])
    ra, rb = a * cos - b * sin, b * cos + a * sin
    r = torch.stack([ra, rb], -1).flatten(-2) if c["interleaved"] else torch.cat([ra, rb], -1)
    return torch.cat([r, x[..., n:]], -1)


def _plain_rotate_one(s, n, heads, cos, sin):
    c = s["case"]
    R, D = c["rows"], c["dim"]
    x = s[n].float().view(R, heads, D)
    out = {}
    y = x
    if c["norm"]:
        inv = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
        y = x * inv * s["gain" + n]
    out["y" + n] = _turn(y, cos, sin, c).to(s[n].dtype).view(R, heads * D)
    if c["train"]:
        d = _turn(s["dy" + n].float().view(R, heads, D), cos, -sin, c)
        if c["norm"]:
            u = x * inv
            out["dgain" + n] = (d * u).sum((0, 1))
            d = d * s["gain" + n]
            d = inv * (d - u * (d * u).mean(-1, keepdim=True))
        out["d" + n] = d.to(s[n].dtype).view(R, heads * D)
    return out


def _plain_rotate(s):
    c = s["case"]
    angle = s["pos"].double()[:, None] * _frequencies(c, s["pos"].device)[None]
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    return {**_plain_rotate_one(s, "q", c["heads"], cos, sin), **_plain_rotate_one(s, "k", c["kv_heads"], cos, sin)}


def _padded(t, at, heads):
    """Rows of a packed tensor as [sequences, key heads, rows (of every query head of the group), width]; at: row numbers [sequences, rows]."""
    S, L = at.shape
    return t[at.reshape(-1)].float().view(S, L, heads, -1).transpose(1, 2)


def _softmax(scores, seen):
    scores = torch.where(seen, scores, -math.inf)
    top = scores.amax(-1, keepdim=True)
    e = torch.exp(scores - torch.where(torch.isinf(top), 0.0, top))
    return e / e.sum(-1, keepdim=True).clamp_min(1e-30)


def _plain_attend(s):
    c = s["case"]
    H, G, D, dev = c["heads"], c["kv_heads"], c["dim"], s["q"].device
    T, S = s["q"].shape[0], c["seqs"]
    starts = s["starts"].long() if c["ragged"] else torch.arange(S + 1, device=dev) * c["length"]
    n, L = starts[1:] - starts[:-1], c["length"]
    i = torch.arange(L, device=dev)
    at = (starts[:-1, None] + i).clamp(max=T - 1)
    q = _padded(s["q"], at, H).reshape(S, G, H // G, L, D)
    k, v = _padded(s["k"], at, G)[:, :, None], _padded(s["v"], at, G)[:, :, None]
    seen = (i[None] < n[:, None])[:, None, None, None, :]
    if c["causal"]:
        seen = seen & (i[None] <= i[:, None])
    if c["window"]:
        seen = seen & (i[:, None] - i[None] < c["window"])
    scale = 1 / math.sqrt(D)
    p = _softmax(torch.matmul(q, k.transpose(-1, -2)).mul_(scale), seen)
    y = torch.matmul(p, v)
    mine = (i[None] < n[:, None])                                # rows that exist

    def packed(t):                                               # [S, heads, L, D] -> [T, heads * D]
        return t.transpose(1, 2).reshape(S, L, -1)[mine].to(torch.bfloat16)

    out = {"y": packed(y.view(S, H, L, D))}
    if c["train"]:
        dy = (_padded(s["dy"], at, H) * mine[:, None, :, None]).view(S, G, H // G, L, D)
        dp = torch.matmul(dy, v.transpose(-1, -2))
        out["dv"] = packed(torch.matmul(p.transpose(-1, -2), dy).sum(2))
        ds = dp.sub_((dy * y).sum(-1, keepdim=True)).mul_(p).mul_(scale)
        out["dq"] = packed(torch.matmul(ds, k).view(S, H, L, D))
        out["dk"] = packed(torch.matmul(ds.transpose(-1, -2), q).sum(2))
    return out


def _plain_serve(s):
    c = s["case"]
    H, G, D, page, dev = c["heads"], c["kv_heads"], c["dim"], c["page"], s["q"].device
    T, S = s["q"].shape[0], c["seqs"]
    total = s["lengths"].long()
    starts = s["starts"].long() if c["ragged"] else torch.arange(S + 1, device=dev) * c["new"]
    n = starts[1:] - starts[:-1]
    row = torch.arange(T, device=dev)
    seq = torch.searchsorted(starts[1:].contiguous(), row, right=True)
    pos = total[seq] - n[seq] + row - starts[seq]
    slot = s["pages"].long()[seq, pos // page] * page + pos % page
    s["kc"][slot], s["vc"][slot] = s["k"], s["v"]
    most, L = c["new"], c["page"] * s["pages"].shape[1]
    i, j = torch.arange(most, device=dev), torch.arange(L, device=dev)
    q = _padded(s["q"], (starts[:-1, None] + i).clamp(max=T - 1), H).reshape(S, G, (H // G) * most, D)
    where = s["pages"].long()[:, j // page] * page + j % page
    k, v = _padded(s["kc"], where, G), _padded(s["vc"], where, G)
    mine = total[:, None] - n[:, None] + i                       # position of every new row
    seen = j <= mine[..., None]
    if c["window"]:
        seen = seen & (mine[..., None] - j < c["window"])
    scores = torch.matmul(q, k.transpose(-1, -2)).view(S, G, H // G, most, L).mul_(1 / math.sqrt(D))
    p = _softmax(scores, seen[:, None, None]).view(S, G, (H // G) * most, L)
    y = torch.matmul(p, v).view(S, H, most, D).transpose(1, 2).reshape(S, most, H * D)
    return {"y": y[i[None] < n[:, None]].to(torch.bfloat16), "kc": s["kc"], "vc": s["vc"]}


# ---- the library's calls ----------------------------------------------------------------------------------

@functools.lru_cache(maxsize=None)
def _rotate_function(rows, heads, kv_heads, dim, rotated, interleaved, scaled, norm, dtype, train):
    from paper_1707_08265_b200 import binding as B
    g, dt = B.Graph(), B.DTYPES[dtype]
    pos = g.add_tensor("positions", B.I32, [rows])
    ins, outs, along, wrts, types = [pos], [], [], [], []
    for n, h in (("q", heads), ("k", kv_heads)):
        shape = [rows, h * dim]
        x = g.add_tensor(n, dt, shape)
        y = g.add_tensor("y" + n, dt, shape)
        ins.append(x)
        wrts.append(x)
        types.append(dt)
        if norm:
            gain, u = g.add_tensor("gain" + n, B.F32, [dim]), g.add_tensor("normed" + n, B.F32, shape)
            g.add_op(B.OPS["HeadNorm"], [x, gain], [u], [EPS])
            ins.append(gain)
            wrts.append(gain)
            types.append(B.F32)
            x = u
        g.add_op(B.OPS["Rotate"], [x, pos], [y], [h, rotated, int(interleaved), 500000.0] + ([8.0, 1.0, 4.0, 8192.0] if scaled else []))
        outs.append(y)
    if not train:
        return g.function(ins, outs)
    for n, h, y in (("q", heads, outs[0]), ("k", kv_heads, outs[1])):
        dy, a = g.add_tensor("dy" + n, dt, [rows, h * dim]), g.add_tensor("along" + n, B.F32, [rows, h * dim])
        g.add_op(B.OPS["Mul"], [y, dy], [a])                      # an objective whose gradient is dy
        ins.append(dy)
        along.append(a)
    return g.function(ins, outs + g.add_grad(along, wrts, types))


@functools.lru_cache(maxsize=None)
def _attend_function(rows, seqs, ragged, heads, kv_heads, dim, causal, window, train):
    from paper_1707_08265_b200 import binding as B
    g = B.Graph()
    q, k, v, y = (g.add_tensor(n, B.BF16, [rows, h * dim]) for n, h in (("q", heads), ("k", kv_heads), ("v", kv_heads), ("y", heads)))
    ins = [q, k, v] + ([g.add_tensor("starts", B.I32, [seqs + 1])] if ragged else [])
    g.add_op(B.OPS["Attention"], ins, [y], [heads, kv_heads, int(causal), window, 0.0, 1 if ragged else seqs])
    if not train:
        return g.function(ins, [y])
    dy, along = g.add_tensor("dy", B.BF16, [rows, heads * dim]), g.add_tensor("along", B.F32, [rows, heads * dim])
    g.add_op(B.OPS["Mul"], [y, dy], [along])
    return g.function(ins + [dy], [y] + g.add_grad([along], [q, k, v], [B.BF16] * 3))


@functools.lru_cache(maxsize=None)
def _serve_function(rows, seqs, ragged, pool, most_pages, heads, kv_heads, dim, page, window):
    from paper_1707_08265_b200 import binding as B
    g = B.Graph()
    q, k, v, y = (g.add_tensor(n, B.BF16, [rows, h * dim]) for n, h in (("q", heads), ("k", kv_heads), ("v", kv_heads), ("y", heads)))
    kc, vc, kc2, vc2 = (g.add_tensor(n, B.BF16, [pool, kv_heads * dim]) for n in ("kc", "vc", "kc_new", "vc_new"))
    table = [g.add_tensor("pages", B.I32, [seqs, most_pages]), g.add_tensor("lengths", B.I32, [seqs])]
    if ragged:
        table.append(g.add_tensor("starts", B.I32, [seqs + 1]))
    g.add_op(B.OPS["CacheWrite"], [kc, k] + table, [kc2], [page])
    g.add_op(B.OPS["CacheWrite"], [vc, v] + table, [vc2], [page])
    g.add_op(B.OPS["PagedAttention"], [q, kc2, vc2] + table, [y], [heads, kv_heads, page, window])
    return g.function([q, k, v, kc, vc] + table, [y, kc2, vc2])


def _own(s):
    c = s["case"]
    op = c["op"]
    if op == "rotate":
        f = _rotate_function(c["rows"], c["heads"], c["kv_heads"], c["dim"], c["rotated"], c["interleaved"], c["scaled"], c["norm"], c["dtype"], c["train"])
        feeds, names = [s["pos"]], ["yq", "yk"]
        for n in ("q", "k"):
            feeds += [s[n]] + ([s["gain" + n]] if c["norm"] else [])
        if c["train"]:
            feeds += [s["dyq"], s["dyk"]]
            names += ["dq", "dgainq", "dk", "dgaink"] if c["norm"] else ["dq", "dk"]
        f.run_torch(feeds, [s[n] for n in names])
        return {n: s[n] for n in names}
    if op == "attend":
        f = _attend_function(s["q"].shape[0], c["seqs"], c["ragged"], c["heads"], c["kv_heads"], c["dim"], c["causal"], c["window"], c["train"])
        feeds, names = [s["q"], s["k"], s["v"]] + ([s["starts"]] if c["ragged"] else []), ["y"]
        if c["train"]:
            feeds.append(s["dy"])
            names += ["dq", "dk", "dv"]
        f.run_torch(feeds, [s[n] for n in names])
        return {n: s[n] for n in names}
    f = _serve_function(s["q"].shape[0], c["seqs"], c["ragged"], s["kc"].shape[0], s["pages"].shape[1], c["heads"], c["kv_heads"], c["dim"], c["page"], c["window"])
    f.run_torch([s["q"], s["k"], s["v"], s["kc"], s["vc"], s["pages"], s["lengths"]] + ([s["starts"]] if c["ragged"] else []), [s["y"], s["kc"], s["vc"]])
    return {"y": s["y"], "kc": s["kc"], "vc": s["vc"]}


def run(state):
    if own:
        return _own(state)
    return {"rotate": _plain_rotate, "attend": _plain_attend, "serve": _plain_serve}[state["case"]["op"]](state)


# ---- what a pass cannot do without ------------------------------------------------------------------------

def _pairs(first, rows, window):
    """Pairs (row, key it sees) of rows at positions first .. first + rows - 1 that see every key up to their own, within the window."""
    if not window:
        return rows * first + rows * (rows + 1) // 2
    short = max(0, min(rows, window - 1 - first))                # rows that see fewer than window keys
    return short * first + short * (short + 1) // 2 + (rows - short) * window


def work(case):
    c, op = case, case["op"]
    H, G, D = c["heads"], c["kv_heads"], c["dim"]
    if op == "rotate":
        n, e = c["rows"] * (H + G) * D, {"f32": 4, "bf16": 2}[c["dtype"]]
        gains = 8 * D if c["norm"] else 0
        w = {"bytes": 2 * n * e + 4 * c["rows"] + gains, "flops": (9 if c["norm"] else 3) * n}
        if c["train"]:
            w = {"bytes": w["bytes"] + 2 * n * e + gains, "flops": (22 if c["norm"] else 6) * n}
        return w
    if op == "attend":
        lengths = _lengths(c)
        T = sum(lengths)
        pairs = sum(_pairs(0, n, c["window"]) if c["causal"] else n * n for n in lengths) * H
        rows = T * (H + G) * D * 2                                # q and y's part, k and v's part: bytes of each
        return {"bytes": (4 if c["train"] else 2) * rows, "flops": (14 if c["train"] else 4) * D * pairs}
    new, total = _rows_and_totals(c)
    pairs = sum(_pairs(t - n, n, c["window"]) for n, t in zip(new, total)) * H
    seen = sum(min(t, c["window"] + n - 1) if c["window"] else t for n, t in zip(new, total))
    return {"bytes": 4 * G * D * seen + 4 * sum(new) * (H + 2 * G) * D, "flops": 4 * D * pairs}


# ---- the definition in 64 bits ----------------------------------------------------------------------------

def _exact_rotate(s, c):
    R, D, n = c["rows"], c["dim"], c["rotated"]
    out = {}
    freq = []
    for i in range(n // 2):
        f = 500000.0 ** (-2.0 * i / n)
        if c["scaled"]:
            turns = 8192.0 * f / (2 * math.pi)
            keep = min(1.0, max(0.0, (turns - 1.0) / 3.0))
            f = keep * f + (1 - keep) * f / 8.0
        freq.append(f)
    z = torch.polar(torch.ones(R, n // 2, dtype=torch.float64, device="cuda"), s["pos"].double()[:, None] * torch.tensor(freq, dtype=torch.float64, device="cuda"))
    first = torch.arange(0, n, 2) if c["interleaved"] else torch.arange(n // 2)
    second = first + 1 if c["interleaved"] else first + n // 2

    def turned(t, by):
        w = torch.complex(t[..., first], t[..., second]) * by[:, None]
        t = t.clone()
        t[..., first], t[..., second] = w.real, w.imag
        return t

    for name, heads in (("q", c["heads"]), ("k", c["kv_heads"])):
        x = s[name].double().view(R, heads, D)
        gain = s["gain" + name].double() if c["norm"] else torch.ones(D, dtype=torch.float64, device="cuda")
        rms = torch.sqrt(torch.sum(x ** 2, -1, keepdim=True) / D + EPS) if c["norm"] else torch.ones(R, heads, 1, dtype=torch.float64, device="cuda")
        out["y" + name] = turned(x / rms * gain, z).reshape(R, heads * D)
        if c["train"]:
            d = turned(s["dy" + name].double().view(R, heads, D), z.conj())
            if c["norm"]:
                out["dgain" + name] = torch.sum(d * x / rms, (0, 1))
                d = d * gain
                d = d / rms - x * torch.sum(d * x, -1, keepdim=True) / (D * rms ** 3)
            out["d" + name] = d.reshape(R, heads * D)
    return out


def _exact_rows(q, k, v, seen, scale):
    a = (q @ k.t()) * scale
    a = a.masked_fill(~seen, -math.inf)
    w = torch.exp(a - a.max(1, keepdim=True).values)
    return w / w.sum(1, keepdim=True)


def _exact_attend(s, c):
    H, G, D, scale = c["heads"], c["kv_heads"], c["dim"], c["dim"] ** -0.5
    out = {n: torch.zeros(s[m].shape, dtype=torch.float64, device="cuda") for n, m in (("y", "q"), ("dq", "q"), ("dk", "k"), ("dv", "v"))}
    a = 0
    for n in _lengths(c):
        rows = slice(a, a + n)
        a += n
        at = torch.arange(n, device="cuda")
        seen = torch.ones(n, n, dtype=torch.bool, device="cuda")
        if c["causal"]:
            seen = at[:, None] >= at
            if c["window"]:
                seen &= at > at[:, None] - c["window"]
        for h in range(H):
            mine, theirs = slice(h * D, (h + 1) * D), slice(h // (H // G) * D, (h // (H // G) + 1) * D)
            q, k, v = s["q"][rows, mine].double(), s["k"][rows, theirs].double(), s["v"][rows, theirs].double()
            p = _exact_rows(q, k, v, seen, scale)
            out["y"][rows, mine] = p @ v
            if c["train"]:
                dy = s["dy"][rows, mine].double()
                out["dv"][rows, theirs] += p.t() @ dy
                dp = dy @ v.t()
                ds = p * (dp - torch.sum(p * dp, 1, keepdim=True)) * scale
                out["dq"][rows, mine] = ds @ k
                out["dk"][rows, theirs] += ds.t() @ q
    return out if c["train"] else {"y": out["y"]}


def _exact_serve(s, c):
    H, G, D, page, scale = c["heads"], c["kv_heads"], c["dim"], c["page"], c["dim"] ** -0.5
    new, total = _rows_and_totals(c)
    kc, vc, y = s["kc"].clone(), s["vc"].clone(), torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    pages, a = s["pages"].cpu().tolist(), 0
    for r, (n, t) in enumerate(zip(new, total)):
        rows = slice(a, a + n)
        a += n
        where = (torch.tensor(pages[r], device="cuda")[:, None] * page + torch.arange(page, device="cuda")).reshape(-1)[:t]
        kc[where[t - n:]], vc[where[t - n:]] = s["k"][rows], s["v"][rows]
        at, mine = torch.arange(t, device="cuda"), torch.arange(t - n, t, device="cuda")[:, None]
        seen = at <= mine
        if c["window"]:
            seen = seen & (at > mine - c["window"])
        for h in range(H):
            cols, theirs = slice(h * D, (h + 1) * D), slice(h // (H // G) * D, (h // (H // G) + 1) * D)
            k, v = kc[where][:, theirs].double(), vc[where][:, theirs].double()
            y[rows, cols] = _exact_rows(s["q"][rows, cols].double(), k, v, seen, scale) @ v
    return {"y": y, "kc": kc.double(), "vc": vc.double()}


def exact(case, seed):
    return {"rotate": _exact_rotate, "attend": _exact_attend, "serve": _exact_serve}[case["op"]](prepare(case, seed), case)
