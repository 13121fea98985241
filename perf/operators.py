"""Measured cases of the language-model operators: what one pass computes, in plain torch and through the library.

Operators (operator types of the graph, see include/dragon.h):
  RMSNorm                  y = h / sqrt(mean(h^2) + eps) * g on rows of h = x + r (the residual's addition), with its gradient
  BlockScale, Quantize     scales amax / 448 of blocks of 128 (1 x 128 of a row, 128 x 128 of a weight) and e4m3 values
  ScaledInnerProduct       Y = Xq Wq^T with both operands in e4m3 and a scale for each block of 128 along the contraction
  GlobalNorm, ClipByNorm   the 2-norm over many gradient tensors, and every tensor times min(1, limit / norm)
  GatedScan                h_t = f_t h_(t-1) + (1 - f_t) x_t with f = sigmoid(gate), over rows of packed sequences, with its gradient

``own`` false: elementary torch operations in 32 bits (64 for the long sum of the norm).  ``own`` true: the library's
functions, compiled once per shape as a user's program keeps them, run on the state's buffers.
"""
import functools
import math

import torch

own = False

EPS = 1e-6
BLOCK = 128
E4M3_MAX = 448.0
TINY = 2.0 ** -126          # the smallest scale
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


# ---- cases ------------------------------------------------------------------------------------------------

def listed():
    return [
        # one decoding step of eight sequences: residual addition and norm of eight rows, where the launch is what counts
        {"name": "norm_token", "op": "norm", "rows": 8, "cols": 4096, "dtype": "bf16", "train": False},
        # a training step's norm at the benchmark MLP's activation size: forward, then the gradient with the residual branch's
        {"name": "norm_train", "op": "norm", "rows": 8192, "cols": 4096, "dtype": "bf16", "train": True},
        # a prefill of ragged length in front of an 8-bit projection whose width is no multiple of 128
        {"name": "norm8_ragged", "op": "norm8", "rows": 4099, "cols": 5000, "dtype": "bf16"},
        # a weight matrix brought into 8 bits once, in blocks of 128 x 128
        {"name": "quantize_weight", "op": "quantize", "rows": 8192, "cols": 8192, "block_rows": 128, "dtype": "bf16"},
        # a projection for five tokens: the weights' bytes are what counts
        {"name": "product_token", "op": "product", "m": 5, "n": 8192, "k": 4096, "dtype": "bf16"},
        # a short prefill, every extent ragged, 32-bit output
        {"name": "product_ragged", "op": "product", "m": 777, "n": 2056, "k": 2064, "dtype": "f32"},
        # the benchmark MLP's first product with a wider hidden layer
        {"name": "product_large", "op": "product", "m": 8192, "n": 8192, "k": 4096, "dtype": "bf16"},
        # the gradients of one small layer
        {"name": "clip_small", "op": "clip", "layers": 1, "width": 256, "inner": 640, "rows_embed": 1000, "dtype": "f32"},
        # the gradients of a model of some 440 million weights
        {"name": "clip_large", "op": "clip", "layers": 12, "width": 2048, "inner": 5632, "rows_embed": 32000, "dtype": "bf16"},
        # one decoding step of the recurrence for 64 sequences, each with its state
        {"name": "scan_token", "op": "scan", "seqs": 64, "length": 1, "cols": 4096, "dtype": "bf16", "resets": False, "state": True, "train": False},
        # packed documents in a few rows of a batch, odd width, training
        {"name": "scan_packed", "op": "scan", "seqs": 3, "length": 2047, "cols": 1025, "dtype": "f32", "resets": True, "state": True, "train": True},
        # one long sequence, training
        {"name": "scan_long", "op": "scan", "seqs": 1, "length": 65536, "cols": 1024, "dtype": "bf16", "resets": False, "state": False, "train": True},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "norm", "norm8", "quantize", "product", "product", "clip", "scan", "scan"])
    if op in ("norm", "norm8"):
        cols = _log(rng, 32, 16384)
        cols = cols if rng.random() < 0.3 else max(8, cols // 8 * 8)
        rows = min(_log(rng, 1, 16384), max(1, 33554432 // cols))
        c = {"op": op, "rows": rows, "cols": cols, "dtype": rng.choice(["bf16", "bf16", "f32"])}
        if op == "norm":
            c["train"] = rng.random() < 0.6
        return c
    if op == "quantize":
        cols, rows = _log(rng, 16, 16384), _log(rng, 1, 8192)
        cols = cols if rng.random() < 0.3 else max(16, cols // 16 * 16)
        return {"op": op, "rows": min(rows, max(1, 67108864 // cols)), "cols": cols, "block_rows": rng.choice([1, 128]), "dtype": rng.choice(["bf16", "f32"])}
    if op == "product":
        m, n, k = _log(rng, 1, 8192), _log(rng, 64, 8192), max(16, _log(rng, 64, 8192) // 16 * 16)
        m = max(1, min(m, 8192 * 8192 * 4096 // (n * k)))
        return {"op": op, "m": m, "n": n if rng.random() < 0.3 else max(8, n // 8 * 8), "k": k, "dtype": rng.choice(["bf16", "bf16", "f32"])}
    if op == "clip":
        return {"op": op, "layers": rng.randint(1, 12), "width": _log(rng, 64, 2048), "inner": _log(rng, 100, 5632), "rows_embed": _log(rng, 10, 32000),
                "dtype": rng.choice(["bf16", "f32"])}
    cols = _log(rng, 16, 8192)
    cols = cols if rng.random() < 0.3 else max(8, cols // 8 * 8)
    length = _log(rng, 1, 65536)
    length = max(1, min(length, 67108864 // cols))
    seqs = max(1, min(_log(rng, 1, 64), 33554432 // (cols * length)))
    return {"op": op, "seqs": seqs, "length": length, "cols": cols, "dtype": rng.choice(["bf16", "bf16", "f32"]), "resets": rng.random() < 0.4,
            "state": rng.random() < 0.5, "train": rng.random() < 0.6}


# ---- inputs -----------------------------------------------------------------------------------------------

def _gradient_shapes(c):
    w, i = c["width"], c["inner"]
    shapes = [[c["rows_embed"], w]]
    for _ in range(c["layers"]):
        shapes += [[w, w], [i, w], [w, i], [w]]
    return shapes


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, dtype=torch.float32, scale=1.0, shift=0.0):
        return torch.empty(shape, device="cuda").normal_(shift, scale, generator=gen).to(dtype)

    def empty(*shape, dtype):
        return torch.empty(shape, device="cuda", dtype=dtype)

    c, s, op = dict(case), {"case": dict(case)}, case["op"]
    dt = DT.get(c.get("dtype"))
    if op in ("norm", "norm8", "quantize"):
        R, C = c["rows"], c["cols"]
        s["x"] = normal(R, C, dtype=dt)
        if op != "quantize":
            s["r"] = normal(R, C, dtype=dt, scale=2.0)          # the residual stream carries more than one branch's output
            s["g"] = normal(C, scale=0.2, shift=1.0)
            s["h"] = empty(R, C, dtype=dt)
        if op == "norm":
            s["y"] = empty(R, C, dtype=dt)
            if c["train"]:
                s["dy"], s["dskip"] = normal(R, C, dtype=dt), normal(R, C, dtype=dt)
                s["dx"], s["dg"] = empty(R, C, dtype=torch.float32), empty(C, dtype=torch.float32)
        else:
            br = c.get("block_rows", 1)
            s["q"] = empty(R, C, dtype=torch.float8_e4m3fn)
            s["s"] = empty(-(-R // br), -(-C // BLOCK), dtype=torch.float32)
    elif op == "product":
        M, N, K = c["m"], c["n"], c["k"]
        kb = -(-K // BLOCK)
        s["xq"] = normal(M, K, scale=120.0).clamp_(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)
        s["wq"] = normal(N, K, scale=120.0).clamp_(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)
        s["sx"] = normal(M, kb, scale=0.4).exp_() * (1 / 120.0)
        s["sw"] = normal(-(-N // BLOCK), kb, scale=0.4).exp_() * (1 / (120.0 * math.sqrt(K)))
        s["out"] = empty(M, N, dtype=dt)
    elif op == "clip":
        shapes = _gradient_shapes(c)
        s["grads"] = [normal(*sh, dtype=dt if len(sh) == 2 else torch.float32, scale=1e-3) for sh in shapes]   # matrices in the case's type, vectors in 32 bits
        s["limit"] = 1.0
        s["clipped"] = [torch.empty_like(t) for t in s["grads"]]
        s["norm"] = empty(dtype=torch.float32)
    elif op == "scan":
        S, L, C = c["seqs"], c["length"], c["cols"]
        s["gate"] = normal(S * L, C, dtype=dt, scale=1.5, shift=1.5)       # most gates keep: memories of a few to some hundred rows
        s["x"] = normal(S * L, C, dtype=dt)
        s["h"] = empty(S * L, C, dtype=dt)
        s["h0"] = normal(S, C) if c["state"] else None
        s["reset"] = (torch.rand(S * L, device="cuda", generator=gen) < 1 / 400).to(torch.int32) if c["resets"] else None
        if c["train"]:
            s["dh"] = normal(S * L, C, dtype=dt)
            s["dgate"], s["dx"] = empty(S * L, C, dtype=torch.float32), empty(S * L, C, dtype=torch.float32)
            s["dh0"] = empty(S, C, dtype=torch.float32) if c["state"] else None
    else:
        raise ValueError(op)
    return s


# ---- the plain forms --------------------------------------------------------------------------------------

def _scales(v, block_rows):
    R, C = v.shape
    pr, pc = -R % block_rows, -C % BLOCK
    w = torch.nn.functional.pad(v.abs(), (0, pc, 0, pr)).view((R + pr) // block_rows, block_rows, (C + pc) // BLOCK, BLOCK)
    return (w.amax(dim=(1, 3)) / E4M3_MAX).clamp_min(TINY)


def _spread(s, rows, cols, block_rows):
    return s.repeat_interleave(block_rows, 0)[:rows].repeat_interleave(BLOCK, 1)[:, :cols]


def _plain_norm(s):
    h = (s["x"].float() + s["r"].float()).to(s["h"].dtype)      # the carried sum is a tensor of its own type; the norm reads it
    hf = h.float()
    rstd = torch.rsqrt((hf * hf).mean(1, keepdim=True) + EPS)
    return h, hf, rstd


def _doubling(a, b):
    """b_t + a_t (b_(t-1) + a_(t-1) (...)) along dimension 1, in log2 steps."""
    n = 1
    while n < a.shape[1]:
        b = torch.cat([b[:, :n], b[:, n:] + a[:, n:] * b[:, :-n]], 1)
        a = torch.cat([a[:, :n], a[:, n:] * a[:, :-n]], 1)
        n *= 2
    return b


def _plain_scan(s):
    c = s["case"]
    S, L, C = c["seqs"], c["length"], c["cols"]
    gate, x = s["gate"].float().view(S, L, C), s["x"].float().view(S, L, C)
    f, keep = torch.sigmoid(gate), torch.sigmoid(-gate)
    fresh = torch.zeros(S, L, 1, dtype=torch.bool, device=x.device) if s["reset"] is None else (s["reset"] != 0).view(S, L, 1)
    a = torch.where(fresh, 0.0, f)                              # what of the row before comes through
    b = keep * x
    start = torch.zeros(S, C, device=x.device) if s["h0"] is None else s["h0"]
    first = torch.zeros(S, L, 1, dtype=torch.bool, device=x.device)
    first[:, 0] = True
    h = _doubling(torch.where(first, 0.0, a), torch.where(first, b + a * start[:, None], b))
    out = {"h": h.to(s["h"].dtype).view(S * L, C)}
    if c["train"]:
        dh = s["dh"].float().view(S, L, C)
        later = torch.cat([a[:, 1:], torch.zeros_like(a[:, :1])], 1)
        d = _doubling(later.flip(1), dh.flip(1)).flip(1)
        before = torch.where(fresh, 0.0, torch.cat([start[:, None], h[:, :-1]], 1))
        out["dx"] = (d * keep).view(S * L, C)
        out["dgate"] = (d * (before - x) * (f * keep)).view(S * L, C)
        if s["h0"] is not None:
            out["dh0"] = d[:, 0] * a[:, 0]
    return out


def _plain(s):
    c = s["case"]
    op = c["op"]
    if op == "norm":
        h, hf, rstd = _plain_norm(s)
        out = {"h": h, "y": (hf * rstd * s["g"]).to(s["y"].dtype)}
        if c["train"]:
            dy = s["dy"].float()
            t = dy * s["g"]
            out["dx"] = s["dskip"].float() + rstd * (t - hf * (rstd * rstd * (t * hf).mean(1, keepdim=True)))
            out["dg"] = (dy * hf * rstd).sum(0)
        return out
    if op == "norm8":
        h, hf, rstd = _plain_norm(s)
        y = hf * rstd * s["g"]
        sc = _scales(y, 1)
        return {"h": h, "s": sc, "q": (y / _spread(sc, *y.shape, 1)).to(torch.float8_e4m3fn)}
    if op == "quantize":
        x = s["x"].float()
        sc = _scales(x, c["block_rows"])
        return {"s": sc, "q": (x / _spread(sc, *x.shape, c["block_rows"])).to(torch.float8_e4m3fn)}
    if op == "product":
        x = s["xq"].float() * _spread(s["sx"], c["m"], c["k"], 1)
        w = s["wq"].float() * _spread(s["sw"], c["n"], c["k"], BLOCK)
        return {"out": torch.matmul(x, w.t()).to(s["out"].dtype)}
    if op == "clip":
        norm = torch.stack([g.double().square().sum() for g in s["grads"]]).sum().sqrt()
        factor = (s["limit"] / norm.clamp_min(s["limit"])).float()
        return {"norm": norm.float(), "clipped": [(g.float() * factor).to(g.dtype) for g in s["grads"]]}
    return _plain_scan(s)


# ---- the library's calls ----------------------------------------------------------------------------------

@functools.lru_cache(maxsize=None)
def _norm_function(rows, cols, dtype, train, eight_bit):
    from paper_1707_08265_b200 import binding as B
    g, dt = B.Graph(), B.DTYPES[dtype]
    x, r = g.add_tensor("x", dt, [rows, cols]), g.add_tensor("r", dt, [rows, cols])
    gain, h = g.add_tensor("g", B.F32, [cols]), g.add_tensor("h", dt, [rows, cols])
    y = g.add_tensor("y", B.F32 if eight_bit else dt, [rows, cols])
    g.add_op(B.OPS["Add"], [x, r], [h])
    g.add_op(B.OPS["RMSNorm"], [h, gain], [y], [EPS])
    if eight_bit:
        s, q = g.add_tensor("s", B.F32, [rows, -(-cols // BLOCK)]), g.add_tensor("q", B.F8E4M3, [rows, cols])
        g.add_op(B.OPS["BlockScale"], [y], [s], [1])
        g.add_op(B.OPS["Quantize"], [y, s], [q])
        return g.function([x, r, gain], [h, s, q])
    if not train:
        return g.function([x, r, gain], [h, y])
    dy, dskip = g.add_tensor("dy", dt, [rows, cols]), g.add_tensor("dskip", dt, [rows, cols])
    along_y, along_h = g.add_tensor("along_y", B.F32, [rows, cols]), g.add_tensor("along_h", B.F32, [rows, cols])
    g.add_op(B.OPS["Mul"], [y, dy], [along_y])                  # objectives whose gradients are dy and dskip
    g.add_op(B.OPS["Mul"], [h, dskip], [along_h])
    dx, dg = g.add_grad([along_y, along_h], [x, gain])
    return g.function([x, r, gain, dy, dskip], [h, y, dx, dg])


@functools.lru_cache(maxsize=None)
def _quantize_function(rows, cols, dtype, block_rows):
    from paper_1707_08265_b200 import binding as B
    g = B.Graph()
    x, q = g.add_tensor("x", B.DTYPES[dtype], [rows, cols]), g.add_tensor("q", B.F8E4M3, [rows, cols])
    s = g.add_tensor("s", B.F32, [-(-rows // block_rows), -(-cols // BLOCK)])
    g.add_op(B.OPS["BlockScale"], [x], [s], [block_rows])
    g.add_op(B.OPS["Quantize"], [x, s], [q])
    return g.function([x], [s, q])


@functools.lru_cache(maxsize=None)
def _product_function(m, n, k, dtype):
    from paper_1707_08265_b200 import binding as B
    g, kb = B.Graph(), -(-k // BLOCK)
    xq, sx = g.add_tensor("xq", B.F8E4M3, [m, k]), g.add_tensor("sx", B.F32, [m, kb])
    wq, sw = g.add_tensor("wq", B.F8E4M3, [n, k]), g.add_tensor("sw", B.F32, [-(-n // BLOCK), kb])
    out = g.add_tensor("out", B.DTYPES[dtype], [m, n])
    g.add_op(B.OPS["ScaledInnerProduct"], [xq, sx, wq, sw], [out])
    return g.function([xq, sx, wq, sw], [out])


@functools.lru_cache(maxsize=None)
def _clip_function(layers, width, inner, rows_embed, dtype, limit):
    from paper_1707_08265_b200 import binding as B
    g = B.Graph()
    shapes = _gradient_shapes({"layers": layers, "width": width, "inner": inner, "rows_embed": rows_embed})
    types = [B.DTYPES[dtype] if len(sh) == 2 else B.F32 for sh in shapes]
    grads = [g.add_tensor("g%d" % i, t, sh) for i, (t, sh) in enumerate(zip(types, shapes))]
    norm = g.add_tensor("norm", B.F32, [])
    g.add_op(B.OPS["GlobalNorm"], grads, [norm])
    clipped = [g.add_tensor("c%d" % i, t, sh) for i, (t, sh) in enumerate(zip(types, shapes))]
    for a, b in zip(grads, clipped):
        g.add_op(B.OPS["ClipByNorm"], [a, norm], [b], [limit])
    return g.function(grads, [norm] + clipped)


@functools.lru_cache(maxsize=None)
def _scan_function(seqs, length, cols, dtype, resets, state, train):
    from paper_1707_08265_b200 import binding as B
    g, dt, rows = B.Graph(), B.DTYPES[dtype], seqs * length
    gate, x, h = (g.add_tensor(n, dt, [rows, cols]) for n in ("gate", "x", "h"))
    ins = [gate, x]
    if state:
        ins.append(g.add_tensor("h0", B.F32, [seqs, cols]))
    if resets:
        ins.append(g.add_tensor("reset", B.I32, [rows]))
    g.add_op(B.OPS["GatedScan"], ins, [h], [seqs])
    if not train:
        return g.function(ins, [h])
    dh, along = g.add_tensor("dh", dt, [rows, cols]), g.add_tensor("along", B.F32, [rows, cols])
    g.add_op(B.OPS["Mul"], [h, dh], [along])
    grads = g.add_grad([along], ins[:3] if state else ins[:2])
    return g.function(ins + [dh], [h] + grads)


def _own(s):
    c = s["case"]
    op = c["op"]
    if op == "norm":
        f = _norm_function(c["rows"], c["cols"], c["dtype"], c["train"], False)
        if not c["train"]:
            f.run_torch([s["x"], s["r"], s["g"]], [s["h"], s["y"]])
            return {"h": s["h"], "y": s["y"]}
        f.run_torch([s["x"], s["r"], s["g"], s["dy"], s["dskip"]], [s["h"], s["y"], s["dx"], s["dg"]])
        return {"h": s["h"], "y": s["y"], "dx": s["dx"], "dg": s["dg"]}
    if op == "norm8":
        _norm_function(c["rows"], c["cols"], c["dtype"], False, True).run_torch([s["x"], s["r"], s["g"]], [s["h"], s["s"], s["q"]])
        return {"h": s["h"], "s": s["s"], "q": s["q"]}
    if op == "quantize":
        _quantize_function(c["rows"], c["cols"], c["dtype"], c["block_rows"]).run_torch([s["x"]], [s["s"], s["q"]])
        return {"s": s["s"], "q": s["q"]}
    if op == "product":
        _product_function(c["m"], c["n"], c["k"], c["dtype"]).run_torch([s["xq"], s["sx"], s["wq"], s["sw"]], [s["out"]])
        return {"out": s["out"]}
    if op == "clip":
        f = _clip_function(c["layers"], c["width"], c["inner"], c["rows_embed"], c["dtype"], s["limit"])
        f.run_torch(s["grads"], [s["norm"]] + s["clipped"])
        return {"norm": s["norm"], "clipped": s["clipped"]}
    f = _scan_function(c["seqs"], c["length"], c["cols"], c["dtype"], c["resets"], c["state"], c["train"])
    feeds = [t for t in (s["gate"], s["x"], s["h0"], s["reset"]) if t is not None]
    if not c["train"]:
        f.run_torch(feeds, [s["h"]])
        return {"h": s["h"]}
    out = {"h": s["h"], "dgate": s["dgate"], "dx": s["dx"]}
    if c["state"]:
        out["dh0"] = s["dh0"]
    f.run_torch(feeds + [s["dh"]], list(out.values()))
    return out


def run(state):
    return _own(state) if own else _plain(state)


# ---- what a pass cannot do without ------------------------------------------------------------------------

def work(case):
    c, op = case, case["op"]
    e = {"f32": 4, "bf16": 2}[c["dtype"]]
    if op == "norm":
        n = c["rows"] * c["cols"]
        w = {"bytes": 4 * n * e + 4 * c["cols"], "flops": 6 * n}
        if c["train"]:
            w = {"bytes": w["bytes"] + n * (2 * e + 4) + 4 * c["cols"], "flops": 18 * n}
        return w
    if op == "norm8":
        n = c["rows"] * c["cols"]
        return {"bytes": n * (3 * e + 1) + 4 * c["cols"] + 4 * c["rows"] * -(-c["cols"] // BLOCK), "flops": 8 * n}
    if op == "quantize":
        n = c["rows"] * c["cols"]
        return {"bytes": n * (e + 1) + 4 * -(-c["rows"] // c["block_rows"]) * -(-c["cols"] // BLOCK), "flops": 3 * n}
    if op == "product":
        m, n, k = c["m"], c["n"], c["k"]
        kb = -(-k // BLOCK)
        return {"bytes": (m + n) * k + 4 * kb * (m + -(-n // BLOCK)) + m * n * e, "flops": 2 * m * n * k}
    if op == "clip":
        n = [(math.prod(sh), e if len(sh) == 2 else 4) for sh in _gradient_shapes(c)]
        return {"bytes": 2 * sum(a * b for a, b in n) + 4, "flops": 3 * sum(a for a, _ in n)}
    n = c["seqs"] * c["length"] * c["cols"]
    state = 4 * c["seqs"] * c["cols"] if c["state"] else 0
    reset = 4 * c["seqs"] * c["length"] if c["resets"] else 0
    if c["train"]:
        return {"bytes": n * (4 * e + 8) + 2 * state + reset, "flops": 24 * n}
    return {"bytes": 3 * n * e + state + reset, "flops": 10 * n}


# ---- the definition in 64 bits ----------------------------------------------------------------------------

def _exact_e4m3(v):
    """Nearest e4m3 value (ties to even), from the format: steps of 2^(e-3), e >= -6, largest magnitude 448."""
    _, e = torch.frexp(v)
    step = torch.pow(2.0, (e - 1).clamp_min(-6).double() - 3)
    return (torch.round(v / step) * step).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)


def _exact_quantize(v, block_rows):
    R, C = v.shape
    nr, nc = -(-R // block_rows), -(-C // BLOCK)
    padded = v.new_zeros(nr * block_rows, nc * BLOCK)
    padded[:R, :C] = v
    tiles = padded.view(nr, block_rows, nc, BLOCK)
    s = torch.maximum(tiles.abs().amax(3).amax(1) / E4M3_MAX, torch.tensor(TINY, dtype=torch.float64, device=v.device))
    q = _exact_e4m3((tiles / s[:, None, :, None]).reshape(nr * block_rows, nc * BLOCK)[:R, :C])
    return s, q


def _exact_scan(s, c):
    S, L, C = c["seqs"], c["length"], c["cols"]
    gate, x = s["gate"].double().view(S, L, C), s["x"].double().view(S, L, C)
    reset = None if s["reset"] is None else s["reset"].view(S, L)
    f = 1 / (1 + torch.exp(-gate))
    rest = 1 / (1 + torch.exp(gate))
    start = torch.zeros(S, C, dtype=torch.float64, device=x.device) if s["h0"] is None else s["h0"].double()
    states, h = torch.empty_like(x), start
    before = torch.empty_like(x)
    for t in range(L):
        p = h if reset is None else torch.where(reset[:, t, None] != 0, torch.zeros_like(h), h)
        before[:, t] = p
        h = f[:, t] * p + rest[:, t] * x[:, t]
        states[:, t] = h
    out = {"h": states.view(S * L, C)}
    if c["train"]:
        dh, d = s["dh"].double().view(S, L, C), torch.zeros_like(start)
        total = torch.empty_like(x)
        for t in reversed(range(L)):
            d = dh[:, t] + d
            total[:, t] = d
            d = d * f[:, t]
            if reset is not None:
                d = torch.where(reset[:, t, None] != 0, torch.zeros_like(d), d)
        out["dx"] = (total * rest).view(S * L, C)
        out["dgate"] = (total * (before - x) * f * rest).view(S * L, C)
        if s["h0"] is not None:
            out["dh0"] = d
    return out


def exact(case, seed):
    s, c, op = prepare(case, seed), case, case["op"]
    if op in ("norm", "norm8"):
        h = (s["x"].double() + s["r"].double()).to(torch.float32).to(s["h"].dtype)   # the stored sum: one rounding to its type (bf16 sums of bf16 are exact in 32 bits up to that)
        v, gain = h.double(), s["g"].double()
        inv = 1 / torch.sqrt(torch.sum(v ** 2, 1) / c["cols"] + EPS)[:, None]
        y = v * inv * gain
        if op == "norm8":
            sc, q = _exact_quantize(y, 1)
            return {"h": h, "s": sc, "q": q}
        out = {"h": h, "y": y}
        if c["train"]:
            dy = s["dy"].double()
            u = v * inv                                                            # normalised rows
            du = dy * gain
            out["dx"] = s["dskip"].double() + inv * (du - u * (torch.sum(du * u, 1) / c["cols"])[:, None])
            out["dg"] = torch.sum(dy * u, 0)
        return out
    if op == "quantize":
        sc, q = _exact_quantize(s["x"].double(), c["block_rows"])
        return {"s": sc, "q": q}
    if op == "product":
        M, N, K = c["m"], c["n"], c["k"]
        total = torch.zeros(M, N, dtype=torch.float64, device="cuda")
        for b in range(-(-K // BLOCK)):
            k0, k1 = b * BLOCK, min(K, (b + 1) * BLOCK)
            part = s["xq"][:, k0:k1].double() @ s["wq"][:, k0:k1].double().t()
            total += part * s["sx"][:, b, None].double() * s["sw"][torch.arange(N, device="cuda") // BLOCK, b].double()[None]
        return {"out": total}
    if op == "clip":
        parts = [torch.sum(g.double() ** 2) for g in s["grads"]]
        norm = math.sqrt(math.fsum(float(p) for p in parts))
        k = min(1.0, s["limit"] / norm) if norm > 0 else 1.0
        return {"norm": torch.tensor(norm, dtype=torch.float64), "clipped": [g.double() * k for g in s["grads"]]}
    return _exact_scan(s, c)
