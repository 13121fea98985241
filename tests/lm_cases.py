"""Shared by the tests of the language-model operators: graphs, seeded inputs and running a description on the GPU."""
import numpy as np

from oracle import interp
from paper_1707_08265_b200 import workloads as wl

U32, U16 = 2.0 ** -24, 2.0 ** -8            # half a step, relative, of fp32 and bf16


def as_type(a, dtype):
    return interp.round_bf16(a) if dtype == "bf16" else interp.round_e4m3(a) if dtype == "f8e4m3" else np.asarray(a, np.float32).astype(np.float64)


def torch_type(dtype):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16, "i32": torch.int32, "f8e4m3": torch.float8_e4m3fn}[dtype]


def to_gpu(a, dtype):
    import torch
    if dtype == "i32":
        return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32).reshape(np.shape(a))).cuda().to(torch_type(dtype))


def run_gpu(desc, inputs, outputs, feeds, function=None, fill=True):
    """(outputs as fp64 arrays, function); every output buffer is full of NaN (or 0x7f) before, with a guard behind it."""
    import torch
    from paper_1707_08265_b200 import binding as B
    f = function or B.Graph.from_desc(desc).function(inputs, outputs)
    used = f.used_inputs()
    dev = [to_gpu(a, desc["tensors"][t]["dtype"]) if u else None for a, t, u in zip(feeds, inputs, used)]
    bufs, outs = [], []
    for t in outputs:
        info = desc["tensors"][t]
        n = int(np.prod(info["shape"])) if info["shape"] else 1
        size = torch.empty(0, dtype=torch_type(info["dtype"])).element_size()
        raw = torch.full((n * size + 64,), 0x7F, dtype=torch.uint8, device="cuda")
        bufs.append((raw, n * size))
        outs.append(raw[:n * size].view(torch_type(info["dtype"])).view(info["shape"]))
    f.run_torch(dev, outs)
    assert f.status() == 0
    torch.cuda.synchronize()
    for raw, n in bufs:
        assert bool((raw[n:] == 0x7F).all()), "a kernel wrote behind its output"
    return [o.double().cpu().numpy() for o in outs], f


def norm_graph(rows, cols, x="bf16", r="bf16", h="bf16", y="bf16", gain="f32", eight_bit=False, grad=False, skip=None, eps=1e-6, fetch_h=True):
    g = wl.GraphDesc()
    ids = {"x": g.tensor("x", [rows, cols], x)}
    if r:
        ids["r"] = g.tensor("r", [rows, cols], r)
    ids["g"] = g.tensor("g", [cols], gain)
    ids["h"] = g.op("Add", [ids["x"], ids["r"]], "h", [rows, cols], h) if r else ids["x"]
    ids["y"] = g.op("RMSNorm", [ids["h"], ids["g"]], "y", [rows, cols], y, attrs=[eps])
    inputs = [ids["x"]] + ([ids["r"]] if r else []) + [ids["g"]]
    outputs = ([ids["h"]] if r and fetch_h else []) + ([] if eight_bit == "only" else [ids["y"]])
    if eight_bit:
        ids["s"] = g.op("BlockScale", [ids["y"]], "s", [rows, -(-cols // 128)])
        ids["q"] = g.op("Quantize", [ids["y"], ids["s"]], "q", [rows, cols], "f8e4m3")
        outputs += [ids["s"], ids["q"]]
    if grad:
        ids["dy"] = g.tensor("dy", [rows, cols], y)
        objs = [g.op("Mul", [ids["y"], ids["dy"]], "along_y")]
        inputs.append(ids["dy"])
        if skip:
            ids["dskip"] = g.tensor("dskip", [rows, cols], skip)
            objs.append(g.op("Mul", [ids["h"], ids["dskip"]], "along_h"))
            inputs.append(ids["dskip"])
        ids["dx"], ids["dg"] = g.grad(objs, [ids["x"], ids["g"]])
        outputs += [ids["dx"], ids["dg"]]
    return g, ids, inputs, outputs


def normals(desc, inputs, seed, scale={}):
    rng = np.random.default_rng(seed)
    out = []
    for t in inputs:
        info = desc["tensors"][t]
        out.append(as_type(rng.standard_normal(info["shape"]) * scale.get(info["name"], 1.0), info["dtype"]))
    return out


def e4m3_half_step(v):
    """Half the distance between neighbouring e4m3 values at magnitude |v| (the wider one next to a power of two)."""
    _, e = np.frexp(np.abs(v) * (1 + 1e-5))
    return np.exp2(np.maximum(e - 1, -6) - 4.0)


def scan_graph(seqs, length, cols, gate="bf16", x="bf16", h="bf16", h0="f32", reset=False, grad=False, dh=None):
    g, rows = wl.GraphDesc(), seqs * length
    ids = {"gate": g.tensor("gate", [rows, cols], gate), "x": g.tensor("x", [rows, cols], x)}
    ins = [ids["gate"], ids["x"]]
    if h0:
        ids["h0"] = g.tensor("h0", [seqs, cols], h0)
        ins.append(ids["h0"])
    if reset:
        ids["reset"] = g.tensor("reset", [rows], "i32")
        ins.append(ids["reset"])
    ids["h"] = g.op("GatedScan", ins, "h", [rows, cols], h, attrs=[seqs])
    inputs, outputs = list(ins), [ids["h"]]
    if grad:
        ids["dh"] = g.tensor("dh", [rows, cols], dh or h)
        obj = g.op("Mul", [ids["h"], ids["dh"]], "along")
        grads = g.grad([obj], ins[:3] if h0 else ins[:2])
        ids.update(zip(["dgate", "dx", "dh0"], grads))
        inputs.append(ids["dh"])
        outputs += grads
    return g, ids, inputs, outputs


def scan_bounds(desc, ids, feeds_by_name, seqs):
    """Absolute error bounds of an fp32 evaluation in any association: every row adds a relative error of (6 + |z|) 2^-23
    (the gate's exponential to an error of |z| 2^-24 in its argument plus a few roundings, the two products, the sum) to the
    sum of magnitudes that reaches it, H = f H + (1 - f)|x| forwards and E = |dh| + f E backwards."""
    z, x = feeds_by_name["gate"], feeds_by_name["x"]
    rows, cols = z.shape
    shape = (seqs, rows // seqs, cols)
    z, x = z.reshape(shape), x.reshape(shape)
    f, keep = 1 / (1 + np.exp(-z)), 1 / (1 + np.exp(z))
    fresh = feeds_by_name.get("reset")
    fresh = np.zeros(shape[:2], bool) if fresh is None else fresh.reshape(shape[:2]) != 0
    H = np.abs(feeds_by_name["h0"]) if "h0" in feeds_by_name else np.zeros((seqs, cols))
    e = np.zeros((seqs, cols))
    u = (6 + np.abs(z)) * 2 * U32
    out = {k: np.empty(shape) for k in ("h", "dx", "dgate")}
    Hp, ep = np.empty(shape), np.empty(shape)
    for t in range(shape[1]):
        H, e = np.where(fresh[:, t, None], 0, H), np.where(fresh[:, t, None], 0, e)
        Hp[:, t], ep[:, t] = H, e
        H = f[:, t] * H + keep[:, t] * np.abs(x[:, t])
        e = f[:, t] * e + u[:, t] * H
        out["h"][:, t] = e
    if "dh" in feeds_by_name:
        dh = np.abs(feeds_by_name["dh"].reshape(shape))
        E, ed = np.zeros((seqs, cols)), np.zeros((seqs, cols))
        for t in reversed(range(shape[1])):
            E = dh[:, t] + E
            ed = ed + 2 * U32 * E
            out["dx"][:, t] = keep[:, t] * (ed + u[:, t] * E)
            out["dgate"][:, t] = f[:, t] * keep[:, t] * ((ed + 3 * u[:, t] * E) * (Hp[:, t] + np.abs(x[:, t])) + E * ep[:, t])
            ed = np.where(fresh[:, t, None], 0, f[:, t] * ed + u[:, t] * f[:, t] * E)
            E = np.where(fresh[:, t, None], 0, f[:, t] * E)
        out["dh0"] = ed
    return {k: v.reshape(rows, cols) if k != "dh0" else v for k, v in out.items()}
