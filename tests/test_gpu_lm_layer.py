"""A layer of the language-model operators as it is used: trained for a few steps under clipping, and served in 8 bits."""
import numpy as np
import pytest

from lm_cases import as_type, run_gpu, to_gpu, torch_type
from oracle import interp
from paper_1707_08265_b200 import workloads as wl


def layer_feeds(g, ids, seed, vocab):
    rng = np.random.default_rng(seed)
    inputs = [ids["r"]] + ([ids["reset"]] if "reset" in ids else []) + [ids["labels"]] + ids["weights"]
    feeds = []
    for t in inputs:
        info = g.desc["tensors"][t]
        if info["name"] == "labels":
            feeds.append(rng.integers(0, vocab, info["shape"]).astype(np.int32))
        elif info["name"] == "reset":
            feeds.append((rng.random(info["shape"]) < 0.03).astype(np.int32))
        else:
            scale = 1.0 / np.sqrt(info["shape"][1]) if info["name"].startswith("W") else 1.0
            feeds.append(as_type(rng.standard_normal(info["shape"]) * scale, info["dtype"]))
    return inputs, feeds


def far(got, want):
    return np.linalg.norm(got - want) / np.linalg.norm(want)


# Every value passes at most eight roundings to bf16 (y, f or x, h, r2, y2, and three gradients on its way back), each at most
# 2^-8 of the value, in each of two evaluations that may round differently: 16 * 2^-8 bounds the relative 2-norm.
FAR = 16 * 2.0 ** -8


@pytest.mark.gpu
@pytest.mark.parametrize("seqs,length,width,inner,vocab,resets", [(2, 130, 64, 96, 40, True), (3, 64, 128, 128, 256, False), (1, 300, 72, 136, 104, True)])
def test_layer_loss_and_gradients(seqs, length, width, inner, vocab, resets):
    g, ids = wl.recurrent_layer(seqs, length, width, inner, vocab, resets)
    inputs, feeds = layer_feeds(g, ids, seqs + length, vocab)
    outputs = [ids["loss"], ids["r2"]] + ids["grads"]
    got, f = run_gpu(g.desc, inputs, outputs, feeds)
    want = interp.run_function(g.desc, inputs, outputs, feeds)
    assert abs(got[0] - want[0]) <= FAR * abs(want[0])
    for t, a, b in zip(outputs[1:], got[1:], want[1:]):
        assert far(a, b) <= FAR, g.desc["tensors"][t]["name"]
    assert "rms_norm_bwd" in f.describe() and "gated_scan_bwd" in f.describe()


@pytest.mark.gpu
def test_training_steps_in_a_workspace():
    """Loss and gradients, then the update of every weight under one clipped norm, weights and gradients by name on the device;
    each step's gradients and update follow the oracle from the weights the device holds."""
    import torch
    from paper_1707_08265_b200 import binding as B
    seqs, length, width, inner, vocab, limit, lr = 2, 80, 64, 64, 48, 0.05, 0.5
    g, ids = wl.recurrent_layer(seqs, length, width, inner, vocab)
    inputs, feeds = layer_feeds(g, ids, 1, vocab)
    names = [g.desc["tensors"][t]["name"] for t in ids["weights"]]
    shapes = [g.shape(t) for t in ids["weights"]]
    u, uids = wl.clipped_updater(shapes, limit)
    ws = B.Workspace()
    step = B.Graph.from_desc(g.desc).function(inputs, [ids["loss"]] + ids["grads"])
    update = B.Graph.from_desc(u.desc).function(uids["W"] + uids["g"] + [uids["lr"]], uids["W_new"] + [uids["norm"]])

    def put(name, a, dtype):
        t = to_gpu(a, dtype).cpu()
        ws.feed(name, B.DTYPES[dtype], list(t.shape), t.data_ptr())

    def take(name, shape, dtype="f32"):
        t = torch.empty(shape, dtype=torch_type(dtype))
        ws.fetch(name, t.data_ptr(), t.numel() * t.element_size())
        torch.cuda.synchronize()
        return t.double().numpy()

    for t, a in zip(inputs, feeds):
        put(g.desc["tensors"][t]["name"], a, g.desc["tensors"][t]["dtype"])
    master = [a for t, a in zip(inputs, feeds) if t in ids["weights"]]
    for i, a in enumerate(master):
        put("W%d" % i, a, "f32")
    put("lr", np.float32(lr), "f32")
    losses = []
    for k in range(4):
        ws.run(step, ["loss"] + ["g%d" % i for i in range(len(names))])
        ws.run(update, ["W%d" % i for i in range(len(names))] + ["norm"])
        losses.append(float(take("loss", [])))
        want = interp.run_function(g.desc, inputs, [ids["loss"]] + ids["grads"], feeds)
        assert abs(losses[-1] - want[0]) <= FAR * abs(want[0])
        grads = [take("g%d" % i, s) for i, s in enumerate(shapes)]
        for n, a, b in zip(names, grads, want[1:]):
            assert far(a, b) <= FAR, n
        # the update from the gradients that the device holds: fp32 against fp64
        norm = np.sqrt(sum((a ** 2).sum() for a in grads))
        assert abs(take("norm", []) - norm) <= 20 * 2.0 ** -24 * norm
        new = [take("W%d" % i, s) for i, s in enumerate(shapes)]
        for w, d, a in zip(master, grads, new):
            expect = w - lr * d * min(1.0, limit / norm)
            assert np.abs(a - expect).max() <= 30 * 2.0 ** -24 * (np.abs(w) + lr * np.abs(d)).max()
        master = new
        feeds = list(feeds)
        for t, n, a in zip(ids["weights"], names, new):
            feeds[inputs.index(t)] = as_type(a, g.desc["tensors"][t]["dtype"])
            put(n, feeds[inputs.index(t)], g.desc["tensors"][t]["dtype"])
    assert norm > limit                      # the steps were clipped ones


@pytest.mark.gpu
@pytest.mark.parametrize("seqs,width,inner", [(1, 128, 256), (5, 256, 144), (33, 400, 272)])
def test_decoding_steps_in_eight_bits(seqs, width, inner):
    """Weights brought into e4m3 on the device, then three steps whose states go from one to the next; against the layer
    evaluated in fp64 with the same 8-bit weights."""
    from paper_1707_08265_b200 import binding as B
    rng = np.random.default_rng(seqs)
    g, ids = wl.recurrent_step(seqs, width, inner)
    weights = {}
    for n in ("Wf", "Wx", "Wo"):
        shape = g.shape(ids[n])
        q = wl.GraphDesc()
        w = q.tensor("w", shape, "bf16")
        s = q.op("BlockScale", [w], "s", g.shape(ids["s" + n]), attrs=[128])
        v = q.op("Quantize", [w, s], "q", shape, "f8e4m3")
        (weights["s" + n], weights[n]), _ = run_gpu(q.desc, [w], [s, v], [as_type(rng.standard_normal(shape) / np.sqrt(shape[1]), "bf16")])
    names = ["g1", "states", "Wf", "sWf", "Wx", "sWx", "Wo", "sWo"]
    states = as_type(rng.standard_normal((seqs, inner)), "f32")
    f = B.Graph.from_desc(g.desc).function([ids["r"]] + [ids[n] for n in names], [ids["r2"], ids["new_states"]])
    assert [line.split("[")[0] for line in f.describe().splitlines() if line[0] != " "][:4] == ["rms_norm", "gemm_e4m3", "gemm_e4m3", "gated_scan"]
    for _ in range(3):
        fixed = {"g1": as_type(1 + 0.1 * rng.standard_normal(width), "f32"), "states": states, **weights}
        feeds = [as_type(rng.standard_normal((seqs, width)), "bf16")] + [fixed[n] for n in names]
        inputs, outputs = [ids["r"]] + [ids[n] for n in names], [ids["r2"], ids["new_states"]]
        (r2, new), _ = run_gpu(g.desc, inputs, outputs, feeds, f)
        w_r2, w_new = interp.run_function(g.desc, inputs, outputs, feeds)
        # where fp32 and fp64 fall on two sides of a tie an e4m3 value (a 16th of its size at most, one in some 10^5) differs
        assert far(new, w_new) <= 1e-3 and far(r2, w_r2) <= 2.0 ** -7
        states = new


def test_plans_of_the_layer():
    from paper_1707_08265_b200 import binding as B
    g, ids = wl.recurrent_layer(2, 64, 64, 64, 64)
    inputs, _ = layer_feeds(g, ids, 0, 64)
    text = B.Graph.from_desc(g.desc).function(inputs, [ids["loss"]] + ids["grads"]).describe()
    kinds = [line.split("[")[0].split(" ")[0] for line in text.splitlines() if line[0] != " "]
    assert kinds.count("rms_norm") == 2 and kinds.count("rms_norm_bwd") == 2 and kinds.count("gated_scan") == 1 and kinds.count("gated_scan_bwd") == 1
    u, uids = wl.clipped_updater([[64, 64], [48]], 1.0)
    text = B.Graph.from_desc(u.desc).function(uids["W"] + uids["g"] + [uids["lr"]], uids["W_new"]).describe()
    kinds = [line.split("[")[0] for line in text.splitlines() if line[0] != " "]
    assert kinds == ["global_norm", "vm", "vm"] and "->factor" in text
