"""A layer of the attention operators as it is used: loss and gradients, trained for a few steps, served from a paged cache."""
import numpy as np
import pytest

from attention_cases import as_type
from lm_cases import run_gpu, to_gpu, torch_type
from oracle import interp
from paper_1707_08265_b200 import binding as B
from paper_1707_08265_b200 import workloads as wl

# Every value passes at most fourteen roundings to bf16 (y, q or k or v, turned, the probabilities, a, r2, y2, and on its way back the
# gradients of y2, r2, a, the scores, turned, q, y), each at most 2^-8 of the value, in each of two evaluations that may round
# differently: 28 * 2^-8 bounds the relative 2-norm.
FAR = 28 * 2.0 ** -8


def far(got, want):
    return np.linalg.norm(got - want) / np.linalg.norm(want)


def feeds_of(g, inputs, seed, **fixed):
    rng = np.random.default_rng(seed)
    out = []
    for t in inputs:
        info = g.desc["tensors"][t]
        if info["name"] in fixed:
            a = np.asarray(fixed[info["name"]])
            out.append(a.astype(np.int32) if info["dtype"] == "i32" else a)
        elif info["name"] == "labels":
            out.append(rng.integers(0, 40, info["shape"]).astype(np.int32))
        else:
            scale = 1 / np.sqrt(info["shape"][1]) if info["name"].startswith("W") else 0.2 if info["name"].startswith("gain") else 1.0
            out.append(as_type(rng.standard_normal(info["shape"]) * scale + info["name"].startswith("gain"), info["dtype"]))
    return out


def of_each(starts, rows):
    pos = np.zeros(rows, np.int32)
    for a, b in zip(starts[:-1], starts[1:]):
        pos[a:b] = np.arange(b - a)
    return pos


@pytest.mark.gpu
@pytest.mark.parametrize("rows,width,heads,kv,head_width,sequences,starts,window,interleaved", [
    (300, 64, 4, 2, 32, 1, None, 0, 0), (260, 96, 3, 3, 40, 2, None, 0, 1), (290, 128, 8, 1, 64, 1, [0, 100, 101, 290], 0, 0), (520, 64, 2, 1, 128, 1, None, 150, 0)])
def test_layer_loss_and_gradients(rows, width, heads, kv, head_width, sequences, starts, window, interleaved):
    g, ids = wl.attention_layer(rows, width, heads, kv, head_width, 40, sequences, len(starts) - 1 if starts else 0, window, interleaved)
    inputs = [ids[n] for n in ("r", "pos", "labels")] + ([ids["starts"]] if starts else []) + ids["weights"]
    each = starts or [k * (rows // sequences) for k in range(sequences + 1)]
    feeds = feeds_of(g, inputs, rows, pos=of_each(each, rows), **({"starts": starts} if starts else {}))
    outputs = [ids["loss"], ids["r2"]] + ids["grads"]
    got, f = run_gpu(g.desc, inputs, outputs, feeds)
    want = interp.run_function(g.desc, inputs, outputs, feeds)
    assert abs(got[0] - want[0]) <= FAR * abs(want[0])
    for t, a, b in zip(outputs[1:], got[1:], want[1:]):
        assert far(a, b) <= FAR, g.desc["tensors"][t]["name"]


@pytest.mark.gpu
def test_training_steps_in_a_workspace():
    """Loss and gradients, then the update of every weight under one clipped norm, all by name on the device; each step's loss and
    gradients follow the oracle from the weights that the device holds."""
    import torch
    rows, limit, lr = 200, 0.05, 0.5
    g, ids = wl.attention_layer(rows, 64, 4, 2, 32, 48, sequences=2)
    inputs = [ids[n] for n in ("r", "pos", "labels")] + ids["weights"]
    feeds = feeds_of(g, inputs, 8, pos=of_each([0, 100, 200], rows))
    names, shapes = [g.desc["tensors"][t]["name"] for t in ids["weights"]], [g.shape(t) for t in ids["weights"]]
    u, uids = wl.clipped_updater(shapes, limit)
    ws = B.Workspace()
    step = B.Graph.from_desc(g.desc).function(inputs, [ids["loss"]] + ids["grads"])
    update = B.Graph.from_desc(u.desc).function(uids["W"] + uids["g"] + [uids["lr"]], uids["W_new"])

    def put(name, a, dtype):
        t = to_gpu(a, dtype).cpu()
        ws.feed(name, B.DTYPES[dtype], list(t.shape), t.data_ptr())

    def take(name, shape):
        t = torch.empty(shape, dtype=torch.float32)
        ws.fetch(name, t.data_ptr(), t.numel() * 4)
        torch.cuda.synchronize()
        return t.double().numpy()

    for t, a in zip(inputs, feeds):
        put(g.desc["tensors"][t]["name"], a, g.desc["tensors"][t]["dtype"])
    for k, t in enumerate(ids["weights"]):
        put("W%d" % k, feeds[inputs.index(t)], "f32")
    put("lr", np.float32(lr), "f32")
    for _ in range(3):
        ws.run(step, ["loss"] + ["g%d" % k for k in range(len(names))])
        ws.run(update, ["W%d" % k for k in range(len(names))])
        want = interp.run_function(g.desc, inputs, [ids["loss"]] + ids["grads"], feeds)
        assert abs(float(take("loss", [])) - want[0]) <= FAR * abs(want[0])
        for k, (n, s, w) in enumerate(zip(names, shapes, want[1:])):
            assert far(take("g%d" % k, s), w) <= FAR, n
        feeds = list(feeds)
        for k, t in enumerate(ids["weights"]):
            feeds[inputs.index(t)] = as_type(take("W%d" % k, shapes[k]), g.desc["tensors"][t]["dtype"])
            put(names[k], feeds[inputs.index(t)], g.desc["tensors"][t]["dtype"])


@pytest.mark.gpu
def test_a_prompt_and_tokens_behind_it_give_what_training_gives():
    """Two prompts of different lengths as one chunk, then single tokens, over a paged cache that stays in place under its names; the
    rows of the residual stream are those of the layer over whole sequences."""
    import torch
    prompts, more, width, heads, kv, hw, page, most, pool = [70, 33], 3, 64, 4, 2, 32, 16, 5, 11
    lengths = [n + more for n in prompts]
    starts = [0, lengths[0], sum(lengths)]
    g, ids = wl.attention_layer(starts[-1], width, heads, kv, hw, 40, starts=2)
    inputs = [ids[n] for n in ("r", "pos", "starts", "Wq", "Wk", "Wv", "Wo", "g1", "gq", "gk")]
    feeds = feeds_of(g, inputs, 12, pos=of_each(starts, starts[-1]), starts=starts)
    whole = interp.run_function(g.desc, inputs, [ids["r2"]], feeds)[0]
    by = {g.desc["tensors"][t]["name"]: (a, g.desc["tensors"][t]["dtype"]) for t, a in zip(inputs, feeds)}
    ws = B.Workspace()

    def put(name, a, dtype):
        t = to_gpu(a, dtype).cpu()
        ws.feed(name, B.DTYPES[dtype], list(t.shape), t.data_ptr())

    for n in ("Wq", "Wk", "Wv", "Wo", "gain1", "gain_q", "gain_k"):
        put(n, *by[n])
    for n in ("keys", "values"):
        put(n, np.full((pool * page, kv * hw), np.nan), "bf16")          # nothing that was not written is read
    put("pages", np.random.default_rng(2).permutation(pool)[:2 * most].reshape(2, most).astype(np.int32), "i32")
    rows_of = [[starts[s] + t for t in range(n)] for s, n in enumerate(prompts)]
    steps = [(rows_of[0] + rows_of[1], prompts)] + [([starts[s] + prompts[s] + k for s in range(2)], [n + k + 1 for n in prompts]) for k in range(more)]
    for at, now in steps:
        c, cids = wl.attention_step(len(at), 2, width, heads, kv, hw, page, most, pool)
        here = "_%d" % len(at)              # a name of the workspace has one shape
        for n in ("r", "pos"):
            c.desc["tensors"][cids[n]]["name"] = n + here
        names = ["r", "pos", "keys", "values", "pages", "lengths"] + (["starts"] if len(at) != 2 else []) + ["Wq", "Wk", "Wv", "Wo", "g1", "gq", "gk"]
        f = B.Graph.from_desc(c.desc).function([cids[n] for n in names], [cids["r2"], cids["new_keys"], cids["new_values"]])
        assert f.can_alias(2, 1) and f.can_alias(3, 2)
        put("r" + here, by["r"][0][at], "bf16")
        put("pos" + here, by["pos"][0][at], "i32")
        put("lengths", np.asarray(now, np.int32), "i32")
        if len(at) != 2:
            put("starts", np.asarray([0, prompts[0], sum(prompts)], np.int32), "i32")
        ws.run(f, ["r2" + here, "keys", "values"])
        t = torch.empty([len(at), width], dtype=torch.bfloat16)
        ws.fetch("r2" + here, t.data_ptr(), t.numel() * 2)
        torch.cuda.synchronize()
        assert f.status() == 0
        assert far(t.double().numpy(), whole[at]) <= FAR


def kinds_of(f):
    return [line.split("[")[0].split(" ")[0] for line in f.describe().splitlines() if line[0] != " "]


def test_plans_of_the_layer():
    g, ids = wl.attention_layer(64, 64, 4, 2, 32, 40)
    inputs = [ids[n] for n in ("r", "pos", "labels")] + ids["weights"]
    kinds = kinds_of(B.Graph.from_desc(g.desc).function(inputs, [ids["loss"]] + ids["grads"]))
    assert [kinds.count(k) for k in ("head_norm+rotate", "head_norm+rotate_bwd", "attention", "attention_bwd")] == [1, 1, 1, 1]      # queries and keys together
    g, ids = wl.attention_step(3, 3, 64, 4, 2, 32, 16, 4, 12)
    names = ("r", "pos", "keys", "values", "pages", "lengths", "Wq", "Wk", "Wv", "Wo", "g1", "gq", "gk")
    kinds = kinds_of(B.Graph.from_desc(g.desc).function([ids[n] for n in names], [ids["r2"], ids["new_keys"], ids["new_values"]]))
    assert [kinds.count(k) for k in ("head_norm+rotate", "cache_write", "paged_attention")] == [1, 1, 1]
