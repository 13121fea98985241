"""Gradients in bf16 through the operators that were there before a caller could ask for them: products, norms, the recurrence, broadcast
sums and chains of additions.  They are the f32 gradients but for roundings to bf16."""
import numpy as np
import pytest

from lm_cases import as_type, run_gpu
from oracle import interp
from paper_1707_08265_b200 import workloads as wl

pytestmark = pytest.mark.gpu


def build(kind, x_type):
    """(graph, objectives, derivative targets, inputs): every target has a gradient of several contributions or a path of its own."""
    g = wl.GraphDesc()

    def t(name, shape, dt="f32"):
        return g.tensor(name, shape, dt)

    if kind == "product":
        x, w, v, d, e = t("x", [70, 64], x_type), t("w", [48, 64], "bf16"), t("v", [32, 48], "bf16"), t("d", [70, 32]), t("e", [70, 48])
        h = g.op("InnerProduct", [x, w], "h", [70, 48], "bf16")
        z = g.op("InnerProduct", [h, v], "z", [70, 32])
        return g, [g.op("Mul", [z, d], "along"), g.op("Mul", [h, e], "along_h")], [x, w, v], [x, w, v, d, e]
    if kind == "norm":
        x, r, gain, d = t("x", [50, 96], x_type), t("r", [50, 96], x_type), t("gain", [96]), t("d", [50, 96])
        h = g.op("Add", [x, r], "h", [50, 96], x_type)
        y = g.op("RMSNorm", [h, gain], "y", [50, 96], "bf16")
        return g, [g.op("Mul", [y, d], "along"), g.op("Mul", [h, d], "along_h")], [x, r, gain], [x, r, gain, d]
    if kind == "scan":
        gate, x, h0, d = t("gate", [60, 40], x_type), t("x", [60, 40], x_type), t("h0", [3, 40], x_type), t("d", [60, 40])
        h = g.op("GatedScan", [gate, x, h0], "h", [60, 40], "bf16", attrs=[3])
        return g, [g.op("Mul", [h, d], "along")], [gate, x, h0], [gate, x, h0, d]
    if kind == "broadcast":
        x, b, s, d = t("x", [90, 56], x_type), t("b", [56], x_type), t("s", [], "f32"), t("d", [90, 56])
        y = g.op("Mul", [g.op("BiasAdd", [x, b], "xb", [90, 56]), s], "y", [90, 56])
        return g, [g.op("Mul", [y, d], "along")], [x, b, s], [x, b, s, d]
    if kind == "additions":      # a chain of them, in front of a product: what reaches the targets is one gradient
        x, y, c, w, d = t("x", [33, 64], x_type), t("y", [33, 64], x_type), t("c", [33, 64], "f32"), t("w", [40, 64], "bf16"), t("d", [33, 40])
        a = g.op("Add", [x, y], "a", [33, 64], "bf16")
        b = g.op("Sub", [a, c], "b", [33, 64], "bf16")
        z = g.op("InnerProduct", [b, w], "z", [33, 40])
        return g, [g.op("Mul", [z, d], "along"), g.op("Mul", [a, c], "along_a")], [x, y, c], [x, y, c, w, d]
    x, w, b, labels = t("x", [64, 48], x_type), t("w", [40, 48], "bf16"), t("b", [40]), t("labels", [64], "i32")
    z = g.op("BiasAdd", [g.op("InnerProduct", [x, w], "xw", [64, 40]), b], "z", [64, 40])
    return g, [g.op("SoftmaxCrossEntropy", [z, labels], "loss", [])], [x, w, b], [x, w, b, labels]


@pytest.mark.parametrize("kind", ["product", "norm", "scan", "broadcast", "additions", "loss"])
@pytest.mark.parametrize("x_type", ["f32", "bf16"])
@pytest.mark.parametrize("which", ["all", "first", "others"])
def test_gradients_in_bf16(kind, x_type, which):
    def run(types, feeds=None):
        g, objs, wrts, inputs = build(kind, x_type)
        grads = g.grad(objs, wrts, types)
        if feeds is None:
            rng = np.random.default_rng(len(kind))
            feeds = []
            for i in inputs:
                info = g.desc["tensors"][i]
                feeds.append(rng.integers(0, 40, info["shape"]).astype(np.int32) if info["dtype"] == "i32" else as_type(rng.standard_normal(info["shape"]), info["dtype"]))
        got, _ = run_gpu(g.desc, inputs, grads, feeds)
        return got, interp.run_function(g.desc, inputs, grads, feeds), feeds

    wide, exact, feeds = run(["f32"] * 3)
    types = [("bf16" if which == "all" or (i == 0) == (which == "first") else "f32") for i in range(3)]
    got, _, _ = run(types, feeds)
    for i, (a, w, x, dt) in enumerate(zip(got, wide, exact, types)):
        assert np.array_equal(a, interp.round_bf16(a)) if dt == "bf16" else True
        # at most three roundings of 2^-8 more than the f32 gradient has (where a product or a sum leaves it, where contributions are
        # added, where it is written), each of an element of that tensor's gradient or of a contribution to it
        assert np.linalg.norm(a - w) <= 3 * 2.0 ** -8 * (np.linalg.norm(w) + np.linalg.norm(x)), i
        assert np.linalg.norm(a - x) <= np.linalg.norm(w - x) + 3 * 2.0 ** -8 * 2 * np.linalg.norm(x), i
