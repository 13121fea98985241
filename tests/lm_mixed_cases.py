"""Graphs in which the language-model operators meet each other and the older ones in orders other than a layer's own."""
import random

from oracle import prune
from paper_1707_08265_b200 import workloads as wl

SUM_READERS = ("scales of rows", "scales of tiles", "given scales", "norm over tensors", "clipped", "scan of it", "scan gated by it", "gain of another norm")


def sum_read_before_its_norm(reader, dtype, rows=70, cols=264):
    """h = Add(x, r), fetched; an operator that reads h; then RMSNorm(h).  Returns (graph, inputs, outputs: h, the reader's, y)."""
    g = wl.GraphDesc()
    shape = [cols] if reader == "gain of another norm" else [rows, cols]
    blocks = -(-cols // 128)
    x, r, w = g.tensor("x", shape, dtype), g.tensor("r", shape, dtype), g.tensor("w", [cols])
    inputs = [x, r, w]
    h = g.op("Add", [x, r], "h", shape, dtype)
    if reader == "scales of rows":
        s = g.op("BlockScale", [h], "s", [rows, blocks], attrs=[1])
        read = [s, g.op("Quantize", [h, s], "q", shape, "f8e4m3")]
    elif reader == "scales of tiles":
        read = [g.op("BlockScale", [h], "s", [-(-rows // 128), blocks], attrs=[128])]
    elif reader == "given scales":
        s = g.tensor("s", [rows, blocks])
        inputs.append(s)
        read = [g.op("Quantize", [h, s], "q", shape, "f8e4m3")]
    elif reader == "norm over tensors":
        read = [g.op("GlobalNorm", [x, h], "n", [])]
    elif reader == "clipped":
        n = g.op("GlobalNorm", [h], "n", [])
        read = [n, g.op("ClipByNorm", [h, n], "c", shape, dtype, attrs=[0.5])]
    elif reader == "gain of another norm":
        z = g.tensor("z", [3, cols])
        inputs.append(z)
        read = [g.op("RMSNorm", [z, h], "yz", [3, cols])]
    else:
        z = g.tensor("z", shape, dtype)
        inputs.append(z)
        read = [g.op("GatedScan", [z, h] if reader == "scan of it" else [h, z], "states", shape, dtype)]
    y = g.op("RMSNorm", [h, w], "y", shape, dtype)
    return g, inputs, [h] + read + [y]


def broadcast_gradient(kind, dtype="f32", rows=37, cols=264):
    """Gradients of tensors that a wider operator broadcasts: what reads them sums first.  Returns (graph, inputs, outputs)."""
    g = wl.GraphDesc()
    wide = g.tensor("M", [rows, cols])
    if kind in ("norm of a vector", "norm of one row", "norm of a sum", "norm of a vector, constant"):
        shape = [1, cols] if kind == "norm of one row" else [cols]
        x, w = g.tensor("x", shape, dtype), g.tensor("w", [cols])
        inputs, h = [x, w], x
        if kind == "norm of a sum":
            r = g.tensor("r", shape, dtype)
            inputs.append(r)
            h = g.op("Add", [x, r], "h", shape, dtype)
        y = g.op("RMSNorm", [h, w], "y", shape, dtype)
        objs = [g.op("Add" if kind.endswith("constant") else "Mul", [y, wide], "z")]
    elif kind == "scan of one row":
        x, gate, h0 = g.tensor("x", [1, cols], dtype), g.tensor("gate", [1, cols], dtype), g.tensor("h0", [1, cols])
        inputs = [gate, x, h0]
        objs = [g.op("Mul", [g.op("GatedScan", inputs, "h", [1, cols], dtype), wide], "z")]
    elif kind == "gain of two uses":        # the gain's gradient is [cols] from the norm, [rows, cols] from the product
        x, w = g.tensor("x", [5, cols], dtype), g.tensor("w", [cols])
        inputs = [x, w]
        objs = [g.op("RMSNorm", [x, w], "y", [5, cols], dtype), g.op("Mul", [wide, w], "z")]
    elif kind == "vector of two uses":      # operators that are all in the graph VM
        x = g.tensor("x", [cols], dtype)
        inputs = [x]
        objs = [g.op("Mul", [wide, x], "z"), g.op("Tanh", [x], "t")]
    elif kind == "objective of two uses":   # an objective counts once for each of its own elements
        x = g.tensor("x", [cols], dtype)
        inputs = [x]
        t = g.op("Tanh", [x], "t")
        objs = [t, g.op("Mul", [wide, t], "z")]
    elif kind == "scalar of two widths":    # gradients over two domains that do not broadcast against each other
        a, v = g.tensor("a", []), g.tensor("v", [rows + 1])
        inputs = [a, v]
        objs = [g.op("Mul", [wide, a], "z"), g.op("Mul", [v, a], "u")]
    elif kind == "product of one row":
        x, w = g.tensor("x", [1, 64], "bf16"), g.tensor("w", [cols, 64], "bf16")
        inputs = [x, w]
        objs = [g.op("Mul", [g.op("InnerProduct", [x, w], "y", [1, cols]), wide], "z")]
    elif kind == "loss":
        x, labels = g.tensor("x", [6, 40]), g.tensor("labels", [6], "i32")
        inputs = [x, labels]
        objs = [g.op("Mul", [g.op("SoftmaxCrossEntropy", [x, labels], "loss", []), wide], "z")]
    wrts = [t for t in inputs if g.desc["tensors"][t]["dtype"] != "i32"]
    return g, inputs + [wide], objs + g.grad(objs, wrts)


BROADCAST_KINDS = ("norm of a vector", "norm of one row", "norm of a sum", "norm of a vector, constant", "scan of one row", "gain of two uses", "vector of two uses",
                   "objective of two uses", "scalar of two widths", "product of one row", "loss")


def random_mixture(seed, rows=37, cols=264, n_ops=14, types=("f32",)):
    """A random graph of the language-model operators and the graph VM's over [rows, cols], [cols] and scalar tensors of the
    given types, values kept near one; some tensors fetched, gradients of some with respect to some.  Returns (graph, inputs,
    outputs, the outputs that are e4m3)."""
    rng = random.Random(seed)
    g = wl.GraphDesc()

    def dt():
        return types[0] if len(types) == 1 else rng.choice(types)

    big, vec = [rows, cols], [cols]
    wide = [g.tensor("x%d" % i, big, dt()) for i in range(3)]
    rowv = [g.tensor("v%d" % i, vec, dt()) for i in range(2)] + [g.tensor("one_row", [1, cols], dt())]
    h0 = g.tensor("h0", [1, cols], dt())
    inputs = wide + rowv + [h0]
    smooth = list(inputs)                      # tensors through which gradients pass
    made, eight, no_grad = [], [], []

    def name(t):
        return "%s_%d" % (t, len(made) + len(eight) + len(no_grad))

    kinds = ["Add", "Add", "Mul", "Tanh", "Sin", "RMSNorm", "RMSNorm", "GatedScan", "GatedScan", "vector norm", "row scan", "scales", "tiles", "GlobalNorm", "Clip", "Sum"]
    kinds += ["InnerProduct"] if cols % 8 == 0 else []      # (it takes rows of 16 bytes)
    for _ in range(n_ops):
        kind = rng.choice(kinds)
        a, b, v = rng.choice(wide), rng.choice(wide), rng.choice(rowv)
        if kind in ("Add", "Mul"):
            b = rng.choice([b, b, v])
            wide.append(g.op(kind, [a, b], name(kind), big, dt()))
        elif kind in ("Tanh", "Sin"):
            src = rng.choice([a, v])
            t = g.op(kind, [src], name(kind), g.shape(src), dt())
            (wide if g.shape(src) == big else rowv).append(t)
        elif kind == "RMSNorm":
            gain = rng.choice([t for t in rowv if g.shape(t) == vec])
            wide.append(g.op("RMSNorm", [a, gain], name(kind), big, dt(), attrs=[0.1]))
        elif kind == "vector norm":
            gain = rng.choice([t for t in rowv if g.shape(t) == vec])
            rowv.append(g.op("RMSNorm", [v, gain], name("vnorm"), g.shape(v), dt(), attrs=[0.1]))
        elif kind == "GatedScan":
            ins = [a, b] + ([h0] if rng.random() < 0.5 else [])
            wide.append(g.op("GatedScan", ins, name(kind), big, dt(), attrs=[1]))
        elif kind == "row scan":
            one = [t for t in rowv if g.shape(t) == [1, cols]]
            rowv.append(g.op("GatedScan", [rng.choice(one), rng.choice(one), h0], name("rowscan"), [1, cols], dt(), attrs=[1]))
        elif kind == "Sum":
            wide.append(g.op("Mean", [a], name("mean"), big, dt()))
        elif kind == "InnerProduct":
            p = g.op("InnerProduct", [a, b], name("prod"), [rows, rows], dt())
            no_grad.append(p)
        elif kind in ("scales", "tiles"):
            r = 1 if kind == "scales" else 128
            s = g.op("BlockScale", [a], name("s"), [-(-rows // r), -(-cols // 128)], attrs=[r])
            no_grad.append(s)
            eight.append(g.op("Quantize", [a, s], name("q"), big, "f8e4m3"))
        elif kind == "GlobalNorm":
            no_grad.append(g.op("GlobalNorm", rng.sample(wide, min(len(wide), 3)) + [v], name("norm"), []))
        else:
            n = g.op("GlobalNorm", [a, b], name("norm"), [])
            no_grad.append(n)
            c = g.op("ClipByNorm", [a, n], name("clip"), big, dt(), attrs=[20.0])
            no_grad.append(c if rng.random() < 0.5 else g.op("Sub", [b, c], name("upd"), big, dt()))
        made = [t for t in wide + rowv if t not in inputs]
    objs = rng.sample(made, min(len(made), 2))
    reached = [t for t in smooth if t in prune.backward_marks(g.desc, objs, smooth)]
    grads = g.grad(objs, rng.sample(reached, min(len(reached), 4))) if reached else []
    outputs = rng.sample(made, min(len(made), 3)) + rng.sample(no_grad, min(len(no_grad), 3)) + rng.sample(eight, min(len(eight), 1)) + grads
    return g, inputs, outputs, eight
