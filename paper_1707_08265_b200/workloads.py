"""Seeded synthetic graphs and tensors for the five benchmark workloads.

This module holds no arithmetic of the method: it only writes graph
descriptions (plain dicts, the format documented in ``GraphDesc``) and draws
input values.  Both the CUDA library's tests and the CPU checker are driven
from these descriptions, so it imports neither.

Workloads (sizes are arguments so that tests can shrink them):
  toy_function        f = x*sin(a*x+b) and y = a*x, the example of Sec. 2.2
  toy_function_grad   the same with the gradient stage objs={f}, wrts={x,a,b} (Sec. 2.3)
  random_dag          random elementwise DAG (64 operators over 4 inputs by default)
  mlp                 InnerProduct/BiasAdd/ReLU/InnerProduct/BiasAdd/SoftmaxCrossEntropy
                      with an unused Tanh side branch and gradients for weights and biases
  random_row_dag      random broadcast/row-reduction DAG over [R,C] and [C] tensors, with
                      gradients for every input
  recurrent_layer     RMSNorm / InnerProduct / GatedScan / InnerProduct with a residual stream, RMSNorm, InnerProduct,
                      SoftmaxCrossEntropy, with gradients for every weight (a language model's layer and its loss)
  recurrent_step      the same layer one row per sequence with its weights in e4m3 (RMSNorm with 8-bit output,
                      ScaledInnerProduct, GatedScan from fed states): a decoding step
  attention_layer     RMSNorm / InnerProduct / HeadNorm / Rotate / Attention / InnerProduct with a residual stream, RMSNorm,
                      InnerProduct, SoftmaxCrossEntropy, with gradients for every weight
  attention_step      the same layer over a paged cache (CacheWrite, PagedAttention): single tokens, or chunks of new ones
  clipped_updater     W' = W - lr * clipped gradient for several weights under one global norm
"""
import numpy as np

BASE_SEED = 170708265

UNARY = ("Sin", "Exp", "Tanh", "Sigmoid", "ReLU")
BINARY = ("Add", "Sub", "Mul", "Div")
ROWRED = ("Sum", "Mean")


class GraphDesc:
    """Builder of the neutral graph description.

    ``desc`` = {"tensors": [{"name","dtype","shape"}], "ops": [{"type","in","out"}],
    "grads": [{"objs","wrts","grad_ids"}]}; ids are list positions (creation order).  An operator
    with numbers of its own (eps, block rows, limit, sequences) has them as "attrs".
    """

    def __init__(self):
        self.desc = {"tensors": [], "ops": [], "grads": []}

    def tensor(self, name, shape, dtype="f32"):
        self.desc["tensors"].append({"name": name, "dtype": dtype, "shape": [int(s) for s in shape]})
        return len(self.desc["tensors"]) - 1

    def shape(self, t):
        return self.desc["tensors"][t]["shape"]

    def op(self, type_, ins, out_name, out_shape=None, out_dtype="f32", attrs=()):
        if out_shape is None:
            out_shape = _broadcast_shape([self.shape(i) for i in ins])
        o = self.tensor(out_name, out_shape, out_dtype)
        self.desc["ops"].append({"type": type_, "in": [int(i) for i in ins], "out": [o]})
        if attrs:
            self.desc["ops"][-1]["attrs"] = [float(a) for a in attrs]
        return o

    def grad(self, objs, wrts, dtypes=None):
        """dtypes: the gradients' types, "f32" or "bf16" (None: "f32" throughout)."""
        gids = []
        s = len(self.desc["grads"])
        for w, dt in zip(wrts, dtypes or ["f32"] * len(wrts)):
            t = self.desc["tensors"][w]
            gids.append(self.tensor("grad%d/%s" % (s, t["name"]), t["shape"], dt))
        self.desc["grads"].append({"objs": list(objs), "wrts": list(wrts), "grad_ids": gids})
        return gids


def _broadcast_shape(shapes):
    rank = max(len(s) for s in shapes)
    out = [1] * rank
    for s in shapes:
        s = [1] * (rank - len(s)) + list(s)
        for k, d in enumerate(s):
            if d != 1:
                assert out[k] in (1, d), shapes
                out[k] = d
    return out


def toy_function(n):
    """Sec. 2.2: tensors x, a, b, t1 = a*x (this is y), t2 = t1+b, t3 = sin(t2), f = x*t3."""
    g = GraphDesc()
    x = g.tensor("x", [n])
    a = g.tensor("a", [])
    b = g.tensor("b", [])
    y = g.op("Mul", [a, x], "y")
    t2 = g.op("Add", [y, b], "t2")
    t3 = g.op("Sin", [t2], "t3")
    f = g.op("Mul", [x, t3], "f")
    return g, {"x": x, "a": a, "b": b, "y": y, "t2": t2, "t3": t3, "f": f}


def toy_function_grad(n):
    g, ids = toy_function(n)
    dx, da, db = g.grad([ids["f"]], [ids["x"], ids["a"], ids["b"]])
    ids.update(dx=dx, da=da, db=db)
    return g, ids


def toy_feeds(n, seed):
    rng = np.random.default_rng(seed)
    x = rng.uniform(-4.0, 4.0, size=n).astype(np.float32)
    a = np.float32(rng.standard_normal())
    b = np.float32(rng.standard_normal())
    return x, np.asarray(a, dtype=np.float32), np.asarray(b, dtype=np.float32)


def random_dag(n, seed, n_inputs=4, n_ops=64, n_fetch=2):
    """Random elementwise DAG: operator types uniform over BINARY+UNARY, each operand uniform
    over the inputs and the earlier operator nodes; fetches are drawn without replacement
    among operator nodes that nothing consumes."""
    rng = np.random.default_rng(seed)
    g = GraphDesc()
    nodes = [g.tensor("in%d" % k, [n]) for k in range(n_inputs)]
    inputs = list(nodes)
    kinds = BINARY + UNARY
    for k in range(n_ops):
        t = kinds[int(rng.integers(len(kinds)))]
        nin = 2 if t in BINARY else 1
        ins = [nodes[int(rng.integers(len(nodes)))] for _ in range(nin)]
        nodes.append(g.op(t, ins, "n%d" % k))
    consumed = {i for op in g.desc["ops"] for i in op["in"]}
    sinks = [t for t in nodes[n_inputs:] if t not in consumed]
    pick = rng.choice(len(sinks), size=min(n_fetch, len(sinks)), replace=False)
    fetch = [sinks[int(p)] for p in sorted(pick)]
    return g, inputs, fetch


def normal_feeds(shapes, seed):
    rng = np.random.default_rng(seed)
    return [rng.standard_normal(size=s, dtype=np.float32) for s in shapes]


def mlp(batch, d_in, d_hidden, d_out):
    """Two-layer perceptron with a side branch Tanh(X) that no target needs."""
    g = GraphDesc()
    X = g.tensor("X", [batch, d_in], "bf16")
    W1 = g.tensor("W1", [d_hidden, d_in], "bf16")
    b1 = g.tensor("b1", [d_hidden], "bf16")
    W2 = g.tensor("W2", [d_out, d_hidden], "bf16")
    b2 = g.tensor("b2", [d_out], "bf16")
    labels = g.tensor("labels", [batch], "i32")
    side = g.op("Tanh", [X], "side", out_dtype="bf16")
    z1 = g.op("InnerProduct", [X, W1], "z1", [batch, d_hidden], "f32")
    a1 = g.op("BiasAdd", [z1, b1], "a1", [batch, d_hidden], "f32")
    h = g.op("ReLU", [a1], "h", out_dtype="bf16")
    z2 = g.op("InnerProduct", [h, W2], "z2", [batch, d_out], "f32")
    z = g.op("BiasAdd", [z2, b2], "z", [batch, d_out], "bf16")
    loss = g.op("SoftmaxCrossEntropy", [z, labels], "loss", [], "f32")
    dW1, db1, dW2, db2 = g.grad([loss], [W1, b1, W2, b2])
    ids = dict(X=X, W1=W1, b1=b1, W2=W2, b2=b2, labels=labels, side=side, z1=z1, a1=a1, h=h,
               z2=z2, z=z, loss=loss, dW1=dW1, db1=db1, dW2=dW2, db2=db2)
    return g, ids


def mlp_feeds(batch, d_in, d_hidden, d_out, seed):
    """float32 arrays holding bf16-representable values (truncated mantissas), plus int32 labels."""
    rng = np.random.default_rng(seed)

    def bf16able(a):
        u = a.astype(np.float32).view(np.uint32)
        return ((u + 0x8000) & 0xFFFF0000).astype(np.uint32).view(np.float32)

    X = bf16able(rng.standard_normal(size=(batch, d_in), dtype=np.float32))
    W1 = bf16able(rng.standard_normal(size=(d_hidden, d_in), dtype=np.float32) / np.float32(np.sqrt(d_in)))
    b1 = bf16able(rng.standard_normal(size=(d_hidden,), dtype=np.float32) / np.float32(np.sqrt(d_in)))
    W2 = bf16able(rng.standard_normal(size=(d_out, d_hidden), dtype=np.float32) / np.float32(np.sqrt(d_hidden)))
    b2 = bf16able(rng.standard_normal(size=(d_out,), dtype=np.float32) / np.float32(np.sqrt(d_hidden)))
    labels = rng.integers(0, d_out, size=batch).astype(np.int32)
    return X, W1, b1, W2, b2, labels


def random_row_dag(rows, cols, seed, n_full=6, n_row=2, n_ops=1024, n_fetch=4):
    """Random DAG over FULL [rows, cols] and ROW [cols] tensors; operator types uniform over
    BINARY+UNARY+ROWRED; fetches drawn among FULL-shaped operator nodes nothing consumes.
    The gradient stage (objs = fetches, wrts = the inputs connected to a fetch) is attached by
    the caller with ``g.grad(fetch, wrts)``: which inputs are connected is the pruner's
    business, and this module holds none of it."""
    rng = np.random.default_rng(seed)
    g = GraphDesc()
    nodes = [g.tensor("full%d" % k, [rows, cols]) for k in range(n_full)]
    nodes += [g.tensor("row%d" % k, [cols]) for k in range(n_row)]
    inputs = list(nodes)
    kinds = BINARY + UNARY + ROWRED
    for k in range(n_ops):
        t = kinds[int(rng.integers(len(kinds)))]
        nin = 2 if t in BINARY else 1
        ins = [nodes[int(rng.integers(len(nodes)))] for _ in range(nin)]
        nodes.append(g.op(t, ins, "n%d" % k))
    consumed = {i for op in g.desc["ops"] for i in op["in"]}
    sinks = [t for t in nodes[len(inputs):] if t not in consumed and len(g.shape(t)) == 2]
    pick = rng.choice(len(sinks), size=min(n_fetch, len(sinks)), replace=False)
    fetch = [sinks[int(p)] for p in sorted(pick)]
    return g, inputs, fetch


def updater(shape, kind="sgd"):
    """The weight update as a graph of its own (Sec. 3.2 of the paper: the updater is split from the
    training graph so that neither becomes cyclic; it names Momentum, RMSProp and Adam).
      sgd:      W' = W - lr*g
      momentum: v' = mu*v + g,  W' = W - lr*v'
      rmsprop:  v' = rho*v + (1-rho)*g*g,  W' = W - lr * g / (sqrt(v') + eps)
      adam:     m' = beta1*m + (1-beta1)*g,  v' = beta2*v + (1-beta2)*g*g,  W' = W - lr * m' / (sqrt(v') + eps)
                (lr and eps carry the bias corrections of the step: lr_t = lr*sqrt(1-beta2^t)/(1-beta1^t))
    The hyper-parameters are scalar tensors, 1-x fed beside x; returns (graph, ids)."""
    g = GraphDesc()
    ids = {"W": g.tensor("W", shape), "g": g.tensor("g", shape)}

    def scalars(*names):
        for n in names:
            ids[n] = g.tensor(n, [])

    def decayed(state, keep, mix, value, name):      # keep*state + mix*value
        return g.op("Add", [g.op("Mul", [ids[keep], ids[state]], name + "_keep"), g.op("Mul", [ids[mix], value], name + "_mix")], name)

    if kind == "sgd":
        scalars("lr")
        step = g.op("Mul", [ids["lr"], ids["g"]], "step")
    elif kind == "momentum":
        ids["lr"] = g.tensor("lr", [])
        ids["v"] = g.tensor("v", shape)
        ids["mu"] = g.tensor("mu", [])
        ids["v_new"] = g.op("Add", [g.op("Mul", [ids["mu"], ids["v"]], "mv"), ids["g"]], "v_new")
        step = g.op("Mul", [ids["lr"], ids["v_new"]], "step")
    elif kind in ("rmsprop", "adam"):
        if kind == "adam":
            ids["m"] = g.tensor("m", shape)
        ids["v"] = g.tensor("v", shape)
        if kind == "adam":
            scalars("lr", "beta1", "one_minus_beta1", "beta2", "one_minus_beta2", "eps")
            ids["m_new"] = decayed("m", "beta1", "one_minus_beta1", ids["g"], "m_new")
            num, keep, mix = ids["m_new"], "beta2", "one_minus_beta2"
        else:
            scalars("lr", "rho", "one_minus_rho", "eps")
            num, keep, mix = ids["g"], "rho", "one_minus_rho"
        ids["v_new"] = decayed("v", keep, mix, g.op("Mul", [ids["g"], ids["g"]], "g2"), "v_new")
        den = g.op("Add", [g.op("Sqrt", [ids["v_new"]], "root"), ids["eps"]], "den")
        step = g.op("Mul", [g.op("Mul", [ids["lr"], num], "lr_num"), g.op("Reciprocal", [den], "inv")], "step")
    else:
        raise ValueError(kind)
    ids["W_new"] = g.op("Sub", [ids["W"], step], "W_new")
    return g, ids


def recurrent_layer(seqs, length, width, inner, vocab, resets=False):
    """One layer over ``seqs`` sequences of ``length`` rows and the loss behind it:
      y = RMSNorm(r; g1),  h = GatedScan(y Wf^T, y Wx^T; h0),  r2 = r + h Wo^T,  z = RMSNorm(r2; g2) Wv^T,  loss(z, labels)
    r: the residual stream, bf16 [rows, width].  Returns (graph, ids); ids["grads"]: gradients of (Wf, Wx, Wo, Wv, g1, g2, h0)."""
    g, rows = GraphDesc(), seqs * length
    ids = {"r": g.tensor("r", [rows, width], "bf16"), "h0": g.tensor("h0", [seqs, inner])}
    if resets:
        ids["reset"] = g.tensor("reset", [rows], "i32")
    for n, sh in (("Wf", [inner, width]), ("Wx", [inner, width]), ("Wo", [width, inner]), ("Wv", [vocab, width])):
        ids[n] = g.tensor(n, sh, "bf16")
    ids["g1"], ids["g2"] = g.tensor("gain1", [width]), g.tensor("gain2", [width])
    ids["labels"] = g.tensor("labels", [rows], "i32")
    y = g.op("RMSNorm", [ids["r"], ids["g1"]], "y", [rows, width], "bf16")
    f = g.op("InnerProduct", [y, ids["Wf"]], "f", [rows, inner], "bf16")
    x = g.op("InnerProduct", [y, ids["Wx"]], "x", [rows, inner], "bf16")
    h = g.op("GatedScan", [f, x, ids["h0"]] + ([ids["reset"]] if resets else []), "h", [rows, inner], "bf16", attrs=[seqs])
    o = g.op("InnerProduct", [h, ids["Wo"]], "o", [rows, width])
    ids["r2"] = g.op("Add", [o, ids["r"]], "r2", [rows, width], "bf16")
    y2 = g.op("RMSNorm", [ids["r2"], ids["g2"]], "y2", [rows, width], "bf16")
    z = g.op("InnerProduct", [y2, ids["Wv"]], "z", [rows, vocab])
    ids["loss"] = g.op("SoftmaxCrossEntropy", [z, ids["labels"]], "loss", [])
    ids["weights"] = [ids[n] for n in ("Wf", "Wx", "Wo", "Wv", "g1", "g2", "h0")]
    ids["grads"] = g.grad([ids["loss"]], ids["weights"])
    return g, ids


def recurrent_step(seqs, width, inner):
    """One decoding step of the layer for ``seqs`` sequences, its weights in e4m3 with scales of 128 x 128 blocks:
    r2 = r + GatedScan(y Wf^T, y Wx^T; states) Wo^T with y and the new states in e4m3 with scales of 1 x 128 blocks."""
    g = GraphDesc()

    def blocks(n):
        return -(-n // 128)

    ids = {"r": g.tensor("r", [seqs, width], "bf16"), "g1": g.tensor("gain1", [width]), "states": g.tensor("states", [seqs, inner])}
    for n, sh in (("Wf", [inner, width]), ("Wx", [inner, width]), ("Wo", [width, inner])):
        ids[n], ids["s" + n] = g.tensor(n, sh, "f8e4m3"), g.tensor("s" + n, [blocks(sh[0]), blocks(sh[1])])

    def product(x, out):
        s = g.op("BlockScale", [x], "s_" + out, [seqs, blocks(g.shape(x)[1])])
        q = g.op("Quantize", [x, s], "q_" + out, g.shape(x), "f8e4m3")
        return lambda n, o, dt: g.op("ScaledInnerProduct", [q, s, ids[n], ids["s" + n]], o, [seqs, g.shape(ids[n])[0]], dt)

    y = g.op("RMSNorm", [ids["r"], ids["g1"]], "y", [seqs, width])
    of_y = product(y, "y")
    f, x = of_y("Wf", "f", "f32"), of_y("Wx", "x", "f32")
    ids["new_states"] = g.op("GatedScan", [f, x, ids["states"]], "new_states", [seqs, inner], attrs=[seqs])
    o = product(ids["new_states"], "h")("Wo", "o", "f32")
    ids["r2"] = g.op("Add", [ids["r"], o], "r2", [seqs, width], "bf16")
    return g, ids


def _queries_keys_values(g, ids, rows, width, heads, kv_heads, head_width, interleaved):
    """y = RMSNorm(r; g1) and its products; queries and keys normalised head by head and turned by their positions."""
    ids["r"] = g.tensor("r", [rows, width], "bf16")
    for n, heads_of in (("Wq", heads), ("Wk", kv_heads), ("Wv", kv_heads)):
        ids[n] = g.tensor(n, [heads_of * head_width, width], "bf16")
    ids["Wo"] = g.tensor("Wo", [width, heads * head_width], "bf16")
    ids["g1"], ids["gq"], ids["gk"] = g.tensor("gain1", [width]), g.tensor("gain_q", [head_width]), g.tensor("gain_k", [head_width])
    ids["pos"] = g.tensor("pos", [rows], "i32")
    y = g.op("RMSNorm", [ids["r"], ids["g1"]], "y", [rows, width], "bf16")
    q, k, v = (g.op("InnerProduct", [y, ids["W" + n]], n, [rows, g.shape(ids["W" + n])[0]], "bf16") for n in "qkv")

    def turned(x, gain, name, count):
        u = g.op("HeadNorm", [x, gain], name + "_normed", g.shape(x))
        return g.op("Rotate", [u, ids["pos"]], name + "_turned", g.shape(x), "bf16", attrs=[count, head_width, interleaved])

    return turned(q, ids["gq"], "q", heads), turned(k, ids["gk"], "k", kv_heads), v


def attention_layer(rows, width, heads, kv_heads, head_width, vocab, sequences=1, starts=0, window=0, interleaved=0):
    """One layer over ``rows`` rows, those of ``sequences`` equally long sequences or (starts) of that many packed ones, and the loss:
      y = RMSNorm(r; g1),  q, k, v = y Wq^T, y Wk^T, y Wv^T,  a = Attention(Rotate(HeadNorm(q)), Rotate(HeadNorm(k)), v),
      r2 = r + a Wo^T,  z = RMSNorm(r2; g2) We^T,  loss(z, labels)
    r: the residual stream, bf16 [rows, width]; pos: every row's position.  Returns (graph, ids); ids["grads"]: gradients of ids["weights"]."""
    g, ids = GraphDesc(), {}
    q, k, v = _queries_keys_values(g, ids, rows, width, heads, kv_heads, head_width, interleaved)
    ids["We"], ids["g2"], ids["labels"] = g.tensor("We", [vocab, width], "bf16"), g.tensor("gain2", [width]), g.tensor("labels", [rows], "i32")
    ins = [q, k, v]
    if starts:
        ids["starts"] = g.tensor("starts", [starts + 1], "i32")
        ins.append(ids["starts"])
    a = g.op("Attention", ins, "a", [rows, heads * head_width], "bf16", attrs=[heads, kv_heads, 1, window, 0.0, sequences])
    o = g.op("InnerProduct", [a, ids["Wo"]], "o", [rows, width])
    ids["r2"] = g.op("Add", [o, ids["r"]], "r2", [rows, width], "bf16")
    y2 = g.op("RMSNorm", [ids["r2"], ids["g2"]], "y2", [rows, width], "bf16")
    z = g.op("InnerProduct", [y2, ids["We"]], "z", [rows, vocab])
    ids["loss"] = g.op("SoftmaxCrossEntropy", [z, ids["labels"]], "loss", [])
    ids["weights"] = [ids[n] for n in ("Wq", "Wk", "Wv", "Wo", "We", "g1", "gq", "gk", "g2")]
    ids["grads"] = g.grad([ids["loss"]], ids["weights"])
    return g, ids


def attention_step(rows, sequences, width, heads, kv_heads, head_width, page, most_pages, pool, window=0, interleaved=0):
    """The layer for ``rows`` new tokens of ``sequences`` sequences (one each, or those that starts gives) over a cache of ``pool``
    pages of ``page`` rows: the new keys and values go into the cache (ids["new_keys"], ids["new_values"]: fetched into the memory
    of keys and values they are written in place), the queries meet all that stands in it.  lengths counts the new tokens."""
    g, ids = GraphDesc(), {}
    cols = kv_heads * head_width
    q, k, v = _queries_keys_values(g, ids, rows, width, heads, kv_heads, head_width, interleaved)
    for n in ("keys", "values"):
        ids[n] = g.tensor(n, [pool * page, cols], "bf16")
    ids["pages"], ids["lengths"] = g.tensor("pages", [sequences, most_pages], "i32"), g.tensor("lengths", [sequences], "i32")
    table = [ids["pages"], ids["lengths"]]
    if rows != sequences:
        ids["starts"] = g.tensor("starts", [sequences + 1], "i32")
        table.append(ids["starts"])
    for n, new in (("keys", k), ("values", v)):
        ids["new_" + n] = g.op("CacheWrite", [ids[n], new] + table, "new_" + n, [pool * page, cols], "bf16", attrs=[page])
    a = g.op("PagedAttention", [q, ids["new_keys"], ids["new_values"]] + table, "a", [rows, heads * head_width], "bf16",
             attrs=[heads, kv_heads, page, window, 0.0])
    o = g.op("InnerProduct", [a, ids["Wo"]], "o", [rows, width])
    ids["r2"] = g.op("Add", [o, ids["r"]], "r2", [rows, width], "bf16")
    return g, ids


def clipped_updater(shapes, limit):
    """W_i' = W_i - lr * g_i * min(1, limit / norm(g_1, g_2, ...)) for every shape: the norm and the factor are one launch, the
    clipping is part of every update's own pass.  Returns (graph, ids) with lists W, g, W_new and the norm."""
    g = GraphDesc()
    ids = {"W": [g.tensor("W%d" % i, s) for i, s in enumerate(shapes)], "g": [g.tensor("g%d" % i, s) for i, s in enumerate(shapes)], "lr": g.tensor("lr", [])}
    ids["norm"] = g.op("GlobalNorm", ids["g"], "norm", [])
    ids["W_new"] = []
    for i, (w, d, s) in enumerate(zip(ids["W"], ids["g"], shapes)):
        c = g.op("ClipByNorm", [d, ids["norm"]], "clipped%d" % i, s, attrs=[limit])
        ids["W_new"].append(g.op("Sub", [w, g.op("Mul", [ids["lr"], c], "step%d" % i, s)], "W_new%d" % i, s))
    return g, ids
