"""Node-at-a-time interpreter of a pruned function: forward values and reverse-mode gradients.

TEST INFRASTRUCTURE ONLY (see oracle/__init__.py).

The paper fixes the graph model and the execution order (Sec. 3.2: kept forward
operators in creating order, gradient operators in inverse order) but gives no
operator semantics; those below are this project's reading of the operator
names.  Everything is evaluated with NumPy in ``dtype`` (float64 by default;
float32 gives the "CPU fp32 floor" used for conditioning checks), one whole
tensor per operator, no fusion, no reordering.

  Add, Sub, Mul      a+b, a-b, a*b with NumPy broadcasting
  Div(a, b)          a / (1 + |b|)
  Sin, Tanh, Sigmoid, ReLU   the usual; Exp(x) = exp(clip(x, -10, 10))
  Sqrt, Reciprocal   sqrt(x), 1/x (the updaters of Sec. 3.2 divide by a root: RMSProp, Adam)
  Sum, Mean          over the last axis, result broadcast back to the operand's shape
  InnerProduct(X, W) X[M,K] @ W[N,K]^T; operands are rounded to bf16 first (the
                     contraction consumes bf16), products and sums are wide
  BiasAdd(Y, b)      Y[m,n] + b[n]
  SoftmaxCrossEntropy(Z, labels)  scalar  -(1/M) sum_m log softmax(Z[m,:])[labels[m]]
  RMSNorm(h, g)      h / sqrt(mean(h^2) + eps) * g over rows
  BlockScale(x)      max(amax / 448, 2^-126) over blocks of rows x 128
  Quantize(x, s)     nearest e4m3 value (ties to even, magnitudes capped at 448) of x / s
  ScaledInnerProduct(Xq, sx, Wq, sw)  (Xq * sx) @ (Wq * sw)^T with the scales spread over their blocks
  GlobalNorm(t...)   sqrt of the sum of all squares; ClipByNorm(t, norm) = t * min(1, limit / norm)
  GatedScan(gate, x [, h0] [, reset])  row by row h = f*h + (1-f)*x, f = sigmoid(gate)
  HeadNorm(x, g)     every head of len(g) elements over its root mean square, times g
  Rotate(x, positions)  pairs of every head turned by position * frequency (the numbers: include/dragon.h)
  Attention(q, k, v [, starts])  softmax(scale q k^T) v inside every sequence, head by head (operands rounded to bf16)
  CacheWrite(cache, rows, pages, lengths [, starts])  the cache with the new rows in their places
  PagedAttention(q, kcache, vcache, pages, lengths [, starts])  the new rows of every sequence over its pages

Gradient rules (dy = gradient of the output): Add (dy,dy); Sub (dy,-dy);
Mul (dy*b, dy*a); Div (dy/(1+|b|), -dy*a*sgn(b)/(1+|b|)^2) with sgn(0)=0;
Sin dy*cos x; Exp dy*y*[-10<=x<=10]; Tanh dy*(1-y^2); Sigmoid dy*y*(1-y);
ReLU dy*[x>0]; Sqrt dy/(2y); Reciprocal -dy*y^2; Sum: row-sum of dy broadcast back; Mean: the same / C;
InnerProduct dX = dY@W, dW = dY^T@X (dY rounded to bf16 first);
BiasAdd (dy, column sums of dy); SoftmaxCrossEntropy dZ = dL*(softmax - onehot)/M.
A gradient with respect to a broadcast operand is summed over the broadcast
axes; contributions from several consumers add (reverse mode, Sec. 2.3); the
seed is one for every element of every objective of the stage.

A forward tensor declared bf16 is rounded to bf16 (round to nearest even, taken
on the float32 image of the value) when it is produced.
"""
import numpy as np

from .prune import function_sets


def round_bf16(a):
    """Round to bfloat16 (nearest even), result returned in the dtype of ``a``."""
    a = np.asarray(a)
    f = np.ascontiguousarray(a, dtype=np.float32)
    u = f.view(np.uint32).astype(np.uint64)
    lsb = (u >> 16) & 1
    r = ((u + 0x7FFF + lsb) >> 16) << 16
    nan = np.isnan(f)
    out = r.astype(np.uint32).view(np.float32)
    out = np.where(nan, np.float32(np.nan), out)
    return out.astype(a.dtype if a.dtype.kind == "f" else np.float32).reshape(a.shape)      # a scalar stays one


def _unbroadcast(g, shape):
    """Sum ``g`` over the axes along which a tensor of ``shape`` was broadcast."""
    shape = tuple(shape)
    while g.ndim > len(shape):
        g = g.sum(axis=0)
    for ax, (gs, ts) in enumerate(zip(g.shape, shape)):
        if ts == 1 and gs != 1:
            g = g.sum(axis=ax, keepdims=True)
    return g.reshape(shape)


def round_e4m3(a):
    """Nearest e4m3 value, ties to even: steps of 2^(e-3) with e >= -6, magnitudes capped at 448, NaN kept."""
    a = np.asarray(a, dtype=np.float64)
    _, e = np.frexp(a)
    step = np.exp2(np.maximum(e - 1, -6) - 3.0)
    with np.errstate(invalid="ignore"):
        return np.clip(np.rint(a / step) * step, -448.0, 448.0)


def _attr(op, default=None):
    return op["attrs"][0] if op.get("attrs") else default


def _spread(s, shape, rows):
    """Scales of rows x 128 blocks, one per element of a tensor of ``shape``."""
    return np.repeat(np.repeat(s, rows, axis=0)[:shape[0]], 128, axis=1)[:, :shape[1]]


def _scan_operands(op, ins):
    seqs = int(_attr(op, 1))
    rows, cols = ins[0].shape
    h0 = next((a for a in ins[2:] if a.dtype.kind == "f"), None)
    reset = next((a for a in ins[2:] if a.dtype.kind != "f"), None)
    length = rows // seqs
    shape = (seqs, length, cols)
    fresh = np.zeros((seqs, length), dtype=bool) if reset is None else (reset.reshape(seqs, length) != 0)
    start = np.zeros((seqs, cols), dtype=ins[0].dtype) if h0 is None else h0
    f = 1 / (1 + np.exp(-ins[0].reshape(shape)))
    keep = 1 / (1 + np.exp(ins[0].reshape(shape)))
    return f, keep, ins[1].reshape(shape), start, fresh


def _scan(op, ins):
    """(states, state in front of every row), both [sequences, rows, columns]."""
    f, keep, x, h, fresh = _scan_operands(op, ins)
    out, before = np.empty_like(x), np.empty_like(x)
    for t in range(x.shape[1]):
        before[:, t] = np.where(fresh[:, t, None], 0.0, h)
        h = f[:, t] * before[:, t] + keep[:, t] * x[:, t]
        out[:, t] = h
    return out, before


def _numbers(op, defaults):
    given = list(op.get("attrs") or [])
    return given + list(defaults)[len(given):]


def rotation(op, cols, positions, dtype=np.float64):
    """(cos, sin) [rows, pairs] with the amplitude, and the elements of a head that are first and second of a pair."""
    heads, dims, interleaved, base, factor, low, high, original, amplitude = _numbers(op, [1, 0, 0, 10000.0, 1.0, 0.0, 0.0, 0.0, 1.0])
    dims = int(dims) or cols // int(heads)
    i = np.arange(dims // 2)
    f = np.asarray(base, np.longdouble) ** (-2 * i.astype(np.longdouble) / dims)
    keep = np.zeros(dims // 2)
    if original > 0:
        turns = original * f / (2 * np.pi)
        keep = np.clip((turns - low) / (high - low), 0, 1) if high > low else (turns >= low).astype(np.float64)
    angle = positions.astype(np.longdouble)[:, None] * (f * (keep + (1 - keep) / factor))
    first = 2 * i if interleaved else i
    second = first + 1 if interleaved else i + dims // 2
    return (amplitude * np.cos(angle)).astype(dtype), (amplitude * np.sin(angle)).astype(dtype), first, second


def _rotate(op, x, positions, back=False):
    heads = int(op["attrs"][0])
    c, s, first, second = rotation(op, x.shape[1], positions, x.dtype)
    if back:
        s = -s
    h = x.reshape(x.shape[0], heads, -1)
    out = h.copy()
    a, b = h[..., first], h[..., second]
    out[..., first] = a * c[:, None] - b * s[:, None]
    out[..., second] = b * c[:, None] + a * s[:, None]
    return out.reshape(x.shape)


def sequence_rows(rows, sequences, starts):
    """[first, last) of every sequence."""
    if starts is None:
        return [(s * (rows // sequences), (s + 1) * (rows // sequences)) for s in range(sequences)]
    return [(int(a), int(b)) for a, b in zip(starts[:-1], starts[1:])]


def _softmax(x):
    """Over the last axis; zeros where all scores are -inf."""
    top = x.max(axis=-1, keepdims=True)
    e = np.exp(x - np.where(top == -np.inf, 0, top))
    total = e.sum(axis=-1, keepdims=True)
    return e / np.where(total == 0, 1, total)


def attention_parts(op, ins, bf16=True):
    """For every sequence and query head: (rows, columns of the head, columns of its key head, probabilities, scale)."""
    heads, kv_heads, causal, window, scale, sequences = _numbers(op, [1, 0, 1, 0, 0.0, 1])
    heads, kv_heads = int(heads), int(kv_heads) or int(heads)
    q, k = ins[0], ins[1]
    width = q.shape[1] // heads
    scale = scale or 1 / np.sqrt(width)
    for a, b in sequence_rows(q.shape[0], int(sequences), ins[3] if len(ins) > 3 else None):
        i = np.arange(b - a)
        seen = np.ones((b - a, b - a), bool)
        if causal:
            seen &= i[:, None] >= i
        if window:
            seen &= i[:, None] - i < window
        for h in range(heads):
            mine, theirs = slice(h * width, (h + 1) * width), slice(h // (heads // kv_heads) * width, (h // (heads // kv_heads) + 1) * width)
            x = np.where(seen, scale * (q[a:b, mine] @ k[a:b, theirs].T), -np.inf)
            yield slice(a, b), mine, theirs, _softmax(x) if b > a else x, scale


def cache_places(page, rows, pool, pages, lengths, starts):
    """For every row of the new tokens (sequence, position), and the row of the cache it has, -1 for none."""
    out = [(-1, -1, -1)] * rows
    for s, (a, b) in enumerate(sequence_rows(rows, len(lengths), starts)):
        for r in range(a, b):
            p = int(lengths[s]) - (b - a) + r - a
            ok = 0 <= p < pages.shape[1] * page and 0 <= pages[s, p // page] < pool // page
            out[r] = (s, p, int(pages[s, p // page]) * page + p % page if ok else -1)
    return out


def paged_parts(op, ins):
    """For every new row and query head that sees anything: (row, columns, columns of the key head, rows of the cache, probabilities)."""
    heads, kv_heads, page, window, scale = _numbers(op, [1, 0, 16, 0, 0.0])
    heads, kv_heads, page = int(heads), int(kv_heads) or int(heads), int(page)
    q, kc, pages, lengths = ins[0], ins[1], ins[3], ins[4]
    width = q.shape[1] // heads
    scale = scale or 1 / np.sqrt(width)
    for r, (s, p, _) in enumerate(cache_places(page, q.shape[0], kc.shape[0], pages, lengths, ins[5] if len(ins) > 5 else None)):
        if p < 0:
            continue
        j = np.arange(max(0, p - int(window) + 1) if window else 0, p + 1)
        at = pages[s, j // page] * page + j % page
        for h in range(heads):
            mine, theirs = slice(h * width, (h + 1) * width), slice(h // (heads // kv_heads) * width, (h // (heads // kv_heads) + 1) * width)
            x = scale * (kc[at, theirs] @ q[r, mine])
            yield r, mine, theirs, at, _softmax(x)


def _forward(op, ins, dtype, bf16_contraction=True):
    t = op["type"]
    if t == "HeadNorm":
        x = ins[0].reshape(ins[0].shape[0], -1, ins[1].shape[0])
        return (x / np.sqrt((x ** 2).mean(axis=-1, keepdims=True) + _attr(op, 1e-6)) * ins[1]).reshape(ins[0].shape)
    if t == "Rotate":
        return _rotate(op, ins[0], ins[1])
    if t == "Attention":
        rb = round_bf16 if bf16_contraction else (lambda a: a)
        ins = [rb(a) for a in ins[:3]] + list(ins[3:])
        y = np.zeros_like(ins[0])
        for rows, mine, theirs, p, _ in attention_parts(op, ins):
            y[rows, mine] = p @ ins[2][rows, theirs]
        return y
    if t == "CacheWrite":
        out = ins[0].copy()
        places = cache_places(int(_attr(op)), ins[1].shape[0], out.shape[0], ins[2], ins[3], ins[4] if len(ins) > 4 else None)
        for r, (_, _, at) in enumerate(places):
            if at >= 0:
                out[at] = ins[1][r]
        return out
    if t == "PagedAttention":
        q = round_bf16(ins[0]) if bf16_contraction else ins[0]
        y = np.zeros_like(q)
        for r, mine, theirs, at, p in paged_parts(op, [q] + list(ins[1:])):
            y[r, mine] = p @ ins[2][at, theirs]
        return y
    if t == "RMSNorm":
        return ins[0] / np.sqrt((ins[0] ** 2).mean(axis=-1, keepdims=True) + _attr(op, 1e-6)) * ins[1]
    if t == "BlockScale":
        rows = int(_attr(op, 1))
        R, C = ins[0].shape
        s = np.empty((-(-R // rows), -(-C // 128)), dtype=dtype)
        for i in range(s.shape[0]):
            for j in range(s.shape[1]):
                s[i, j] = max(np.abs(ins[0][i * rows:(i + 1) * rows, j * 128:(j + 1) * 128]).max() / 448, 2.0 ** -126)
        return s
    if t == "Quantize":
        return round_e4m3(ins[0] / _spread(ins[1], ins[0].shape, 1 if ins[1].shape[0] == ins[0].shape[0] else 128))
    if t == "ScaledInnerProduct":
        return (ins[0] * _spread(ins[1], ins[0].shape, 1)) @ (ins[2] * _spread(ins[3], ins[2].shape, 128)).T
    if t == "GlobalNorm":
        return np.asarray(np.sqrt(sum(float((a.astype(np.float64) ** 2).sum()) for a in ins)), dtype=dtype)
    if t == "ClipByNorm":
        limit = _attr(op)
        return ins[0] * (1.0 if ins[1] <= limit else limit / ins[1])      # (a NaN norm makes everything NaN)
    if t == "GatedScan":
        return _scan(op, ins)[0].reshape(ins[0].shape)
    if t == "Add":
        return ins[0] + ins[1]
    if t == "Sub":
        return ins[0] - ins[1]
    if t == "Mul":
        return ins[0] * ins[1]
    if t == "Div":
        return ins[0] / (1 + np.abs(ins[1]))
    if t == "Sin":
        return np.sin(ins[0])
    if t == "Exp":
        return np.exp(np.clip(ins[0], -10, 10))
    if t == "Tanh":
        return np.tanh(ins[0])
    if t == "Sigmoid":
        return 1 / (1 + np.exp(-ins[0]))
    if t == "ReLU":
        return np.maximum(ins[0], 0)
    if t == "Sqrt":
        return np.sqrt(ins[0])
    if t == "Reciprocal":
        return 1 / ins[0]
    if t == "Sum":
        return np.broadcast_to(ins[0].sum(axis=-1, keepdims=True), ins[0].shape).copy()
    if t == "Mean":
        return np.broadcast_to(ins[0].mean(axis=-1, keepdims=True), ins[0].shape).copy()
    if t == "InnerProduct":
        rb = round_bf16 if bf16_contraction else (lambda a: a)
        return rb(ins[0]) @ rb(ins[1]).T
    if t == "BiasAdd":
        return ins[0] + ins[1][None, :]
    if t == "SoftmaxCrossEntropy":
        z, lab = ins[0], ins[1].astype(np.int64)
        zs = z - z.max(axis=1, keepdims=True)
        lse = np.log(np.exp(zs).sum(axis=1))
        return np.asarray(-(zs[np.arange(z.shape[0]), lab] - lse).mean(), dtype=dtype)
    raise ValueError("unknown operator type %r" % t)


def _backward(op, ins, out, dy, pos, bf16_contraction=True):
    """Gradients with respect to the operand positions in ``pos`` (un-reduced, operand-broadcast)."""
    t = op["type"]
    g = {}
    if t == "HeadNorm":
        x = ins[0].reshape(ins[0].shape[0], -1, ins[1].shape[0])
        r = 1 / np.sqrt((x ** 2).mean(axis=-1, keepdims=True) + _attr(op, 1e-6))
        dy = dy.reshape(x.shape)
        for p in pos:
            d = dy * ins[1]
            g[p] = (r * d - x * r ** 3 * (d * x).mean(axis=-1, keepdims=True)).reshape(ins[0].shape) if p == 0 else (dy * x * r).sum(axis=(0, 1))
    elif t == "Rotate":
        g[0] = _rotate(op, dy, ins[1], back=True)
    elif t == "Attention":
        rb = round_bf16 if bf16_contraction else (lambda a: a)
        q, k, v = (rb(a) for a in ins[:3])
        dy = rb(dy)
        d = [np.zeros_like(q), np.zeros_like(k), np.zeros_like(v)]
        for rows, mine, theirs, p, scale in attention_parts(op, [q, k, v] + list(ins[3:])):
            do = dy[rows, mine]
            dp = do @ v[rows, theirs].T
            ds = scale * p * (dp - (p * dp).sum(axis=1, keepdims=True))
            d[0][rows, mine] = ds @ k[rows, theirs]
            d[1][rows, theirs] += ds.T @ q[rows, mine]
            d[2][rows, theirs] += p.T @ do
        for p in pos:
            g[p] = d[p]
    elif t == "RMSNorm":
        h, gain = ins
        r = 1 / np.sqrt((h ** 2).mean(axis=-1, keepdims=True) + _attr(op, 1e-6))
        for p in pos:
            d = dy * gain
            g[p] = r * d - h * r ** 3 * (d * h).mean(axis=-1, keepdims=True) if p == 0 else dy * h * r
    elif t == "GatedScan":
        f, keep, x, _, fresh = _scan_operands(op, ins)
        before = _scan(op, ins)[1]
        dh, total = dy.reshape(x.shape), np.empty_like(x)
        d = np.zeros_like(x[:, 0])
        for k in reversed(range(x.shape[1])):
            total[:, k] = dh[:, k] + d
            d = np.where(fresh[:, k, None], 0.0, total[:, k] * f[:, k])
        for p in pos:
            if p == 0:
                g[p] = (total * (before - x) * f * keep).reshape(ins[0].shape)
            elif p == 1:
                g[p] = (total * keep).reshape(ins[0].shape)
            else:
                g[p] = d
    elif t == "Add":
        for p in pos:
            g[p] = dy
    elif t == "Sub":
        for p in pos:
            g[p] = dy if p == 0 else -dy
    elif t == "Mul":
        for p in pos:
            g[p] = dy * ins[1 - p]
    elif t == "Div":
        den = 1 + np.abs(ins[1])
        for p in pos:
            g[p] = dy / den if p == 0 else -dy * ins[0] * np.sign(ins[1]) / (den * den)
    elif t == "Sin":
        g[0] = dy * np.cos(ins[0])
    elif t == "Exp":
        g[0] = dy * out * ((ins[0] >= -10) & (ins[0] <= 10))
    elif t == "Tanh":
        g[0] = dy * (1 - out * out)
    elif t == "Sigmoid":
        g[0] = dy * out * (1 - out)
    elif t == "ReLU":
        g[0] = dy * (ins[0] > 0)
    elif t == "Sqrt":
        g[0] = dy / (2 * out)
    elif t == "Reciprocal":
        g[0] = -dy * out * out
    elif t in ("Sum", "Mean"):
        r = np.broadcast_to(np.broadcast_to(dy, ins[0].shape).sum(axis=-1, keepdims=True), ins[0].shape)
        g[0] = r / ins[0].shape[-1] if t == "Mean" else r.copy()
    elif t == "InnerProduct":
        rb = round_bf16 if bf16_contraction else (lambda a: a)
        d = rb(dy)
        for p in pos:
            g[p] = d @ rb(ins[1]) if p == 0 else d.T @ rb(ins[0])
    elif t == "BiasAdd":
        for p in pos:
            g[p] = dy if p == 0 else dy.sum(axis=0)
    elif t == "SoftmaxCrossEntropy":
        z, lab = ins[0], ins[1].astype(np.int64)
        zs = z - z.max(axis=1, keepdims=True)
        e = np.exp(zs)
        sm = e / e.sum(axis=1, keepdims=True)
        sm[np.arange(z.shape[0]), lab] -= 1
        g[0] = dy * sm / z.shape[0]
    else:
        raise ValueError("unknown operator type %r" % t)
    return g


def run_function(desc, inputs, outputs, feeds, dtype=np.float64, return_all=False,
                 bf16_contraction=True):
    """Evaluate ``function(inputs, outputs)`` on ``feeds`` (arrays, order of ``inputs``).

    Pruned inputs may be fed as None.  ``bf16_contraction=False`` switches off the bf16
    rounding of InnerProduct operands (used only by the finite-difference pins, which need
    a differentiable function).  Returns the fetched arrays in the order of
    ``outputs`` (and, with ``return_all``, the dict of every forward value and the
    per-stage gradient dicts as well).
    """
    tensors, ops, grads = desc["tensors"], desc["ops"], desc.get("grads", [])
    sets = function_sets(desc, inputs, outputs)
    val = {}
    for i, f in zip(inputs, feeds):
        if sets["marked"][i]:
            a = np.asarray(f)
            val[i] = a if tensors[i]["dtype"] == "i32" else a.astype(dtype)
            assert tuple(val[i].shape) == tuple(tensors[i]["shape"]), (i, val[i].shape)
    for k in sets["fwd_ops"]:                       # creating order
        op = ops[k]
        with np.errstate(over="ignore", invalid="ignore"):
            y = _forward(op, [val[i] for i in op["in"]], dtype, bf16_contraction)
        (o,) = op["out"]
        y = np.asarray(y, dtype=dtype)
        if tensors[o]["dtype"] == "bf16":
            y = round_bf16(y)
        assert tuple(y.shape) == tuple(tensors[o]["shape"]), (k, y.shape, tensors[o]["shape"])
        val[o] = y
    gval = [dict() for _ in grads]
    for s, g in enumerate(grads):
        for o in g["objs"]:
            gval[s][o] = np.ones(tensors[o]["shape"], dtype=dtype)
    for (s, k, pos) in sets["grad_ops"]:            # inverse order inside a stage
        op = ops[k]
        (o,) = op["out"]
        dy = gval[s][o]
        ins = [val[i] for i in op["in"]]
        wanted = {op["in"][q] for q in pos}           # Op(n, n): both positions contribute to dn
        contrib = _backward(op, ins, val[o], dy, [p for p, i in enumerate(op["in"]) if i in wanted],
                            bf16_contraction)
        for p, gp in contrib.items():
            x = op["in"][p]
            gp = _unbroadcast(np.asarray(gp, dtype=dtype), tensors[x]["shape"])
            gval[s][x] = gval[s][x] + gp if x in gval[s] else gp
    grad_node = {}
    for s, g in enumerate(grads):
        for w, gid in zip(g["wrts"], g["grad_ids"]):
            grad_node[gid] = (s, w)
    res = []
    for t in outputs:
        if t in grad_node:
            s, w = grad_node[t]
            res.append(gval[s][w])
        else:
            res.append(val[t])
    if return_all:
        return res, val, gval
    return res


def finite_difference(desc, inputs, feeds, objs, wrt, h=1e-6, bf16_contraction=True):
    """Central differences of sum(all elements of all objs) with respect to input ``wrt``, in fp64."""
    k = inputs.index(wrt)
    base = [None if f is None else np.array(f, dtype=np.float64 if np.asarray(f).dtype.kind == "f" else None)
            for f in feeds]
    x = base[k]
    g = np.zeros_like(x)
    flat, gflat = x.reshape(-1), g.reshape(-1)

    def total():
        return sum(float(np.sum(v)) for v in run_function(desc, inputs, list(objs), base,
                                                              bf16_contraction=bf16_contraction))

    for j in range(flat.size):
        old = flat[j]
        step = h * max(1.0, abs(old))
        flat[j] = old + step
        up = total()
        flat[j] = old - step
        dn = total()
        flat[j] = old
        gflat[j] = (up - dn) / (2 * step)
    return g
