"""Tensors whose element offsets pass 32 bits: the rows behind that border against plain arithmetic in fp64."""
import pytest

from lm_cases import U16, U32

pytestmark = pytest.mark.gpu

FAR = 1 << 32      # elements


def tensor(rows, cols, dtype, seed):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed)
    t = torch.empty(rows, cols, device="cuda", dtype=dtype)
    for r in range(0, rows, 1 << 16):
        t[r:r + (1 << 16)].normal_(generator=gen)
    return t


def function(build):
    from paper_1707_08265_b200 import binding as B
    g = B.Graph()
    return g.function(*build(g, B))


def free():
    import torch
    torch.cuda.synchronize()
    torch.cuda.empty_cache()


@pytest.mark.parametrize("cols", [16384, 12347])
def test_norm_scales_and_values_behind_32_bits(cols):
    import torch
    rows = FAR // cols + 300
    x, gain = tensor(rows, cols, torch.bfloat16, 1), torch.randn(cols, device="cuda")
    y, q = torch.empty(rows, cols, device="cuda", dtype=torch.bfloat16), torch.empty(rows, cols, device="cuda", dtype=torch.float8_e4m3fn)
    s = torch.empty(rows, -(-cols // 128), device="cuda")

    def build(g, B):
        a, w, b = g.add_tensor("x", B.BF16, [rows, cols]), g.add_tensor("g", B.F32, [cols]), g.add_tensor("y", B.BF16, [rows, cols])
        t, e = g.add_tensor("s", B.F32, list(s.shape)), g.add_tensor("q", B.F8E4M3, [rows, cols])
        g.add_op(B.OPS["RMSNorm"], [a, w], [b], [1e-6])
        g.add_op(B.OPS["BlockScale"], [a], [t], [1])
        g.add_op(B.OPS["Quantize"], [a, t], [e])
        return [a, w], [b, t, e]
    f = function(build)
    f.run_torch([x, gain], [y, s, q])
    assert f.status() == 0
    for sl in (slice(0, 40), slice(rows - 290, rows - 250), slice(rows - 40, rows)):
        v = x[sl].double()
        want = v / torch.sqrt((v * v).mean(1, keepdim=True) + 1e-6) * gain.double()
        assert ((y[sl].double() - want).abs() <= (U16 + 64 * U32) * want.abs()).all()
        scale = torch.nn.functional.pad(v.abs(), (0, -cols % 128)).view(v.shape[0], -1, 128).amax(2) / 448
        assert ((s[sl].double() - scale).abs() <= U32 * scale).all()
        p = v / s[sl].double().repeat_interleave(128, 1)[:, :cols]
        assert ((q[sl].double() - p).abs() <= p.abs() * 2.0 ** -4 + 2.0 ** -10 + 3 * U32 * p.abs()).all()
    del x, y, q, s
    free()


def test_clipping_behind_32_bits():
    import torch
    rows, cols = FAR // 16384 + 300, 16384
    x = tensor(rows, cols, torch.bfloat16, 2)
    norm, c = torch.empty((), device="cuda"), torch.empty_like(x)

    def build(g, B):
        a, n, b = g.add_tensor("x", B.BF16, [rows, cols]), g.add_tensor("n", B.F32, []), g.add_tensor("c", B.BF16, [rows, cols])
        g.add_op(B.OPS["GlobalNorm"], [a], [n])
        g.add_op(B.OPS["ClipByNorm"], [a, n], [b], [1000.0])
        return [a], [n, b]
    f = function(build)
    f.run_torch([x], [norm, c])
    assert f.status() == 0
    want = float(sum((x[r:r + 4096].double() ** 2).sum() for r in range(0, rows, 4096))) ** 0.5
    assert abs(float(norm) - want) <= 40 * U32 * want
    for sl in (slice(0, 40), slice(rows - 290, rows - 250), slice(rows - 40, rows)):
        v = x[sl].double() * (1000.0 / want)
        assert ((c[sl].double() - v).abs() <= (U16 + 60 * U32) * v.abs()).all()
    del x, c
    free()


@pytest.mark.parametrize("cols", [8192, 8191])
def test_scan_behind_32_bits(cols):
    """Sequences of 100 rows: the last ones against the same recurrence of these rows alone, forward and gradient."""
    import torch
    seqs = FAR // cols // 100 + 4
    rows = seqs * 100

    def make(n):
        def build(g, B):
            z, x, h, d = (g.add_tensor(t, B.BF16, [n * 100, cols]) for t in ("z", "x", "h", "d"))
            along = g.add_tensor("along", B.F32, [n * 100, cols])
            g.add_op(B.OPS["GatedScan"], [z, x], [h], [n])
            g.add_op(B.OPS["Mul"], [h, d], [along])
            return [z, x, d], [h] + g.add_grad([along], [x])
        return function(build)
    z, x, d = (tensor(rows, cols, torch.bfloat16, k) for k in (3, 4, 5))
    h, dx = torch.empty_like(x), torch.empty(rows, cols, device="cuda")
    f = make(seqs)
    f.run_torch([z, x, d], [h, dx])
    assert f.status() == 0
    last = slice(rows - 300, rows)
    h2, dx2 = torch.empty_like(h[last]), torch.empty_like(dx[last])
    make(3).run_torch([z[last].clone(), x[last].clone(), d[last].clone()], [h2, dx2])
    torch.cuda.synchronize()
    # the same rows fall into tiles at other places: sums of the same values in another grouping
    state, zz, xx = torch.zeros(3, cols, device="cuda", dtype=torch.float64), z[last].double().view(3, 100, cols), x[last].double().view(3, 100, cols)
    want = []
    for t in range(100):
        state = torch.sigmoid(zz[:, t]) * state + torch.sigmoid(-zz[:, t]) * xx[:, t]
        want.append(state)
    want = torch.stack(want, 1).view(300, cols)
    bound = 100 * 2 * (6 + 6) * U32 * 6 + U16 * want.abs()
    for a in (h[last], h2):
        assert ((a.double() - want).abs() <= bound).all()
    assert ((dx[last] - dx2).double().abs() <= 100 * 4 * 12 * U32 * 6).all()
    assert dx[last].abs().max() > 0.1
    del z, x, d, h, dx
    free()


def test_product_behind_32_bits():
    import torch
    M, N, K = FAR // 32768 + 300, 32768, 144
    gen = torch.Generator(device="cuda").manual_seed(6)
    xq, wq = ((torch.randn(r, K, device="cuda", generator=gen) * 100).clamp(-448, 448).to(torch.float8_e4m3fn) for r in (M, N))
    sx, sw = torch.rand(M, 2, device="cuda", generator=gen) + 0.1, torch.rand(N // 128, 2, device="cuda", generator=gen) + 0.1
    y = torch.empty(M, N, device="cuda", dtype=torch.bfloat16)

    def build(g, B):
        t = [g.add_tensor("xq", B.F8E4M3, [M, K]), g.add_tensor("sx", B.F32, [M, 2]), g.add_tensor("wq", B.F8E4M3, [N, K]), g.add_tensor("sw", B.F32, [N // 128, 2])]
        o = g.add_tensor("y", B.BF16, [M, N])
        g.add_op(B.OPS["ScaledInnerProduct"], t, [o])
        return t, [o]
    f = function(build)
    f.run_torch([xq, sx, wq, sw], [y])
    assert f.status() == 0
    w = wq.double() * sw.double().repeat_interleave(128, 0).repeat_interleave(128, 1)[:, :K]
    for sl in (slice(0, 40), slice(M - 290, M - 250), slice(M - 40, M)):
        x = xq[sl].double() * sx[sl].double().repeat_interleave(128, 1)[:, :K]
        want, mag = x @ w.T, x.abs() @ w.abs().T
        assert ((y[sl].double() - want).abs() <= U16 * want.abs() + (128 + 2 + 2) * U32 * mag).all()
    del y
    free()
