"""HeadNorm and Rotate where they could go wrong: no eps, very large and very small heads, values that are not finite behind
the rotated elements, norms without a rotation behind them."""
import numpy as np
import pytest

from attention_cases import head_bounds, head_feeds, within
from lm_cases import run_gpu
from oracle import interp
from paper_1707_08265_b200 import workloads as wl

pytestmark = pytest.mark.gpu


def norm_graph(rows, heads, width, eps, x="f32", y="f32", rotate=True, dims=None, interleaved=0):
    """A norm, a rotation behind it where asked for, and the gradients of x and the gain."""
    g = wl.GraphDesc()
    shape = [rows, heads * width]
    t, gain = g.tensor("x", shape, x), g.tensor("gain", [width])
    inputs = [t, gain]
    last = g.op("HeadNorm", [t, gain], "u", shape, "f32" if rotate else y, attrs=[eps])
    if rotate:
        pos = g.tensor("pos", [rows], "i32")
        inputs.append(pos)
        last = g.op("Rotate", [last, pos], "y", shape, y, attrs=[heads, dims or width, interleaved])
    dy = g.tensor("dy", shape, y)
    inputs.append(dy)
    grads = g.grad([g.op("Mul", [last, dy], "along")], [t, gain], [x, "f32"])
    return g, inputs, [last] + grads


def check(g, inputs, outputs, feeds, size=1.0):
    """Outputs for heads that are `size` times the feeds' (a power of two: y and dgain are the same, dx 1 / size of it).  The bounds are
    taken where the feeds are; they say 1e-5 for eps, which moves them by that much of themselves."""
    bounds = head_bounds(g, inputs, outputs, feeds)
    sized = [feeds[0] * size] + feeds[1:]
    got, _ = run_gpu(g.desc, inputs, outputs, sized)
    want = interp.run_function(g.desc, inputs, outputs, sized)
    for n, t, a, b in zip(("u" if len(inputs) == 3 else "y", "dx", "dgain"), outputs, got, want):
        k = size if n == "dx" else 1.0
        assert within(a * k, b * k, 1.0001 * bounds[n], g.desc["tensors"][t]["dtype"]) <= 1, n


# heads that leave lanes of the last access without one, and lanes of a head without an element
@pytest.mark.parametrize("heads,width", [(1, 64), (3, 64), (5, 24), (1, 40), (2, 128), (4, 64), (1, 8)])
@pytest.mark.parametrize("rotate", [False, True])
@pytest.mark.parametrize("eps", [0.0, 1e-60])
def test_no_eps(heads, width, rotate, eps):
    g, inputs, outputs = norm_graph(70, heads, width, eps, rotate=rotate)
    check(g, inputs, outputs, head_feeds(g, inputs, heads + width))


@pytest.mark.parametrize("size", [2.0 ** 53, 2.0 ** 44, 2.0 ** -53, 2.0 ** -44])
@pytest.mark.parametrize("heads,width,rotate,x", [(3, 64, True, "f32"), (2, 128, True, "bf16"), (5, 72, False, "f32"), (8, 32, False, "bf16")])
def test_heads_far_from_one(size, heads, width, rotate, x):
    """Squares of up to 2^112 and down to 2^-112: in range, and so is every factor of the formula; the cube of the root is not."""
    g, inputs, outputs = norm_graph(33, heads, width, 0.0, x=x, y="f32", rotate=rotate)
    check(g, inputs, outputs, head_feeds(g, inputs, heads + width), size)


@pytest.mark.parametrize("heads,width,x,y", [(1, 64, "bf16", "bf16"), (3, 64, "f32", "f32"), (6, 80, "bf16", "bf16"), (32, 128, "bf16", "bf16"), (5, 256, "f32", "bf16"), (7, 8, "bf16", "f32")])
@pytest.mark.parametrize("rows", [1, 333])
def test_a_norm_alone_with_gradients(heads, width, x, y, rows):
    g, inputs, outputs = norm_graph(rows, heads, width, 1e-5, x=x, y=y, rotate=False)
    check(g, inputs, outputs, head_feeds(g, inputs, heads + rows))


def test_a_norm_that_a_rotation_and_something_else_read():
    """Its gradient is a sum: the rotation backwards and the norm backwards are passes of their own."""
    g = wl.GraphDesc()
    shape = [50, 3 * 40]
    x, gain, pos, dy, du = g.tensor("x", shape), g.tensor("gain", [40]), g.tensor("pos", [50], "i32"), g.tensor("dy", shape), g.tensor("du", shape)
    u = g.op("HeadNorm", [x, gain], "u", shape, "f32", attrs=[1e-5])
    y = g.op("Rotate", [u, pos], "y", shape, "f32", attrs=[3, 40])
    grads = g.grad([g.op("Mul", [y, dy], "along_y"), g.op("Mul", [u, du], "along_u")], [x, gain])
    inputs, outputs = [x, gain, pos, dy, du], [u, y] + grads
    feeds = head_feeds(g, inputs, 7)
    got, _ = run_gpu(g.desc, inputs, outputs, feeds)
    want = interp.run_function(g.desc, inputs, outputs, feeds)
    # a gradient of the norm of magnitude sqrt(2) |dy| + |du| at most: the bound for a dy of twice their sum
    h, h_in, h_out = norm_graph(50, 3, 40, 1e-5)
    b = head_bounds(h, h_in, h_out, feeds[:3] + [2 * (np.abs(feeds[3]) + np.abs(feeds[4]))])
    for n, a, w in zip(("u", "y", "dx", "dgain"), got, want):
        assert within(a, w, b[n], "f32") <= 1, n


def same_bits(a, b):
    return np.array_equal(a, b) and np.array_equal(np.signbit(a), np.signbit(b))


def copied_graph(rows, heads, width, dims, interleaved, norm, dt, grad=True):
    g = wl.GraphDesc()
    shape = [rows, heads * width]
    x, pos = g.tensor("x", shape, dt), g.tensor("pos", [rows], "i32")
    inputs, last = [x, pos], x
    if norm:
        gain = g.tensor("gain", [width])
        inputs.append(gain)
        last = g.op("HeadNorm", [x, gain], "u", shape, norm, attrs=[1e-5])
    y = g.op("Rotate", [last, pos], "y", shape, dt, attrs=[heads, dims, interleaved])
    if not grad:
        return g, inputs, [y]
    dy = g.tensor("dy", shape, dt)
    inputs.append(dy)
    return g, inputs, [y] + g.grad([g.op("Mul", [y, dy], "along")], [x], [dt])


# halves of 8 elements' lanes and others, neighbours, widths known when the kernel is compiled and others
COPIED = [(2, 64, 48, 0), (2, 64, 44, 0), (2, 64, 48, 1), (4, 128, 32, 0), (4, 128, 30, 1), (3, 40, 20, 0), (3, 40, 16, 0), (1, 256, 2, 1), (5, 80, 8, 0)]


@pytest.mark.parametrize("heads,width,dims,interleaved", COPIED)
@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [np.inf, -np.inf, np.nan])
def test_elements_behind_the_rotated_ones_are_copied(heads, width, dims, interleaved, dt, bad):
    """Whatever stands there: every other element keeps its bits, forwards and in the gradient."""
    g, inputs, outputs = copied_graph(19, heads, width, dims, interleaved, None, dt)
    feeds = head_feeds(g, inputs, width + dims)
    for k in (0, 2):
        feeds[k].reshape(19, heads, width)[:, :, -1] = -0.0
    clean, _ = run_gpu(g.desc, inputs, outputs, feeds)
    behind = np.zeros((19, heads, width), bool)
    behind[:, :, dims:] = True
    behind = behind.reshape(19, -1)
    for k, a in zip((0, 2), clean):
        assert same_bits(a[behind], feeds[k][behind])
    at = np.zeros((19, heads, width), bool)
    at[3, 0, dims] = at[4, heads - 1, width - 3] = at[18, 0, width - 2] = True
    at = at.reshape(19, -1)
    dirty = [f.copy() for f in feeds]
    dirty[0][at] = dirty[2][at] = bad
    got, _ = run_gpu(g.desc, inputs, outputs, dirty)
    for a, c in zip(got, clean):
        assert same_bits(a[~at], c[~at])
        assert np.isnan(a[at]).all() if np.isnan(bad) else (a[at] == bad).all()


@pytest.mark.parametrize("heads,width,dims,interleaved", COPIED)
@pytest.mark.parametrize("u", ["f32", "bf16"])
def test_an_infinity_behind_the_rotated_elements_of_a_normed_head(heads, width, dims, interleaved, u):
    """The head's root mean square is infinite then: the element itself is NaN, the others of the head are 0."""
    g, inputs, outputs = copied_graph(9, heads, width, dims, interleaved, u, "f32", grad=False)
    feeds = head_feeds(g, inputs, width + dims)
    clean, _ = run_gpu(g.desc, inputs, outputs, feeds)
    feeds[0].reshape(9, heads, width)[4, heads - 1, width - 2] = np.inf
    got, _ = run_gpu(g.desc, inputs, outputs, feeds)
    a, c = (t.reshape(9, heads, width) for t in (got[0], clean[0]))
    head = np.zeros((9, heads), bool)
    head[4, heads - 1] = True
    assert same_bits(a[~head], c[~head])
    assert np.isnan(a[4, heads - 1, width - 2]) and (np.delete(a[4, heads - 1], width - 2) == 0).all()
