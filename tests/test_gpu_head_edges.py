"""HeadNorm and Rotate where they could go wrong: no eps, very large and very small heads."""
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
