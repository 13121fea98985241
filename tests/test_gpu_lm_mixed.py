"""The graphs of lm_mixed_cases on the GPU against the fp64 oracle."""
import numpy as np
import pytest

from lm_cases import U16, U32, normals, run_gpu
from lm_mixed_cases import BROADCAST_KINDS, SUM_READERS, broadcast_gradient, random_mixture, sum_read_before_its_norm
from oracle import interp

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("reader", SUM_READERS)
def test_sum_that_is_read_before_its_norm(reader, dtype):
    g, inputs, outputs = sum_read_before_its_norm(reader, dtype)
    feeds = normals(g.desc, inputs, 11, {"r": 3.0})
    feeds = [np.abs(a) + 0.5 if g.desc["tensors"][t]["name"] == "s" else a for a, t in zip(feeds, inputs)]
    got, _ = run_gpu(g.desc, inputs, outputs, feeds)
    want = interp.run_function(g.desc, inputs, outputs, feeds)
    for t, a, b in zip(outputs, got, want):
        info = g.desc["tensors"][t]
        # of the largest value: 70 rows of the scan at (6 + |z|) 2^-23 each with |z| <= 16, 3080 U32, more than any of the sums
        # here; a rounding to bf16 that may go the other way is a step of 2^-7 of the value at most, one to e4m3 a step of 2^-3
        step = {"f32": 0.0, "bf16": 2 * U16, "f8e4m3": 2.0 ** -3}[info["dtype"]]
        assert np.abs(a - b).max() <= (3100 * U32 + step) * np.abs(b).max(), info["name"]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", BROADCAST_KINDS)
def test_gradient_of_a_broadcast_tensor(kind, dtype):
    g, inputs, outputs = broadcast_gradient(kind, dtype)
    feeds = normals(g.desc, inputs, 13)
    for i, t in enumerate(inputs):
        if g.desc["tensors"][t]["dtype"] == "i32":
            feeds[i] = np.arange(6, dtype=np.int32) * 5
    got, _ = run_gpu(g.desc, inputs, outputs, feeds)
    want = interp.run_function(g.desc, inputs, outputs, feeds)
    for t, a, b in zip(outputs, got, want):
        info = g.desc["tensors"][t]
        # of the largest value: sums of at most 10000 terms in trees of 64 or fewer roundings, and twice that for cancellation
        # between them; every value may pass three roundings to bf16 that go the other way (of y, of dy and its own)
        rounded = 0.0 if dtype == "f32" and kind != "product of one row" else 6 * U16
        assert np.abs(a - b).max() <= (1000 * U32 + rounded) * max(np.abs(b).max(), 1e-30), info["name"]


# an operator's own error, relative to the largest value: the scan's 37 rows at (6 + |z|) 2^-23 with |z| <= 16, all others below;
# up to 14 of them one behind another
CHAIN = 14 * 37 * 22 * 2 * U32


@pytest.mark.parametrize("seed", range(80))
def test_random_mixture_of_operators(seed):
    g, inputs, outputs, eight = random_mixture(seed)
    feeds = normals(g.desc, inputs, seed)
    want, val, _ = interp.run_function(g.desc, inputs, outputs, feeds, return_all=True)
    got, f = run_gpu(g.desc, inputs, outputs, feeds)
    by_output = {op["out"][0]: op for op in g.desc["ops"]}
    for t, a, b in zip(outputs, got, want):
        what = "%s of\n%s" % (g.desc["tensors"][t]["name"], f.describe())
        if t in eight:            # a value next to a midpoint may become the neighbour: a step is an 8th of it at most, 2^-9 at least
            assert (np.abs(a - b) <= np.maximum(np.abs(b) * 2.0 ** -3, 2.0 ** -9)).all(), what
        elif t in by_output and by_output[t]["type"] == "InnerProduct":      # operands rounded to bf16, perhaps the other way
            p, q = (np.abs(val[i]) for i in by_output[t]["in"])
            assert (np.abs(a - b) <= (4 * U16 + 2 * CHAIN) * (p @ q.T)).all(), what
        else:
            assert np.abs(a - b).max() <= CHAIN * np.abs(b).max(), what


@pytest.mark.parametrize("rows,cols", [(37, 264), (131, 130), (65, 33), (1, 1001)])
@pytest.mark.parametrize("seed", range(12))
def test_random_mixture_of_operators_and_types(seed, rows, cols):
    """bf16 and f32 tensors among each other: up to 14 roundings to bf16 behind one another, each in two evaluations that may
    round differently, bound the relative 2-norm."""
    g, inputs, outputs, eight = random_mixture(1000 + seed, rows, cols, types=("f32", "bf16"))
    feeds = normals(g.desc, inputs, seed)
    got, f = run_gpu(g.desc, inputs, outputs, feeds)
    for t, a, b in zip(outputs, got, interp.run_function(g.desc, inputs, outputs, feeds)):
        assert np.linalg.norm(a - b) <= 14 * 2 * U16 * np.linalg.norm(b) + (2.0 ** -3 * np.linalg.norm(b) if t in eight else 0), "%s of\n%s" % (
            g.desc["tensors"][t]["name"], f.describe())
