"""The graphs of lm_mixed_cases on the GPU against the fp64 oracle."""
import numpy as np
import pytest

from lm_cases import U16, U32, normals, run_gpu
from lm_mixed_cases import SUM_READERS, sum_read_before_its_norm
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
