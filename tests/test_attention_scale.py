"""Scales of attention that fp32 does not hold, without a GPU."""
import pytest

from paper_1707_08265_b200 import binding as B
from test_attention_host import PAGED, qkv
from test_lm_host import refused


# the kernels work with scale * log2(e) in fp32: 0 times a masked score of -inf, or infinity times a score of 0, is NaN
@pytest.mark.parametrize("scale", [1e-50, 5e-324, 3e38, 2.4e38])
def test_scales_that_fp32_does_not_hold_are_refused(scale):
    refused(B.ERR_INVALID_ARG, "Attention", qkv(), (B.BF16, (6, 64)), (4, 2, 1, 0, scale))
    refused(B.ERR_INVALID_ARG, "PagedAttention", PAGED, (B.BF16, (6, 64)), (4, 2, 16, 0, scale))


@pytest.mark.parametrize("scale", [0.0, 1e-37, 1.0, 2.3e38])
def test_scales_at_the_ends_are_taken(scale):
    for op, ins, attrs in (("Attention", qkv(), (4, 2, 1, 0, scale)), ("PagedAttention", PAGED, (4, 2, 16, 0, scale))):
        g = B.Graph()
        ids = [g.add_tensor("t%d" % i, dt, list(shape)) for i, (dt, shape) in enumerate(ins)]
        g.add_op(B.OPS[op], ids, [g.add_tensor("y", B.BF16, [6, 64])], attrs)
