"""Plans of the language-model operators among themselves and the older ones, without a GPU: what runs in which order."""
import pytest

from lm_cases import norm_graph
from lm_mixed_cases import BROADCAST_KINDS, SUM_READERS, broadcast_gradient, random_mixture, sum_read_before_its_norm
from paper_1707_08265_b200 import binding as B
from paper_1707_08265_b200 import workloads as wl


def steps(desc, inputs, outputs):
    return [s for s in B.Graph.from_desc(desc).function(inputs, outputs).describe().splitlines() if s[0] != " "]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("reader", SUM_READERS)
def test_sum_that_is_read_before_its_norm_is_written_first(reader, dtype):
    """The norm's kernel may write the sum in front of it only where nobody reads the sum before that kernel runs."""
    g, inputs, outputs = sum_read_before_its_norm(reader, dtype)
    lines = steps(g.desc, inputs, outputs)
    assert lines[0].startswith("vm[") and lines[-1].startswith("rms_norm[") and "->sum" not in lines[-1] and "+residual" not in lines[-1]
    # the same where the sum is not fetched
    lines = steps(g.desc, inputs, outputs[1:])
    assert lines[0].startswith("vm[") and "->sum" not in lines[-1] and "+residual" not in lines[-1]
    # the reader alone is not wanted: the norm adds again
    assert steps(g.desc, inputs, [outputs[0], outputs[-1]]) == [lines[-1].replace(" ->y", " +residual ->sum ->y")]


def test_sum_whose_readers_come_behind_the_norm_stays_in_its_kernel():
    g, ids, inputs, outputs = norm_graph(64, 256)
    s = g.op("BlockScale", [ids["h"]], "s", [64, 2])
    assert steps(g.desc, inputs, outputs + [s]) == ["rms_norm[64x256 +residual ->sum ->y]", "quantize[64x256 blocks 1x128 ->scales]"]


@pytest.mark.parametrize("kind", BROADCAST_KINDS)
def test_gradient_of_a_broadcast_tensor_is_summed_before_a_kernel_reads_it(kind):
    g, inputs, outputs = broadcast_gradient(kind)
    lines = steps(g.desc, inputs, outputs)
    names = [s.split("[")[0] for s in lines]
    summing = [i for i, s in enumerate(lines) if "colacc=1" in s or "scalacc=1" in s]
    assert summing, lines
    for i, n in enumerate(names):
        if n in ("rms_norm_bwd", "gated_scan_bwd", "softmax_ce_bwd") and kind != "gain of two uses":
            assert min(summing) < i
    if kind == "product of one row":          # no contraction over more rows than X has
        assert [s for s in lines if s.startswith("gemm")] == ["gemm[1x264x64 -> f32]", "gemm[1x64x264 B^T -> f32]", "gemm[264x64x1 A^T B^T -> f32]"]
    if kind in ("gain of two uses", "vector of two uses", "objective of two uses"):
        # the two contributions meet behind the sum, over the vector's own elements
        assert "colacc=0" in lines[-1] and "n=264 " in lines[-1] and max(summing) < len(lines) - 1
    if kind == "scalar of two widths":
        assert len(summing) == 2 and "n=1 " in lines[-1]


def test_contributions_of_one_shape_stay_one_program():
    g = wl.GraphDesc()
    x, m = g.tensor("x", [264]), g.tensor("M", [37, 264])
    objs = [g.op("Mul", [m, x], "z"), g.op("Mul", [g.op("Sin", [m], "sm"), x], "u")]
    grads = g.grad(objs, [x])
    lines = steps(g.desc, [x, m], objs + grads)
    assert len(lines) == 1 and "colacc=1" in lines[0]


def test_a_norm_that_is_clipped_itself_is_not_overwritten():
    """Every CTA of the clipping launch reads the norm: a tensor that is the norm as well has to stay while it runs."""
    g = B.Graph()
    n, a = g.add_tensor("n", B.F32, []), g.add_tensor("a", B.F32, [100])
    cn, ca = g.add_tensor("cn", B.F32, []), g.add_tensor("ca", B.F32, [100])
    g.add_op(B.OPS["ClipByNorm"], [n, n], [cn], [1.0])
    g.add_op(B.OPS["ClipByNorm"], [a, n], [ca], [1.0])
    f = g.function([n, a], [cn, ca])
    assert not f.can_alias(0, 0) and not f.can_alias(0, 1) and f.can_alias(1, 1) and not f.can_alias(1, 0)
    assert not g.function([n], [cn]).can_alias(0, 0)


def test_random_mixtures_compile():
    """The library refuses a plan that reads memory before it is written; no mixture of operators makes one."""
    for seed in range(300):
        g, inputs, outputs, _ = random_mixture(seed)
        f = B.Graph.from_desc(g.desc).function(inputs, outputs)
        assert f.num_launches() > 0
