"""The language-model operators through the C ABI without a GPU: shapes and refusals, prune sets, plans."""
import pytest

from lm_cases import norm_graph, scan_graph
from oracle import prune
from paper_1707_08265_b200 import binding as B
from paper_1707_08265_b200 import workloads as wl


def refused(code, op, ins, out, attrs=()):
    """ins, out: (dtype, shape); the operator is refused with the given code and leaves no trace in the graph."""
    g = B.Graph()
    ids = [g.add_tensor("i%d" % k, d, list(s)) for k, (d, s) in enumerate(ins)]
    o = g.add_tensor("o", out[0], list(out[1]))
    with pytest.raises(B.DragonError) as e:
        g.add_op(B.OPS[op], ids, [o], attrs)
    assert e.value.code == code and g.num_ops() == 0


F, H, I, Q = B.F32, B.BF16, B.I32, B.F8E4M3


@pytest.mark.parametrize("code,ins,out,attrs", [
    (B.ERR_INVALID_ARG, [(F, (4, 8))], (F, (4, 8)), ()),
    (B.ERR_INVALID_ARG, [(F, (4, 8)), (F, (8,)), (F, (8,))], (F, (4, 8)), ()),
    (B.ERR_SHAPE, [(F, (4, 8)), (F, (4,))], (F, (4, 8)), ()),
    (B.ERR_SHAPE, [(F, (4, 8)), (F, (1, 8))], (F, (4, 8)), ()),
    (B.ERR_SHAPE, [(F, ()), (F, (1,))], (F, ()), ()),
    (B.ERR_SHAPE, [(F, (4, 8)), (F, (8,))], (F, (8, 4)), ()),
    (B.ERR_DTYPE, [(I, (4, 8)), (F, (8,))], (F, (4, 8)), ()),
    (B.ERR_DTYPE, [(Q, (4, 8)), (F, (8,))], (F, (4, 8)), ()),
    (B.ERR_DTYPE, [(F, (4, 8)), (F, (8,))], (Q, (4, 8)), ()),
    (B.ERR_INVALID_ARG, [(F, (4, 8)), (F, (8,))], (F, (4, 8)), (-1e-6,)),
    (B.ERR_INVALID_ARG, [(F, (4, 8)), (F, (8,))], (F, (4, 8)), (float("nan"),)),
    (B.ERR_INVALID_ARG, [(F, (4, 8)), (F, (8,))], (F, (4, 8)), (1e300,)),
    (B.ERR_INVALID_ARG, [(F, (4, 8)), (F, (8,))], (F, (4, 8)), (1e-6, 2.0)),
    (B.ERR_UNSUPPORTED, [(F, (2, 1 << 27)), (F, (1 << 27,))], (F, (2, 1 << 27)), ()),
])
def test_rms_norm_refusals(code, ins, out, attrs):
    refused(code, "RMSNorm", ins, out, attrs)


@pytest.mark.parametrize("code,ins,out,attrs", [
    (B.ERR_SHAPE, [(F, (130, 200))], (F, (130, 1)), ()),
    (B.ERR_SHAPE, [(F, (130, 200))], (F, (130, 2)), (128,)),
    (B.ERR_SHAPE, [(F, (200,))], (F, (2,)), ()),
    (B.ERR_DTYPE, [(F, (130, 200))], (H, (130, 2)), ()),
    (B.ERR_DTYPE, [(Q, (130, 200))], (F, (130, 2)), ()),
    (B.ERR_INVALID_ARG, [(F, (130, 200))], (F, (130, 2)), (64,)),
])
def test_block_scale_refusals(code, ins, out, attrs):
    refused(code, "BlockScale", ins, out, attrs)


@pytest.mark.parametrize("code,ins,out", [
    (B.ERR_DTYPE, [(F, (130, 200)), (F, (130, 2))], (H, (130, 200))),
    (B.ERR_DTYPE, [(F, (130, 200)), (H, (130, 2))], (Q, (130, 200))),
    (B.ERR_SHAPE, [(F, (130, 200)), (F, (130, 1))], (Q, (130, 200))),
    (B.ERR_SHAPE, [(F, (130, 200)), (F, (3, 2))], (Q, (130, 200))),
    (B.ERR_INVALID_ARG, [(F, (130, 200))], (Q, (130, 200))),
])
def test_quantize_refusals(code, ins, out):
    refused(code, "Quantize", ins, out)


@pytest.mark.parametrize("code,ins,out", [
    (B.ERR_DTYPE, [(F, (4, 256)), (F, (4, 2)), (Q, (130, 256)), (F, (2, 2))], (F, (4, 130))),
    (B.ERR_DTYPE, [(Q, (4, 256)), (H, (4, 2)), (Q, (130, 256)), (F, (2, 2))], (F, (4, 130))),
    (B.ERR_DTYPE, [(Q, (4, 256)), (F, (4, 2)), (Q, (130, 256)), (F, (2, 2))], (Q, (4, 130))),
    (B.ERR_SHAPE, [(Q, (4, 256)), (F, (4, 2)), (Q, (130, 272)), (F, (2, 3))], (F, (4, 130))),
    (B.ERR_SHAPE, [(Q, (4, 256)), (F, (4, 3)), (Q, (130, 256)), (F, (2, 2))], (F, (4, 130))),
    (B.ERR_SHAPE, [(Q, (4, 256)), (F, (4, 2)), (Q, (130, 256)), (F, (130, 2))], (F, (4, 130))),
    (B.ERR_SHAPE, [(Q, (4, 256)), (F, (4, 2)), (Q, (130, 256)), (F, (2, 2))], (F, (130, 4))),
    (B.ERR_UNSUPPORTED, [(Q, (4, 250)), (F, (4, 2)), (Q, (130, 250)), (F, (2, 2))], (F, (4, 130))),
    (B.ERR_INVALID_ARG, [(Q, (4, 256)), (F, (4, 2)), (Q, (130, 256))], (F, (4, 130))),
])
def test_scaled_product_refusals(code, ins, out):
    refused(code, "ScaledInnerProduct", ins, out)


@pytest.mark.parametrize("code,op,ins,out,attrs", [
    (B.ERR_DTYPE, "GlobalNorm", [(F, (3,)), (I, (3,))], (F, ()), ()),
    (B.ERR_DTYPE, "GlobalNorm", [(F, (3,))], (H, ()), ()),
    (B.ERR_SHAPE, "GlobalNorm", [(F, (3,))], (F, (1,)), ()),
    (B.ERR_INVALID_ARG, "ClipByNorm", [(F, (3,)), (F, ())], (F, (3,)), ()),
    (B.ERR_INVALID_ARG, "ClipByNorm", [(F, (3,)), (F, ())], (F, (3,)), (0.0,)),
    (B.ERR_INVALID_ARG, "ClipByNorm", [(F, (3,)), (F, ())], (F, (3,)), (float("inf"),)),
    (B.ERR_SHAPE, "ClipByNorm", [(F, (3,)), (F, (1,))], (F, (3,)), (1.0,)),
    (B.ERR_DTYPE, "ClipByNorm", [(F, (3,)), (H, ())], (F, (3,)), (1.0,)),
    (B.ERR_SHAPE, "ClipByNorm", [(F, (3,)), (F, ())], (F, (4,)), (1.0,)),
])
def test_clip_refusals(code, op, ins, out, attrs):
    refused(code, op, ins, out, attrs)


@pytest.mark.parametrize("code,ins,attrs", [
    (B.ERR_INVALID_ARG, [(F, (6, 4))], ()),
    (B.ERR_SHAPE, [(F, (6, 4)), (F, (6, 5))], ()),
    (B.ERR_SHAPE, [(F, (6, 4)), (F, (6, 4))], (4,)),
    (B.ERR_INVALID_ARG, [(F, (6, 4)), (F, (6, 4))], (0,)),
    (B.ERR_INVALID_ARG, [(F, (6, 4)), (F, (6, 4))], (1.5,)),
    (B.ERR_DTYPE, [(I, (6, 4)), (F, (6, 4))], ()),
    (B.ERR_SHAPE, [(F, (6, 4)), (F, (6, 4)), (F, (2, 4))], (3,)),
    (B.ERR_SHAPE, [(F, (6, 4)), (F, (6, 4)), (F, (4,))], ()),
    (B.ERR_SHAPE, [(F, (6, 4)), (F, (6, 4)), (I, (7,))], ()),
    (B.ERR_DTYPE, [(F, (6, 4)), (F, (6, 4)), (F, (1, 4)), (F, (6,))], ()),
    (B.ERR_INVALID_ARG, [(F, (6, 4)), (F, (6, 4)), (I, (6,)), (F, (1, 4))], ()),
    (B.ERR_INVALID_ARG, [(F, (6, 4))] * 5, ()),
])
def test_gated_scan_refusals(code, ins, attrs):
    refused(code, "GatedScan", ins, (F, (6, 4)), attrs)


def test_elementwise_operators_refuse_e4m3():
    refused(B.ERR_DTYPE, "Add", [(Q, (4,)), (F, (4,))], (F, (4,)))
    refused(B.ERR_DTYPE, "Mul", [(F, (4,)), (F, (4,))], (Q, (4,)))


def test_no_gradient_passes_an_eight_bit_tensor_or_a_norm():
    g = B.Graph()
    x, w = g.add_tensor("x", F, [4, 128]), g.add_tensor("w", F, [4, 128])
    s, q, y = g.add_tensor("s", F, [4, 1]), g.add_tensor("q", Q, [4, 128]), g.add_tensor("y", F, [4, 4])
    n, c, z = g.add_tensor("n", F, []), g.add_tensor("c", F, [4, 128]), g.add_tensor("z", F, [4, 128])
    sw = g.add_tensor("sw", F, [1, 1])
    g.add_op(B.OPS["BlockScale"], [x], [s])
    g.add_op(B.OPS["Quantize"], [x, s], [q])
    g.add_op(B.OPS["ScaledInnerProduct"], [q, s, q, sw], [y])
    g.add_op(B.OPS["GlobalNorm"], [x, w], [n])
    g.add_op(B.OPS["ClipByNorm"], [w, n], [c], [1.0])
    g.add_op(B.OPS["Mul"], [c, w], [z])
    dx, = g.add_grad([y], [x])
    dw, = g.add_grad([z], [w])
    for inputs, out in (([x, sw], dx), ([x, w], dw)):
        with pytest.raises(B.DragonError, match="would have to pass operator"):
            g.function(inputs, [out])
    g.function([x, w, c], [dw])                # with the clipped tensor fed, the only chain left is through z
    with pytest.raises(B.DragonError):
        g.add_grad([q], [x])                   # an e4m3 tensor is no objective


def plan(desc, inputs, outputs):
    return [line.split("[")[0] for line in B.Graph.from_desc(desc).function(inputs, outputs).describe().splitlines() if not line.startswith("  ")]


def test_residual_norm_and_eight_bit_output_are_one_launch():
    g, ids, inputs, outputs = norm_graph(64, 256, eight_bit=True)
    f = B.Graph.from_desc(g.desc).function(inputs, outputs)
    assert f.describe() == "rms_norm[64x256 +residual ->sum ->y ->scales ->e4m3]\n" and f.num_launches() == 1
    f = B.Graph.from_desc(g.desc).function(inputs, [ids["q"], ids["s"]])
    assert f.describe() == "rms_norm[64x256 +residual ->scales ->e4m3]\n"
    f = B.Graph.from_desc(g.desc).function(inputs, [ids["h"]])
    assert plan(g.desc, inputs, [ids["h"]]) == ["vm"]


def test_norm_gradient_takes_the_residual_branch_with_it():
    g, ids, inputs, outputs = norm_graph(64, 256, grad=True, skip="bf16")
    f = B.Graph.from_desc(g.desc).function(inputs, outputs)
    assert f.describe() == ("rms_norm[64x256 +residual ->sum ->y]\n"
                            "rms_norm_bwd[64x256 +residual gradient ->dh ->dg]\n")
    # only the gain's gradient: no dh is written, and only dh: no partial sums
    assert "->dh" not in B.Graph.from_desc(g.desc).function(inputs, [ids["dg"]]).describe()
    f = B.Graph.from_desc(g.desc).function(inputs, [ids["dx"]])
    assert "->dg" not in f.describe() and "->y" not in f.describe()


def test_sum_behind_a_contraction_stays_in_its_epilogue():
    g = wl.GraphDesc()
    a, w, r, gain = g.tensor("a", [64, 128], "bf16"), g.tensor("w", [256, 128], "bf16"), g.tensor("r", [64, 256], "bf16"), g.tensor("g", [256])
    h = g.op("Add", [g.op("InnerProduct", [a, w], "p", [64, 256]), r], "h", [64, 256], "bf16")
    y = g.op("RMSNorm", [h, gain], "y", [64, 256], "bf16")
    text = B.Graph.from_desc(g.desc).function([a, w, r, gain], [h, y]).describe()
    assert text.splitlines()[0].startswith("gemm[64x256x128 -> bf16 epilogue") and text.splitlines()[1] == "rms_norm[64x256 ->y]"


def test_clipped_tensors_share_a_launch_and_an_updater_takes_the_factor():
    g = wl.GraphDesc()
    t = [g.tensor("g%d" % i, [i + 1, 3]) for i in range(5)]
    w = g.tensor("w", [1, 3])
    n = g.op("GlobalNorm", t, "n", [])
    c = [g.op("ClipByNorm", [a, n], "c%d" % i, attrs=[1.0], out_shape=[i + 1, 3]) for i, a in enumerate(t)]
    w2 = g.op("Sub", [w, c[0]], "w2", [1, 3])
    lines = B.Graph.from_desc(g.desc).function(t, [n] + c).describe().splitlines()
    assert lines == ["global_norm+clip_by_norm[5 tensors]"]              # small: one launch that reads every tensor once
    big = wl.GraphDesc()
    t2 = [big.tensor("a", [4096, 1024]), big.tensor("b", [4096, 1024], "bf16")]
    n2 = big.op("GlobalNorm", t2, "n", [])
    c2 = [big.op("ClipByNorm", [x, n2], "c%d" % i, [4096, 1024], attrs=[1.0]) for i, x in enumerate(t2)]
    f = B.Graph.from_desc(big.desc)
    assert f.function(t2, [n2] + c2).describe().splitlines() == ["global_norm[2 tensors]", "clip_by_norm[2 tensors]"]
    assert f.function(t2, [n2] + c2[:1]).describe().splitlines() == ["global_norm[2 tensors]", "clip_by_norm[1 tensors]"]
    lines = B.Graph.from_desc(g.desc).function(t + [w], [w2]).describe().splitlines()
    assert lines[0] == "global_norm[5 tensors ->factor]" and lines[1].startswith("vm[flat") and len([s for s in lines if s[0] != " "]) == 2


def test_clipping_may_overwrite_its_tensors():
    g = wl.GraphDesc()
    a, b = g.tensor("a", [100]), g.tensor("b", [50], "bf16")
    n = g.op("GlobalNorm", [a, b], "n", [])
    ca = g.op("ClipByNorm", [a, n], "ca", attrs=[1.0], out_shape=[100])
    cb = g.op("ClipByNorm", [b, n], "cb", attrs=[1.0], out_shape=[50], out_dtype="f32")
    f = B.Graph.from_desc(g.desc).function([a, b], [ca, cb, n])
    assert f.can_alias(0, 0) and not f.can_alias(0, 1) and not f.can_alias(1, 1) and not f.can_alias(0, 2)
    ca2 = g.op("ClipByNorm", [a, n], "ca2", attrs=[1.0], out_shape=[100])
    f = B.Graph.from_desc(g.desc).function([a, b], [ca, ca2])
    assert not f.can_alias(0, 0) and not f.can_alias(0, 1)


def test_scan_plan_and_prune_sets():
    g, ids, inputs, outputs = scan_graph(4, 100, 64, reset=True, grad=True)
    f = B.Graph.from_desc(g.desc).function(inputs, outputs)
    assert f.describe() == "gated_scan[400x64, 4 sequences +h0 +reset]\ngated_scan_bwd[400x64, 4 sequences +h0 +reset]\n"
    assert "states only" in B.Graph.from_desc(g.desc).function(inputs, [ids["dx"]]).describe()
    for outs in (outputs, [ids["h"]], [ids["dgate"]], [ids["dh0"]]):
        f = B.Graph.from_desc(g.desc).function(inputs, outs)
        sets = prune.function_sets(g.desc, inputs, outs)
        assert list(f.marked()) == [int(m) for m in sets["marked"]]
        assert f.kept_ops()[0] == sets["fwd_ops"]


def test_workspace_of_a_training_function_counts_its_parts():
    g, ids, inputs, outputs = scan_graph(1, 1000, 64, grad=True)
    small = B.Graph.from_desc(g.desc).function(inputs, [ids["h"]]).workspace_bytes()
    assert B.Graph.from_desc(g.desc).function(inputs, outputs).workspace_bytes() >= small + 8 * 64 * 4
