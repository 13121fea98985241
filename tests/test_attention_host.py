"""The attention operators through the C ABI without a GPU: shapes and refusals, gradients' types, plans, caches in place."""
import pytest

from attention_cases import attention_graph, head_graph, paged_graph
from paper_1707_08265_b200 import binding as B
from test_lm_host import refused

F, H, I, Q = B.F32, B.BF16, B.I32, B.F8E4M3


@pytest.mark.parametrize("code,ins,out,attrs", [
    (B.ERR_INVALID_ARG, [(F, (4, 64))], (F, (4, 64)), ()),
    (B.ERR_SHAPE, [(F, (4, 64)), (F, (24,))], (F, (4, 64)), ()),
    (B.ERR_SHAPE, [(F, (64,)), (F, (32,))], (F, (64,)), ()),
    (B.ERR_SHAPE, [(F, (4, 64)), (F, (32,))], (F, (4, 32)), ()),
    (B.ERR_DTYPE, [(I, (4, 64)), (F, (32,))], (F, (4, 64)), ()),
    (B.ERR_DTYPE, [(F, (4, 64)), (F, (32,))], (Q, (4, 64)), ()),
    (B.ERR_INVALID_ARG, [(F, (4, 64)), (F, (32,))], (F, (4, 64)), (-1.0,)),
    (B.ERR_INVALID_ARG, [(F, (4, 64)), (F, (32,))], (F, (4, 64)), (float("nan"),)),
    (B.ERR_INVALID_ARG, [(F, (4, 64)), (F, (32,))], (F, (4, 64)), (1e-6, 1.0)),
    (B.ERR_UNSUPPORTED, [(F, (4, 60)), (F, (12,))], (F, (4, 60)), ()),
    (B.ERR_UNSUPPORTED, [(F, (4, 528)), (F, (264,))], (F, (4, 528)), ()),
])
def test_head_norm_refusals(code, ins, out, attrs):
    refused(code, "HeadNorm", ins, out, attrs)


@pytest.mark.parametrize("code,ins,attrs", [
    (B.ERR_INVALID_ARG, [(F, (4, 64)), (I, (4,))], ()),
    (B.ERR_INVALID_ARG, [(F, (4, 64)), (I, (4,))], (0,)),
    (B.ERR_INVALID_ARG, [(F, (4, 64)), (I, (4,))], (1.5,)),
    (B.ERR_INVALID_ARG, [(F, (4, 64))], (2,)),
    (B.ERR_SHAPE, [(F, (4, 64)), (I, (4,))], (3,)),
    (B.ERR_SHAPE, [(F, (4, 64)), (I, (5,))], (2,)),
    (B.ERR_SHAPE, [(F, (4, 64)), (I, (4, 1))], (2,)),
    (B.ERR_DTYPE, [(F, (4, 64)), (F, (4,))], (2,)),
    (B.ERR_DTYPE, [(Q, (4, 64)), (I, (4,))], (2,)),
    (B.ERR_INVALID_ARG, [(F, (4, 64)), (I, (4,))], (2, 34)),
    (B.ERR_INVALID_ARG, [(F, (4, 64)), (I, (4,))], (2, 31)),
    (B.ERR_INVALID_ARG, [(F, (4, 64)), (I, (4,))], (2, -2)),
    (B.ERR_INVALID_ARG, [(F, (4, 64)), (I, (4,))], (2, 32, 2)),
    (B.ERR_INVALID_ARG, [(F, (4, 64)), (I, (4,))], (2, 32, 0, 0.5)),
    (B.ERR_INVALID_ARG, [(F, (4, 64)), (I, (4,))], (2, 32, 0, 1e4, 0.0)),
    (B.ERR_INVALID_ARG, [(F, (4, 64)), (I, (4,))], (2, 32, 0, 1e4, 2.0, 4.0, 1.0)),
    (B.ERR_INVALID_ARG, [(F, (4, 64)), (I, (4,))], (2, 32, 0, 1e4, 2.0, 1.0, 4.0, -1.0)),
    (B.ERR_INVALID_ARG, [(F, (4, 64)), (I, (4,))], (2, 32, 0, 1e4, 2.0, 1.0, 4.0, 100.0, float("inf"))),
    (B.ERR_INVALID_ARG, [(F, (4, 64)), (I, (4,))], (2, 32, 0, 1e4, 2.0, 1.0, 4.0, 100.0, 1.0, 1.0)),
    (B.ERR_UNSUPPORTED, [(F, (4, 60)), (I, (4,))], (5,)),
    (B.ERR_UNSUPPORTED, [(F, (4, 528)), (I, (4,))], (2,)),
])
def test_rotate_refusals(code, ins, attrs):
    refused(code, "Rotate", ins, (F, ins[0][1]), attrs)


def qkv(rows=6, q=64, k=32, v=32, dt=H):
    return [(dt, (rows, q)), (dt, (rows, k)), (dt, (rows, v))]


@pytest.mark.parametrize("code,ins,attrs", [
    (B.ERR_INVALID_ARG, qkv(), ()),
    (B.ERR_INVALID_ARG, qkv()[:2], (4, 2)),
    (B.ERR_INVALID_ARG, qkv(), (4, 3)),
    (B.ERR_INVALID_ARG, qkv(), (2, 4)),
    (B.ERR_INVALID_ARG, qkv(), (4, 2, 2)),
    (B.ERR_INVALID_ARG, qkv(), (4, 2, 0, 5)),
    (B.ERR_INVALID_ARG, qkv(), (4, 2, 1, -1)),
    (B.ERR_INVALID_ARG, qkv(), (4, 2, 1, 1.5)),
    (B.ERR_INVALID_ARG, qkv(), (4, 2, 1, 0, -0.5)),
    (B.ERR_INVALID_ARG, qkv(), (4, 2, 1, 0, 1e300)),
    (B.ERR_INVALID_ARG, qkv(), (4, 2, 1, 0, 0.0, 0)),
    (B.ERR_INVALID_ARG, qkv() + [(I, (3,))], (4, 2, 1, 0, 0.0, 2)),
    (B.ERR_SHAPE, qkv(), (4, 2, 1, 0, 0.0, 4)),
    (B.ERR_SHAPE, qkv(k=48, v=48), (4, 2)),
    (B.ERR_SHAPE, qkv(v=64), (4, 2)),
    (B.ERR_SHAPE, [(H, (6, 64)), (H, (5, 32)), (H, (5, 32))], (4, 2)),
    (B.ERR_SHAPE, qkv() + [(I, (1,))], (4, 2)),
    (B.ERR_SHAPE, qkv() + [(I, (2, 2))], (4, 2)),
    (B.ERR_DTYPE, qkv() + [(F, (3,))], (4, 2)),
    (B.ERR_DTYPE, [(Q, (6, 64))] + qkv()[1:], (4, 2)),
    (B.ERR_UNSUPPORTED, qkv(q=48, k=24, v=24), (4, 2)),
    (B.ERR_UNSUPPORTED, qkv(q=272, k=136, v=136), (2, 1)),
])
def test_attention_refusals(code, ins, attrs):
    refused(code, "Attention", ins, (H, ins[0][1]), attrs)


CACHE = [(H, (64, 32)), (H, (6, 32)), (I, (3, 2)), (I, (3,))]


def but(ins, **changed):
    return [changed.get("i%d" % k, x) for k, x in enumerate(ins)]


@pytest.mark.parametrize("code,ins,out,attrs", [
    (B.ERR_INVALID_ARG, CACHE, (H, (64, 32)), ()),
    (B.ERR_INVALID_ARG, CACHE, (H, (64, 32)), (8,)),
    (B.ERR_INVALID_ARG, CACHE, (H, (64, 32)), (24,)),
    (B.ERR_INVALID_ARG, CACHE[:3], (H, (64, 32)), (16,)),
    (B.ERR_INVALID_ARG, CACHE + [(I, (4,)), (I, (4,))], (H, (64, 32)), (16,)),
    (B.ERR_SHAPE, but(CACHE, i0=(H, (72, 32))), (H, (72, 32)), (16,)),
    (B.ERR_SHAPE, but(CACHE, i1=(H, (6, 40))), (H, (64, 32)), (16,)),
    (B.ERR_SHAPE, but(CACHE, i1=(H, (7, 32))), (H, (64, 32)), (16,)),
    (B.ERR_SHAPE, but(CACHE, i2=(I, (2, 2))), (H, (64, 32)), (16,)),
    (B.ERR_SHAPE, CACHE + [(I, (3,))], (H, (64, 32)), (16,)),
    (B.ERR_DTYPE, but(CACHE, i1=(F, (6, 32))), (H, (64, 32)), (16,)),
    (B.ERR_DTYPE, but(CACHE, i0=(Q, (64, 32)), i1=(Q, (6, 32))), (H, (64, 32)), (16,)),
    (B.ERR_DTYPE, but(CACHE, i3=(F, (3,))), (H, (64, 32)), (16,)),
    (B.ERR_DTYPE, CACHE, (F, (64, 32)), (16,)),
    (B.ERR_UNSUPPORTED, [(H, (64, 12)), (H, (6, 12))] + CACHE[2:], (H, (64, 12)), (16,)),
])
def test_cache_write_refusals(code, ins, out, attrs):
    refused(code, "CacheWrite", ins, out, attrs)


PAGED = [(H, (6, 64)), (H, (64, 32)), (H, (64, 32)), (I, (3, 2)), (I, (3,))]


@pytest.mark.parametrize("code,ins,attrs", [
    (B.ERR_INVALID_ARG, PAGED, (4, 2)),
    (B.ERR_INVALID_ARG, PAGED, (4, 3, 16)),
    (B.ERR_INVALID_ARG, PAGED, (4, 2, 12)),
    (B.ERR_INVALID_ARG, PAGED, (4, 2, 16, -1)),
    (B.ERR_INVALID_ARG, PAGED, (4, 2, 16, 0, -1.0)),
    (B.ERR_INVALID_ARG, PAGED[:4], (4, 2, 16)),
    (B.ERR_SHAPE, but(PAGED, i1=(H, (64, 48)), i2=(H, (64, 48))), (4, 2, 16)),
    (B.ERR_SHAPE, but(PAGED, i2=(H, (80, 32))), (4, 2, 16)),
    (B.ERR_SHAPE, but(PAGED, i1=(H, (72, 32)), i2=(H, (72, 32))), (4, 2, 16)),
    (B.ERR_SHAPE, but(PAGED, i0=(H, (7, 64))), (4, 2, 16)),
    (B.ERR_SHAPE, PAGED + [(I, (5,))], (4, 2, 16)),
    (B.ERR_DTYPE, but(PAGED, i1=(F, (64, 32)), i2=(F, (64, 32))), (4, 2, 16)),
    (B.ERR_DTYPE, but(PAGED, i4=(F, (3,))), (4, 2, 16)),
    (B.ERR_UNSUPPORTED, but(PAGED, i0=(H, (6, 272)), i1=(H, (64, 136)), i2=(H, (64, 136))), (2, 1, 16)),
])
def test_paged_attention_refusals(code, ins, attrs):
    refused(code, "PagedAttention", ins, (H, ins[0][1]), attrs)


def compiled(built, outputs=None):
    g, ids, inputs, outs = built
    return B.Graph.from_desc(g.desc).function(inputs, outputs or outs)


def test_norm_and_rotation_are_one_pass_in_both_directions():
    f = compiled(head_graph(5, 4, 64, grad=True))
    assert [line.split("[")[0] for line in f.describe().splitlines()] == ["head_norm+rotate", "head_norm+rotate_bwd"]
    f = compiled(head_graph(5, 4, 64, norm=False, grad=True))
    assert [line.split("[")[0] for line in f.describe().splitlines()] == ["rotate", "rotate_bwd"]
    f = compiled(head_graph(5, 4, 64, rotate=False, grad=True))
    assert [line.split("[")[0] for line in f.describe().splitlines()] == ["head_norm", "head_norm_bwd"]


def test_a_normed_head_that_is_fetched_is_written_by_the_same_pass():
    f = compiled(head_graph(5, 4, 64, fetch_u=True))
    assert f.describe().count("\n") == 1 and "->normed" in f.describe()


def test_gradients_have_the_types_that_were_asked_for():
    g = B.Graph()
    x, y, a = g.add_tensor("x", H, [4, 8]), g.add_tensor("y", F, [4, 8]), g.add_tensor("a", F, [8])
    g.add_op(B.OPS["Mul"], [x, a], [y])
    dx, da = g.add_grad([y], [x, a], [H, F])
    f = g.function([x, a], [dx, da])
    assert f.num_launches() >= 1
    for bad in ([I, F], [Q, F], [9, F]):
        with pytest.raises(B.DragonError) as e:
            g.add_grad([y], [x, a], bad)
        assert e.value.code == B.ERR_DTYPE
    with pytest.raises(ValueError):
        g.add_grad([y], [x, a], [H])


def test_no_gradient_passes_a_cache():
    g, ids, inputs, outputs = paged_graph(3, 3, 4, 2, 16, 16, 2, 6)
    b = B.Graph.from_desc(g.desc)
    grads = b.add_grad([ids["y"]], [ids["q"]])
    with pytest.raises(B.DragonError):
        b.function(inputs, grads)
    assert "has none" in str(B.lib().dragon_last_error())


def test_keys_and_values_are_written_by_one_launch_and_in_place():
    built = paged_graph(3, 3, 4, 2, 16, 16, 2, 6)
    g, ids, inputs, outputs = built
    f = compiled(built)
    lines = f.describe().splitlines()
    assert lines[0].startswith("cache_write[2 caches") and lines[1].startswith("paged_attention") and len(lines) == 2
    kc, vc = inputs.index(ids["kc"]), inputs.index(ids["vc"])
    assert f.can_alias(kc, 1) and f.can_alias(vc, 2)
    assert not f.can_alias(kc, 2) and not f.can_alias(vc, 1) and not f.can_alias(inputs.index(ids["q"]), 0)


def test_a_cache_that_is_read_later_is_not_written_in_place():
    g, ids, inputs, outputs = paged_graph(3, 3, 4, 2, 16, 16, 2, 6)
    old = g.op("PagedAttention", [ids["q"], ids["kc"], ids["vc"], ids["pages"], ids["lengths"]], "old", [3, 64], "bf16", attrs=[4, 2, 16])
    f = B.Graph.from_desc(g.desc).function(inputs, outputs + [old])
    assert not f.can_alias(inputs.index(ids["kc"]), 1) and not f.can_alias(inputs.index(ids["vc"]), 2)


def test_attention_plan():
    f = compiled(attention_graph(64, 4, 2, 32, grad=True))
    names = [line.split("[")[0] for line in f.describe().splitlines()]
    assert names == ["attention", "attention_bwd"]
    # only the wanted gradients
    g, ids, inputs, outputs = attention_graph(64, 4, 2, 32, grad=True)
    assert "attention_bwd" in B.Graph.from_desc(g.desc).function(inputs, outputs[1:2]).describe()


def test_work_of_few_ctas_is_split():
    """Forward, row sums and gradient are a launch each; one more where the parts of a forward, or of a gradient, are put together."""
    def launches(*args, **kw):
        g, _, inputs, outputs = attention_graph(*args, grad=True, **kw)
        return B.Graph.from_desc(g.desc).function(inputs, outputs).num_launches()

    assert launches(3001, 1, 1, 32) == 5 and launches(2500, 1, 1, 96, window=700) == 4
    assert launches(16384, 8, 2, 128) == 3 and launches(1, 1, 1, 8) == 3 and launches(8192, 32, 8, 128, sequences=4) == 3
