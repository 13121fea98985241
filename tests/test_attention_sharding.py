"""The attention operators on shards of the leading axis: norm and rotation work row by row, attention and its cache are refused."""
import numpy as np
import pytest

from oracle import interp
from paper_1707_08265_b200 import sharding
from paper_1707_08265_b200 import workloads as wl

ROWS = 37


def graph(rows):
    g = wl.GraphDesc()
    x, gain, pos, dy = g.tensor("x", [rows, 48]), g.tensor("gain", [16]), g.tensor("pos", [rows], "i32"), g.tensor("dy", [rows, 48])
    u = g.op("HeadNorm", [x, gain], "u", [rows, 48])
    y = g.op("Rotate", [u, pos], "y", [rows, 48], attrs=[3])
    along = g.op("Mul", [y, dy], "along")
    return g, [x, gain, pos, dy], [u, y] + g.grad([along], [x, gain])


def test_norm_and_rotation_row_by_row():
    rng = np.random.default_rng(3)
    feeds = [rng.standard_normal((ROWS, 48)), rng.standard_normal(16), rng.integers(0, 900, ROWS).astype(np.int32), rng.standard_normal((ROWS, 48))]
    g, inputs, outputs = graph(ROWS)
    kinds = sharding.classify_outputs(g.desc, outputs, ROWS)
    assert kinds == [sharding.LOCAL] * 3 + [sharding.SUM]
    want, parts = interp.run_function(g.desc, inputs, outputs, feeds), []
    for rank in range(3):
        lo, hi = sharding.shard_range(ROWS, rank, 3)
        parts.append(interp.run_function(sharding.shard_desc(g.desc, ROWS, hi - lo), inputs, outputs, sharding.cut_feeds(g.desc, inputs, feeds, ROWS, lo, hi)))
    for j, (k, w) in enumerate(zip(kinds, want)):
        got = np.concatenate([p[j] for p in parts]) if k == sharding.LOCAL else sum(p[j] for p in parts)
        assert np.allclose(got, w, rtol=1e-12, atol=1e-12), j


H, I = "bf16", "i32"


@pytest.mark.parametrize("op,ins,out,attrs", [
    ("HeadNorm", [([64, 256], "f32"), ([64], "f32")], [64, 256], ()),                       # the gain has the extent by chance
    ("Rotate", [([9, 64], "f32"), ([9], I)], [9, 64], (4,)),
    ("Attention", [([64, 32], H)] * 3, [64, 32], (2, 2)),
    ("Attention", [([64, 32], H)] * 3, [64, 32], (2, 2, 1, 0, 0.0, 4)),
    ("Attention", [([9, 32], H)] * 3 + [([64], I)], [9, 32], (2, 2)),
    ("CacheWrite", [([64, 32], H), ([3, 32], H), ([3, 2], I), ([3], I)], [64, 32], (16,)),
    ("CacheWrite", [([48, 32], H), ([64, 32], H), ([64, 2], I), ([64], I)], [48, 32], (16,)),
    ("PagedAttention", [([64, 32], H), ([48, 32], H), ([48, 32], H), ([64, 2], I), ([64], I)], [64, 32], (2, 2, 16)),
])
def test_what_mixes_rows_is_refused(op, ins, out, attrs):
    g = wl.GraphDesc()
    o = g.op(op, [g.tensor("i%d" % k, shape, dtype) for k, (shape, dtype) in enumerate(ins)], "o", out, H, attrs=attrs)
    if op == "Rotate":
        g.desc["tensors"][1]["shape"] = [64]          # positions of other rows
    for f in (lambda: sharding.classify_outputs(g.desc, [o], 64), lambda: sharding.shard_desc(g.desc, 64, 32)):
        with pytest.raises(ValueError, match=op):
            f()
    sharding.classify_outputs(g.desc, [o], 7777)


def test_a_layer_with_attention_is_refused():
    g, ids = wl.attention_layer(64, 32, 2, 1, 16, 40, sequences=2)
    with pytest.raises(ValueError, match="Attention"):
        sharding.classify_outputs(g.desc, [ids["loss"]], 64)
