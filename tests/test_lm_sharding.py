"""The language-model operators on shards of the leading axis: those that work row by row reproduce the whole result on two
gloo ranks, those that mix rows are refused."""
import os

import numpy as np
import pytest
import torch
import torch.distributed as dist
import torch.multiprocessing as mp

from paper_1707_08265_b200 import sharding
from paper_1707_08265_b200 import workloads as wl

ROWS, COLS = 37, 160


def layer(rows):
    """A norm, its 8-bit form, a product with 8-bit weights, a loss with the norm's gradients, a tensor clipped by a fed norm.
    (The norm's rows are the logits: an InnerProduct rounds their gradient to bf16, which does not commute with a rank's share.)"""
    g = wl.GraphDesc()
    h, w, labels = g.tensor("h", [rows, COLS]), g.tensor("w", [COLS]), g.tensor("labels", [rows], "i32")
    wq, sw, norm = g.tensor("wq", [48, COLS], "f8e4m3"), g.tensor("sw", [1, 2]), g.tensor("norm", [])
    y = g.op("RMSNorm", [h, w], "y", [rows, COLS])
    s = g.op("BlockScale", [y], "s", [rows, 2], attrs=[1])
    q = g.op("Quantize", [y, s], "q", [rows, COLS], "f8e4m3")
    p = g.op("ScaledInnerProduct", [q, s, wq, sw], "p", [rows, 48])
    c = g.op("ClipByNorm", [h, norm], "c", [rows, COLS], attrs=[0.5])
    loss = g.op("SoftmaxCrossEntropy", [y, labels], "loss", [])
    grads = g.grad([loss], [h, w])
    return g, [h, w, labels, wq, sw, norm], [y, s, q, p, c, loss] + grads


def layer_feeds():
    from oracle import interp
    rng = np.random.default_rng(5)
    return [rng.standard_normal((ROWS, COLS)), rng.standard_normal(COLS),
            rng.integers(0, COLS, ROWS).astype(np.int32), interp.round_e4m3(rng.standard_normal((48, COLS)) * 50), rng.uniform(0.1, 1, (1, 2)), np.array(3.0)]


def _rank(rank, world, port, out_dir):
    os.environ["MASTER_ADDR"], os.environ["MASTER_PORT"] = "127.0.0.1", str(port)
    dist.init_process_group("gloo", rank=rank, world_size=world)
    from oracle import interp
    g, inputs, outputs = layer(ROWS)
    lo, hi = sharding.shard_range(ROWS, rank, world)
    kinds = sharding.classify_outputs(g.desc, outputs, ROWS)
    part = sharding.shard_desc(g.desc, ROWS, hi - lo)
    feeds = sharding.cut_feeds(g.desc, inputs, layer_feeds(), ROWS, lo, hi)
    res = sharding.run_classified(lambda: [torch.from_numpy(np.array(a, dtype=np.float64)) for a in interp.run_function(part, inputs, outputs, feeds)],
                                  kinds, dist.all_reduce, (hi - lo) / ROWS)
    np.savez(os.path.join(out_dir, "r%d.npz" % rank), *[a.numpy() for a in res])
    dist.destroy_process_group()


def test_row_by_row_operators_on_two_ranks(tmp_path):
    from oracle import interp
    world = 2
    mp.start_processes(_rank, args=(world, 31500 + os.getpid() % 2000, str(tmp_path)), nprocs=world, join=True, start_method="spawn")
    g, inputs, outputs = layer(ROWS)
    want = interp.run_function(g.desc, inputs, outputs, layer_feeds())
    kinds = sharding.classify_outputs(g.desc, outputs, ROWS)
    assert kinds == [sharding.LOCAL] * 5 + [sharding.MEAN, sharding.LOCAL, sharding.MEAN]
    got = [np.load(tmp_path / ("r%d.npz" % r)) for r in range(world)]
    for j, (k, w) in enumerate(zip(kinds, want)):
        parts = [r["arr_%d" % j] for r in got]
        if j == 6:      # the loss is a mean over a rank's own rows: a row's gradient comes out divided by that number
            parts = [p * (len(p) / ROWS) for p in parts]
        for p in [np.concatenate(parts)] if k == sharding.LOCAL else parts:
            assert np.allclose(p, w, rtol=1e-12, atol=1e-12), j


def one(op, ins, out, attrs=()):
    g = wl.GraphDesc()
    t = [g.tensor("i%d" % k, shape, dtype) for k, (shape, dtype) in enumerate(ins)]
    return g, g.op(op, t, "o", out, attrs=attrs)


@pytest.mark.parametrize("op,ins,out,attrs", [
    ("GlobalNorm", [([256, 64], "f32"), ([64], "f32")], [], ()),
    ("GatedScan", [([256, 64], "f32"), ([256, 64], "f32")], [256, 64], ()),
    ("GatedScan", [([256, 64], "f32"), ([256, 64], "f32")], [256, 64], (4,)),
    ("BlockScale", [([256, 64], "f32")], [2, 1], (128,)),
    ("BlockScale", [([256 * 128, 64], "f32")], [256, 1], (128,)),                # its scales have the extent by chance
    ("Quantize", [([256, 64], "f32"), ([2, 1], "f32")], [256, 64], ()),
    ("RMSNorm", [([256], "f32"), ([256], "f32")], [256], ()),                    # the normalised axis itself
    ("RMSNorm", [([256, 256], "f32"), ([256], "f32")], [256, 256], ()),          # the gain has the extent by chance
    ("ScaledInnerProduct", [([5, 128], "f8e4m3"), ([5, 1], "f32"), ([256, 128], "f8e4m3"), ([2, 1], "f32")], [5, 256], ()),
])
def test_operators_that_mix_rows_are_refused(op, ins, out, attrs):
    g, o = one(op, ins, out, attrs)
    with pytest.raises(ValueError, match=op):
        sharding.classify_outputs(g.desc, [o], 256)
    with pytest.raises(ValueError, match=op):
        sharding.shard_desc(g.desc, 256, 128)
    sharding.classify_outputs(g.desc, [o], 7777)        # an extent that they do not have


def test_a_rank_s_own_mean_does_not_go_into_a_norm():
    g = wl.GraphDesc()
    z, labels, b = g.tensor("z", [256, 10]), g.tensor("labels", [256], "i32"), g.tensor("b", [7])
    loss = g.op("SoftmaxCrossEntropy", [z, labels], "loss", [])
    n = g.op("GlobalNorm", [loss, b], "n", [])
    with pytest.raises(ValueError, match="GlobalNorm"):
        sharding.classify_outputs(g.desc, [n], 256)
    g, ids = wl.recurrent_layer(2, 64, 32, 48, 40)
    with pytest.raises(ValueError, match="GatedScan"):
        sharding.classify_outputs(g.desc, [ids["loss"]], 128)
