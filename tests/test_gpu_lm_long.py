"""The language-model operators at sizes where a CTA takes its second and third tile or group of scales, against the oracle."""
import numpy as np
import pytest

from lm_cases import U32, as_type, normals, run_gpu, scan_bounds, scan_graph
from oracle import interp
from paper_1707_08265_b200 import workloads as wl
from test_gpu_lm import close

pytestmark = pytest.mark.gpu


# blocks of 128 along K: 34 in the kernel of many rows (scales come 16 at a time: a third set of two), 17 and 34 in one part of
# the kernel of few rows (tiles that leave no room to split; its scales come 16 at a time too), for each of its tile widths
@pytest.mark.parametrize("M,N,K", [(2500, 2100, 4240), (2432, 2048, 2064), (777, 2056, 2064), (900, 2056, 4240), (40, 19000, 4112), (20, 19000, 2064), (7, 19000, 2064)])
@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_scaled_product_over_many_scale_blocks(M, N, K, out):
    g, kb = wl.GraphDesc(), -(-K // 128)
    t = [g.tensor("xq", [M, K], "f8e4m3"), g.tensor("sx", [M, kb]), g.tensor("wq", [N, K], "f8e4m3"), g.tensor("sw", [-(-N // 128), kb])]
    y = g.op("ScaledInnerProduct", t, "y", [M, N], out)
    rng = np.random.default_rng(M + N + K)
    feeds = [interp.round_e4m3(rng.standard_normal((M, K)) * 120), as_type(np.exp(2 * rng.standard_normal((M, kb))) / 100, "f32"),
             interp.round_e4m3(rng.standard_normal((N, K)) * 120), as_type(np.exp(2 * rng.standard_normal((-(-N // 128), kb))) / 100, "f32")]
    (got,), _ = run_gpu(g.desc, t, [y], feeds)
    x, w = feeds[0] * interp._spread(feeds[1], (M, K), 1), feeds[2] * interp._spread(feeds[3], (N, K), 128)
    # exact products; at most 128 additions in a block, one product of scales, one addition a block
    close(got, interp.round_bf16(x @ w.T) if out == "bf16" else x @ w.T, (128 + kb + 2) * U32 * (np.abs(x) @ np.abs(w).T), out, "y")


# tiles of 64 rows times groups of 64 columns (32 of an odd width): 1688 and 2954 with one tile handing on to the next, 2000 and
# 3500 where every tile begins with a sequence; 444 or 592 CTAs run at a time, so each takes three tiles and more
@pytest.mark.parametrize("seqs,length,cols", [(3, 9000, 200), (3, 9000, 201), (500, 64, 200), (1000, 32, 201)])
@pytest.mark.parametrize("types", [("bf16", "bf16", "bf16"), ("f32", "f32", "f32"), ("f32", "bf16", "f32")])
@pytest.mark.parametrize("reset", [False, True])
def test_scan_over_more_tiles_than_ctas(seqs, length, cols, types, reset):
    gate, x, h = types
    g, ids, inputs, outputs = scan_graph(seqs, length, cols, gate, x, h, "f32", reset, True)
    feeds = normals(g.desc, inputs, length + cols, {"gate": 2.0})
    if reset:
        feeds[inputs.index(ids["reset"])] = (np.random.default_rng(cols).random(seqs * length) < 0.004).astype(np.int32)
    names = {g.desc["tensors"][t]["name"]: a for t, a in zip(inputs, feeds)}
    bound = scan_bounds(g.desc, ids, names, seqs)
    want = dict(zip(outputs, interp.run_function(g.desc, inputs, outputs, feeds)))
    first, f = run_gpu(g.desc, inputs, outputs, feeds)
    got = dict(zip(outputs, first))
    for name in ("h", "dgate", "dx", "dh0"):
        close(got[ids[name]], want[ids[name]], bound[name], h if name == "h" else "f32", name)
    (alone,), _ = run_gpu(g.desc, inputs, [ids["h"]], feeds)
    assert np.array_equal(alone, got[ids["h"]])
    again, _ = run_gpu(g.desc, inputs, outputs, feeds, f)
    assert all(np.array_equal(a, b) for a, b in zip(first, again))
