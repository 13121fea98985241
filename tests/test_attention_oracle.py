"""The oracle's attention operators against differences of themselves and against closed forms."""
import numpy as np
import pytest

from attention_cases import attention_feeds, attention_graph, head_feeds, head_graph, paged_feeds, paged_graph
from oracle import interp


def by_differences(g, inputs, outputs, feeds, wrts, objective, grads):
    want = interp.run_function(g.desc, inputs, grads, feeds, bf16_contraction=False)
    for t, got in zip(wrts, want):
        num = interp.finite_difference(g.desc, inputs, feeds, [objective], t, bf16_contraction=False)
        assert np.max(np.abs(got - num)) <= 1e-6 * (1 + np.max(np.abs(num))), g.desc["tensors"][t]["name"]


@pytest.mark.parametrize("heads,width,dims,interleaved,norm,numbers", [
    (2, 16, 16, 0, True, []), (3, 8, 4, 1, True, [1000.0]), (1, 24, 10, 0, False, [500.0, 4.0, 0.5, 2.0, 60.0, 1.3]), (2, 8, 8, 1, False, [])])
def test_norm_and_rotation_gradients(heads, width, dims, interleaved, norm, numbers):
    g, ids, inputs, outputs = head_graph(3, heads, width, dims, interleaved, norm, numbers, x="f32", y="f32", grad=True)
    feeds = head_feeds(g, inputs, 3)
    along = next(o["out"][0] for o in g.desc["ops"] if o["type"] == "Mul")
    wrts = [ids["x"]] + ([ids["gain"]] if norm else [])
    by_differences(g, inputs, outputs, feeds, wrts, along, outputs[1:])


@pytest.mark.parametrize("heads,kv,causal,window,starts", [(2, 1, 1, 0, None), (2, 2, 0, 0, None), (3, 1, 1, 3, [0, 4, 4, 9]), (1, 1, 0, 0, [1, 6, 8])])
def test_attention_gradients(heads, kv, causal, window, starts):
    g, ids, inputs, outputs = attention_graph(9, heads, kv, 8, causal, window, starts=len(starts) - 1 if starts else 0, q="f32", k="f32", v="f32", y="f32", grad=True,
                                              grad_types=["f32"] * 3)
    feeds = attention_feeds(g, inputs, 4, starts)
    along = next(o["out"][0] for o in g.desc["ops"] if o["type"] == "Mul")
    by_differences(g, inputs, outputs, feeds, [ids[n] for n in "qkv"], along, outputs[1:])


def test_rotation_is_relative():
    """Products of rotated rows depend on the distance of their positions alone, at far positions too."""
    for far in (0, 10 ** 6, 2 ** 31 - 200):
        g, ids, inputs, outputs = head_graph(2, 1, 32, norm=False, x="f32", y="f32")
        feeds = head_feeds(g, inputs, 5)
        dots = []
        for shift in (0, 101):
            feeds[1] = np.array([far + 3, far + 40 + 0], np.int32) + np.int32(shift)
            y, = interp.run_function(g.desc, inputs, outputs, feeds)
            dots.append(y[0] @ y[1])
        assert abs(dots[0] - dots[1]) <= 1e-7


def test_one_row_at_a_time_is_the_whole_attention():
    """Rows written into a paged cache and answered one after another give what Attention gives for all of them."""
    T, heads, kv, width, page = 37, 4, 2, 8, 16
    g, ids, inputs, outputs = attention_graph(T, heads, kv, width, y="f32")
    feeds = attention_feeds(g, inputs, 6)
    want, = interp.run_function(g.desc, inputs, outputs, feeds)
    p, pids, pin, pout = paged_graph(1, 1, heads, kv, width, page, 3, 5, y="f32")
    pf = paged_feeds(p, pin, 7, [T], page, 5)
    names = [p.desc["tensors"][t]["name"] for t in pin]
    for t in range(T):
        for n, a in (("q", feeds[0]), ("k", feeds[1]), ("v", feeds[2])):
            pf[names.index(n)] = a[t:t + 1]
        pf[names.index("lengths")] = np.array([t + 1], np.int32)
        y, kc, vc = interp.run_function(p.desc, pin, pout, pf)
        pf[names.index("kc")], pf[names.index("vc")] = kc, vc
        assert np.max(np.abs(y[0] - want[t])) <= 1e-12
