"""A serving step captured into a graph: caches written in place, the table changed between replays."""
import numpy as np
import pytest

from attention_cases import paged_feeds, paged_graph
from lm_cases import to_gpu
from paper_1707_08265_b200 import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("new,lengths", [([1, 1, 1], [[300, 17, 5000], [301, 18, 5001], [302, 1, 5002]]),             # few rows, in parts
                                         ([1, 90, 2], [[300, 90, 5000], [301, 180, 5002], [302, 270, 5004]])])       # with a chunk
def test_steps_replayed_with_other_lengths(new, lengths):
    import torch
    page, starts = 16, None if len(set(new)) == 1 else np.concatenate([[0], np.cumsum(new)])
    most = -(-max(map(max, lengths)) // page)
    pool = sum(-(-max(n[s] for n in lengths) // page) for s in range(3)) + 1
    g, ids, inputs, outputs = paged_graph(sum(new), 3, 8, 2, 64, page, most, pool, starts=starts is not None)
    feeds = paged_feeds(g, inputs, 70, [max(n[s] for n in lengths) for s in range(3)], page, pool, starts)
    b, names, dt = B.Graph.from_desc(g.desc), [g.desc["tensors"][t]["name"] for t in inputs], [g.desc["tensors"][t]["dtype"] for t in inputs]
    f, eager = b.function(inputs, outputs), b.function(inputs, outputs)
    one, two = ([to_gpu(a, t) for a, t in zip(feeds, dt)] for _ in range(2))
    kc, vc, at = names.index("kc"), names.index("vc"), names.index("lengths")
    assert f.can_alias(kc, 1) and f.can_alias(vc, 2)
    y, want = (torch.empty(g.shape(outputs[0]), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        f.run_torch(one, [y, one[kc], one[vc]])
    gen = torch.Generator(device="cuda").manual_seed(6)
    for n in lengths:
        for name in ("q", "k", "v"):
            t = torch.randn(one[names.index(name)].shape, generator=gen, device="cuda").to(torch.bfloat16)
            one[names.index(name)].copy_(t)
            two[names.index(name)].copy_(t)
        for dev in (one, two):
            dev[at].copy_(torch.tensor(n, dtype=torch.int32))
        y.fill_(float("nan"))
        graph.replay()
        eager.run_torch(two, [want, two[kc], two[vc]])
        torch.cuda.synchronize()
        assert eager.status() == 0 and f.status() == 0
        for a, c in ((y, want), (one[kc], two[kc]), (one[vc], two[vc])):
            assert torch.equal(a, c)
