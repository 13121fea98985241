"""A workspace that serves other purposes between two runs of a function: nothing in it has to be as the last run left it."""
import numpy as np
import pytest

from lm_cases import run_gpu, to_gpu, torch_type
from test_gpu_lm import clip_graph, feeds_of, mixed_functions

pytestmark = pytest.mark.gpu


def functions():
    g, t, n, _ = clip_graph([[4096, 3000], [7], [65, 33]], ["bf16", "f32", "f32"], 0.5)
    g2, t2, n2, c2 = clip_graph([[3]] * 300, ["f32"] * 300, 0.5)
    return mixed_functions() + [(g, {}, t, [n]), (g2, {}, t2, [n2] + c2)]


def buffers(g, outputs):
    import torch
    return [torch.empty(g.shape(t), dtype=torch_type(g.desc["tensors"][t]["dtype"]), device="cuda") for t in outputs]


def check(outs, plain):
    import torch
    torch.cuda.synchronize()
    for o, p in zip(outs, plain):
        assert np.array_equal(o.double().cpu().numpy(), p)
        o.reshape(-1).view(torch.uint8).fill_(0x7F)


@pytest.mark.parametrize("k", range(9))
@pytest.mark.parametrize("fill", [0xA5, 0xFF, 0x01])
def test_workspace_that_was_written_to_between_runs(k, fill):
    import torch
    from paper_1707_08265_b200 import binding as B
    g, _, inputs, outputs = functions()[k]
    feeds = feeds_of(g, inputs, 3)
    plain, _ = run_gpu(g.desc, inputs, outputs, feeds)
    f = B.Graph.from_desc(g.desc).function(inputs, outputs)
    f.ensure_workspace()
    dev = [to_gpu(a, g.desc["tensors"][t]["dtype"]) for a, t in zip(feeds, inputs)]
    outs = buffers(g, outputs)
    graph = None
    for step in range(6):
        f._ws.fill_(fill)
        if step == 3:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                f.run_torch(dev, outs)
        graph.replay() if graph else f.run_torch(dev, outs)
        check(outs, plain)


def test_functions_that_share_one_workspace():
    """All functions in one piece of memory, one after another on one stream, eagerly and from graphs captured before."""
    import torch
    from paper_1707_08265_b200 import binding as B
    jobs = []
    for g, _, inputs, outputs in functions():
        feeds = feeds_of(g, inputs, 5)
        plain, _ = run_gpu(g.desc, inputs, outputs, feeds)
        f = B.Graph.from_desc(g.desc).function(inputs, outputs)
        jobs.append((f, [to_gpu(a, g.desc["tensors"][t]["dtype"]) for a, t in zip(feeds, inputs)], buffers(g, outputs), plain))
    size = max(f.workspace_bytes() for f, _, _, _ in jobs)
    mem = torch.empty(size + 256, dtype=torch.uint8, device="cuda")
    base = (mem.data_ptr() + 255) & ~255
    for f, _, _, _ in jobs:
        f.set_workspace(base, size)
        f._ws = mem
    graphs = []
    for turn in range(3):
        for f, dev, outs, plain in jobs:
            f.run_torch(dev, outs)
            check(outs, plain)
    for f, dev, outs, _ in jobs:
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            f.run_torch(dev, outs)
        graphs.append(gr)
    for order in (range(len(jobs)), reversed(range(len(jobs))), range(len(jobs))):
        for i in order:
            graphs[i].replay()
            check(jobs[i][2], jobs[i][3])
