"""Captured attention and eager calls of the same cache: neither touches the other's workspace."""
import pytest
import torch

from paper_2607_08642_amd import binding
from test_gpu_attend import Attend
from test_gpu_cache import i32, same

pytestmark = pytest.mark.gpu


def capture(a, q, side, first=False):
    """(graph, out) of one captured call on `side`; first: no eager call came before it."""
    out = torch.zeros_like(q)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        if not first:
            a.cache.attend(a.chunk, q, out=out)
            torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=side):
            a.cache.attend(a.chunk, q, out=out)
    torch.cuda.synchronize()
    return graph, out


@pytest.mark.parametrize("first", [False, True])
def test_a_larger_call_between_capture_and_replay(first):
    """An eager call on the captured stream that needs a larger workspace, and tensors that fill what was let go."""
    a = Attend("bf16", [(3000, 1), (1900, 1)], 8, 64, 2, 128, seed=3)
    q = a.q.cuda()
    need = a.cache.workspace_size(a.chunk, 2, 8, binding.dt_attend_options(0.1, 0, 0, 0, None, None))
    assert need > 0                                   # (there are parts to write)
    want = a.run()
    side = torch.cuda.Stream()
    graph, out = capture(a, q, side, first)
    large = binding.Chunk(i32([0, 64, 96]), a.chunk.lens, a.chunk.table, 64, 3000)
    ql = torch.randn(96, 8, 128, device="cuda").bfloat16()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        assert a.cache.workspace_size(large, 96, 8, binding.dt_attend_options(0.1, 0, 0, 0, None, None)) > need
        a.cache.attend(large, ql)
        fill = [torch.full((n,), 7, dtype=torch.uint8, device="cuda") for n in (need,) * 3 + (need // 2,) * 3]
    torch.cuda.synchronize()
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert same(out, want)
        assert all(bool((t == 7).all()) for t in fill)
        assert same(a.cache.attend(a.chunk, q), want)


def test_two_graphs_and_eager_calls_at_once():
    """Graphs of one stream replayed on two others, beside eager calls on the first: the same bits each time."""
    a = Attend("bf16", [(3000, 1), (1900, 1)], 8, 64, 2, 128, seed=4)
    q = a.q.cuda()
    want = a.run()
    streams = [torch.cuda.Stream() for _ in range(3)]
    queries = q, -q
    graphs = [capture(a, x, streams[0]) for x in queries]
    wants = [want, a.cache.attend(a.chunk, queries[1])]
    torch.cuda.synchronize()
    eager = []
    for _ in range(10):
        for (graph, _), s in zip(graphs, streams[1:]):
            with torch.cuda.stream(s):
                graph.replay()
        eager.append(a.cache.attend(a.chunk, q, stream=streams[0]))
    torch.cuda.synchronize()
    for (_, out), w in zip(graphs, wants):
        assert same(out, w)
    for o in eager:
        assert same(o, want)
