"""Sampling at limits of its numbers: rows whose values lie within a hair of one another, or further apart than fp32
reaches; a top-k of the whole vocabulary and beyond; calls of very many rows.  Tokens and log-probabilities against the
definition in 64 bits, with the tolerances of test_gpu_sample.py."""
import ctypes

import pytest
import torch

from paper_2607_08642_amd import binding
from test_gpu_sample import check, rows_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V,ks", [(20, (2, 5, 10, 19)), (2003, (10, 64, 65, 100, 1000, 2002)), (20011, (100, 900, 4000)),
                                  (70001, (100, 1025, 30000))])
def test_values_that_lie_close(dtype, V, ks):
    """Rows of zeros but for a few values of 1e-37 and less: their differences times the bins' number pass fp32's range when
    divided by one another."""
    g = torch.Generator().manual_seed(V)
    x = torch.zeros(7, V)
    at = torch.randperm(V, generator=g)
    x[0, at[0]] = 1e-37
    x[1, at[:3]] = torch.tensor([1e-37, -1e-37, 2e-37])
    x[2, at[:V // 3]] = -1e-37
    x[3, at[:9]] = 1e-37 * torch.arange(-4, 5)
    x[4] = 1e-38 * torch.randint(-9, 10, (V,), generator=g)
    x[5] = 1e-44 * torch.randint(-9, 10, (V,), generator=g)     # (bf16: all zero)
    x[6] = 1e-30 * torch.randn(V, generator=g)
    x, u = x.to({"f32": torch.float32, "bf16": torch.bfloat16}[dtype]), torch.rand(7, generator=g)
    for k in ks:
        check(x, u, k=k)
        check(x, u, k=k, p=0.9, q=0.5)
        check(x, u, k=k, T=1e-37)
    for how in (dict(p=0.9), dict(p=0.3, q=0.9), dict(q=0.5), dict(p=0.9, T=1e-37), dict(q=0.1, T=1e-37)):
        check(x, u, **how)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [300, 20011, 70001])
def test_values_that_lie_far_apart(dtype, V):
    """Differences past fp32's largest number, and temperatures at which they count."""
    g = torch.Generator().manual_seed(V + 1)
    x = 3e38 * (2 * torch.rand(4, V, generator=g) - 1)
    x[1] = 3e38 * torch.randint(-1, 2, (V,), generator=g)
    x[2, V // 2:] = -float("inf")
    x[3] = -3e38
    x[3, V // 3] = 3.2e38
    x, u = x.to({"f32": torch.float32, "bf16": torch.bfloat16}[dtype]), torch.rand(4, generator=g)
    for T in (1.0, 1e37, 2e38, float("inf")):
        for how in (dict(), dict(k=100), dict(k=V // 2, p=0.9), dict(p=0.9), dict(q=0.2), dict(p=0.99, q=0.1)):
            check(x, u, T=T, **how)


def nodes(call):
    """How many nodes a graph of the call has."""
    graph, n = torch.cuda.CUDAGraph(keep_graph=True), ctypes.c_size_t()
    call()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        call()
    assert binding.load().hipGraphGetNodes(ctypes.c_void_p(graph.raw_cuda_graph()), None, ctypes.byref(n)) == 0
    return n.value


def test_top_k_of_the_whole_vocabulary_is_off():
    """As a number, too: the launches and bits of top_k = 0."""
    V = 40011
    x, u = rows_of(3, V, "f32", seed=60, spread=0.7, high=2)
    a, v = x.cuda(), u.cuda()
    for how in (dict(top_p=0.9), dict(min_p=0.05), dict(top_p=0.97, min_p=0.01)):
        want = binding.sample(a, v, logprobs=True, **how)
        for k in (V, V + 1, 2 ** 31 - 1):
            got = binding.sample(a, v, top_k=k, logprobs=True, **how)
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
            assert nodes(lambda: binding.sample(a, v, top_k=k, **how)) == nodes(lambda: binding.sample(a, v, **how))
    check(x, u, k=V, p=0.9)


def test_top_k_beyond_32_bits():
    """Off, as every top_k >= V; a negative one is refused, and one that is no whole number."""
    x, u = rows_of(8, 3001, "f32", seed=61)
    x, u = x.cuda(), u.cuda()
    want = binding.sample(x, u)
    assert not torch.equal(want, binding.sample(x, u, top_k=1))
    for k in (2 ** 31, 2 ** 32, 2 ** 32 + 1, 2 ** 40 + 5, 10 ** 18 + 1, 2 ** 63 - 1, 2 ** 64 + 1):
        assert torch.equal(binding.sample(x, u, top_k=k), want), k
    for k in (-1, -2 ** 31, -2 ** 32 + 1, -2 ** 32, -2 ** 64 + 5):
        with pytest.raises(binding.DTError):
            binding.sample(x, u, top_k=k)
    for k in (5.0, float("inf"), "5"):
        with pytest.raises(TypeError):
            binding.sample(x, u, top_k=k)


def test_large_workspaces_are_not_kept():
    """A call of many rows leaves no memory behind but its results; calls on many streams leave a bounded number."""
    x, u = rows_of(1, 40000, "bf16", seed=62)
    x, u = x.cuda().expand(1 << 14, -1), torch.rand(1 << 14, device="cuda")
    binding.sample(x[:2], u[:2], top_k=20)
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    tokens = binding.sample(x, u, top_k=20)
    torch.cuda.synchronize()
    assert torch.cuda.memory_allocated() - before <= 64 << 20
    want = binding.sample(x[:640], u[:640], top_k=20)
    assert torch.equal(tokens[:640], want)
    before = torch.cuda.memory_allocated()
    for s in [torch.cuda.Stream() for _ in range(32)]:
        s.wait_stream(torch.cuda.current_stream())
        got = binding.sample(x[:640], u[:640], top_k=20, stream=s)
        s.synchronize()
        assert torch.equal(got, want)
    torch.cuda.synchronize()
    del got
    assert torch.cuda.memory_allocated() - before <= 256 << 20
