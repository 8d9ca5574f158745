"""Sampling where rows take several launches (vocabularies of more than 32,753), and some of a call's rows are large ones
(thousands of tokens kept by top-p or min-p): graphs, settings of each row, strides, values that are not finite.  Tokens
and log-probabilities against the definition in 64 bits, with the tolerances of test_gpu_sample.py; the same sums at
another alignment may differ in their last bits, so two log-probabilities by 2^-24 of each and 1e-10 for each."""
import itertools

import pytest
import torch

from paper_2607_08642_amd import binding
from test_gpu_sample import DTYPES, INF, NAN, SETTINGS, check, rows_of

pytestmark = pytest.mark.gpu


def mixed_rows(R, V, dtype, seed):
    """Peaked rows and flat ones in turn."""
    x, u = rows_of(R, V, dtype, seed=seed)
    flat, _ = rows_of(R, V, dtype, seed=seed + 1, spread=0.7, high=1)
    x[1::2] = flat[1::2]
    return x, u


def near(a, b):
    return torch.allclose(a, b, rtol=2.0 ** -23, atol=2e-10)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [40008, 40011, 151936])
def test_rows_of_their_own_settings(dtype, V):
    """Every combination of settings in one call, of which some make their row a large one; the rows in another order
    and at other strides: the same tokens, and the same bits where a row begins at the same place of 16 bytes."""
    grid = list(itertools.product([0.0, 0.7, 1.5], [0, 40], [1.0, 0.9], [0.0, 0.05]))
    grid = grid + grid[::-1]                     # (each on a peaked row and a flat one)
    R = len(grid)
    x, u = mixed_rows(R, V, dtype, 21)
    settings = [torch.tensor([s[i] for s in grid], dtype=torch.int32 if i == 1 else torch.float32) for i in range(4)]
    tokens, logprobs = check(x, u, *settings)
    put = [s.cuda() for s in settings]
    for pad in (1, 8, 64):
        wide = torch.full((R, V + pad), 50.0, dtype=x.dtype, device="cuda")
        wide[:, :V] = x.cuda()
        a, b = binding.sample(wide[:, :V], u.cuda(), *put, logprobs=True)
        assert torch.equal(a.cpu(), tokens) and near(b.cpu(), logprobs)
        if V % 8 == 0 and pad % 8 == 0:
            assert torch.equal(b.cpu(), logprobs)
    back = torch.arange(R - 1, -1, -1)
    a, b = binding.sample(x[back].cuda(), u[back].cuda(), *(s[back].cuda() for s in settings), logprobs=True)
    assert torch.equal(a.cpu()[back], tokens) and near(b.cpu()[back], logprobs)
    if V % 8 == 0:
        assert torch.equal(b.cpu()[back], logprobs)
    for i in range(0, R, 5):                     # (alone)
        a, b = binding.sample(x[i].cuda(), u[i].cuda(), *(s[i].cuda() for s in settings), logprobs=True)
        assert int(a) == int(tokens[i]) and near(b.cpu(), logprobs[i])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_the_order_of_rows_in_one_launch(dtype):
    """The same of rows that one launch reads."""
    for V in (20008, 20011):
        x, u = mixed_rows(24, V, dtype, 23)
        T = torch.linspace(0.4, 2.0, 24)
        tokens, logprobs = check(x, u, T, p=0.95)
        back = torch.arange(23, -1, -1)
        a, b = binding.sample(x[back].cuda(), u[back].cuda(), T[back].cuda(), 0, 0.95, logprobs=True)
        assert torch.equal(a.cpu()[back], tokens) and near(b.cpu()[back], logprobs)
        if V % 8 == 0:
            assert torch.equal(b.cpu()[back], logprobs)


@pytest.mark.parametrize("how", SETTINGS, ids=str)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [40011, 151936])
def test_values_that_are_not_finite(how, dtype, V):
    x, u = rows_of(14, V, dtype, seed=9)
    x[0] = -INF
    x[1] = NAN
    x[2] = -INF
    x[2, V - 3] = -3.0                           # one token is left
    x[3, ::2] = -INF
    x[4, 1::2] = NAN
    x[5, 77] = INF
    x[6, [5, 30000, V - 1]] = INF
    x[7] = INF
    x[8] = torch.finfo(x.dtype).min
    x[9] = torch.finfo(x.dtype).min
    x[9, 10] = torch.finfo(x.dtype).max
    x[10, :2048] = -INF
    x[11, 3:] = -INF
    x[12] = (0.7 * torch.randn(V, generator=torch.Generator().manual_seed(10))).to(DTYPES[dtype])   # (flat)
    x[12, ::3] = -INF
    x[12, 1::5] = NAN
    x[13] = x[12]
    x[13, 4096:20480] = NAN                      # segments of nothing
    tokens, logprobs = check(x, u, **how)
    assert tokens[0] == tokens[1] == -1 and logprobs[0] == logprobs[1] == -INF
    assert tokens[2] == V - 3 and logprobs[2] == 0


@pytest.mark.parametrize("V", [40011, 151936])
def test_streams_and_graphs(V):
    """Captured calls replayed on rows that change from peaked to flat and back (so that the number of large rows does), between
    eager calls on two streams."""
    R = 12
    x, u = mixed_rows(R, V, "bf16", 30)
    x, u = x.cuda(), u.cuda()
    T, P = torch.full((R,), 0.8, device="cuda"), torch.full((R,), 0.9, device="cuda")
    K = torch.zeros(R, dtype=torch.int32, device="cuda")
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()

    def calls(**on):
        return [binding.sample(x, u, T, 20, 0.95, **on), *binding.sample(x, u, T, K, P, 0.001, logprobs=True, **on),
                *binding.sample(x, u, 1.0, 0, 0.97, logprobs=True, **on), binding.sample(x, u, **on)]

    torch.cuda.synchronize()
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        results = calls()
    for n in range(5):
        y, v = mixed_rows(R, V, "bf16", 31 + n)
        x.copy_(y if n != 2 else rows_of(R, V, "bf16", seed=99)[0])     # (once no row is flat)
        if n == 3:
            x.copy_(rows_of(R, V, "bf16", seed=98, spread=0.7, high=1)[0])  # (and once all are)
        u.copy_(v)
        T.fill_(0.5 + n / 4)
        P.copy_(torch.where(torch.arange(R, device="cuda") % 3 == n % 3, 1.0, 0.9))
        K.copy_(torch.where(torch.arange(R, device="cuda") % 4 == n % 4, 40, 0))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in results]
        with torch.cuda.stream(side):
            fill = [torch.full((1 << 20,), 7, device="cuda") for _ in range(3)]
        for want in (calls(), calls(stream=side)):
            torch.cuda.synchronize()
            assert all(torch.equal(g, w) for g, w in zip(got, want))
        assert all(bool((f == 7).all()) for f in fill)
        graph.replay()                           # (the same inputs once more)
        torch.cuda.synchronize()
        assert all(torch.equal(g, w) for g, w in zip(got, results))
    check(x.cpu(), u.cpu(), T.cpu(), K.cpu(), P.cpu(), 0.001)
