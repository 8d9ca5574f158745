"""Sampled tokens against the definition in 64 bits: the same token for every row, and its log-probability.

Tokens are compared exactly: the weights of both sides agree to 4e-14 and the sums to 1e-11 of the largest weight, so a
random number that falls between both sides' borders has a chance below 1e-5 in all of this file; the seeds are fixed.
A log-probability is rounded to fp32 once: 2^-24 of itself, and 1e-10 for the sums."""
import itertools
import math

import numpy as np
import pytest
import torch

import sample_ref as ref
from paper_2607_08642_amd import binding

pytestmark = pytest.mark.gpu
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
NAN, INF = float("nan"), float("inf")


def rows_of(R, V, dtype, seed=0, spread=2.2, high=8):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(R, V, generator=g) * spread
    n = min(V, 30)
    x.scatter_(1, torch.randint(0, V, (R, n), generator=g), high + 3 * torch.randn(R, n, generator=g))
    return x.to(DTYPES[dtype]), torch.rand(R, generator=g)


def column(v, i):
    return v[i].item() if isinstance(v, torch.Tensor) else float(np.float32(v))


def check(x, u, T=1.0, k=0, p=1.0, q=0.0, dev=None):
    """Rows x (host) through the call; `dev`: the device tensor to use for them."""
    put = lambda v: v.cuda() if isinstance(v, torch.Tensor) else v  # noqa: E731
    tokens, logprobs = binding.sample(x.cuda() if dev is None else dev, u.cuda(), put(T), put(k), put(p), put(q), logprobs=True)
    tokens, logprobs = tokens.cpu(), logprobs.cpu()
    rows = x.double().numpy()
    for i in range(len(rows)):
        how = [column(v, i) for v in (T, k, p, q)]
        want, lp = ref.sample(rows[i], u[i].item(), how[0], int(how[1]), how[2], how[3])
        where = (i, how, u[i].item())
        assert int(tokens[i]) == want, (where, int(tokens[i]), want)
        got = float(logprobs[i])
        assert got == lp or abs(got - lp) <= 2.0 ** -24 * abs(lp) + 1e-10, (where, got, lp)
    return tokens, logprobs


SETTINGS = [dict(), dict(T=0.0), dict(T=0.3), dict(T=2.5), dict(k=1), dict(k=5), dict(k=20, p=0.95, T=0.6), dict(p=0.9), dict(p=0.5),
            dict(q=0.05), dict(q=1.0), dict(p=0.0), dict(k=50, p=0.8, q=0.01), dict(p=0.95, q=0.02, T=1.5), dict(p=0.999999),
            dict(k=300), dict(k=1000, p=0.99, T=2.0), dict(k=7, q=0.3)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [1, 2, 3, 8, 9, 63, 64, 65, 1000, 2003, 2047, 2048, 2049, 4097, 33001])
def test_sizes(dtype, V):
    for n, how in enumerate(SETTINGS):
        x, u = rows_of(3, V, dtype, seed=n)
        check(x, u, **how)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("how", SETTINGS, ids=str)
def test_a_large_vocabulary(dtype, how):
    """Peaked rows, and flat ones of which thousands of tokens are kept."""
    x, u = rows_of(6, 151936, dtype, seed=11, high=13)
    flat, v = rows_of(4, 151936, dtype, seed=12, spread=0.7, high=1)
    check(torch.cat([x, flat]), torch.cat([u, v]), **how)


def test_the_largest_vocabulary():
    x, u = rows_of(2, 1 << 19, "bf16", seed=3, spread=0.5, high=2)
    for how in SETTINGS[:16]:
        check(x, u, **how)


@pytest.mark.parametrize("how", SETTINGS, ids=str)
def test_ties(how):
    """Logits of a few values: borders lie among equals, of which the lowest ids are kept."""
    g = torch.Generator().manual_seed(5)
    for V in (10, 500, 6001):
        x = torch.randint(0, 4, (8, V), generator=g).float()
        x[:2] = 0.0                              # all alike
        x[2] = -0.0
        x[2, ::2] = 0.0
        x[3, :] = torch.arange(V) // 7 % 5
        check(x, torch.rand(8, generator=g), **how)


@pytest.mark.parametrize("how", SETTINGS, ids=str)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_values_that_are_not_finite(how, dtype):
    V = 5000
    x, u = rows_of(12, V, dtype, seed=9)
    x[0] = -INF
    x[1] = NAN
    x[2] = -INF
    x[2, 4321] = -3.0                            # one token is left
    x[3, ::2] = -INF
    x[4, 1::2] = NAN
    x[5, 77] = INF
    x[6, [5, 3000, 4999]] = INF
    x[7] = INF
    x[8] = torch.finfo(x.dtype).min              # the type's lowest value is a logit like others
    x[9] = torch.finfo(x.dtype).min
    x[9, 10] = torch.finfo(x.dtype).max
    x[10, :2048] = -INF                          # a segment of nothing
    x[11, 3:] = -INF
    tokens, logprobs = check(x, u, **how)
    assert tokens[0] == tokens[1] == -1 and logprobs[0] == -INF
    assert tokens[2] == 4321 and logprobs[2] == 0


def test_every_border():
    """Random numbers along [0, 1) hit every kept token of a small row in proportion, in the order of ids."""
    x = torch.tensor([[1.0, 3.0, -2.0, 3.0, 0.5, -INF, 2.0]])
    u = torch.arange(0, 4096) / 4096
    for how in (dict(), dict(k=3), dict(p=0.8), dict(q=0.2), dict(T=0.5, k=5, p=0.9)):
        tokens, _ = check(x.expand(4096, 7).contiguous(), u, **how)
        assert bool((tokens.diff() >= 0).all())
        ids, w = ref.kept(x[0].double().numpy(), how.get("T", 1.0), how.get("k", 0), float(np.float32(how.get("p", 1))),
                          float(np.float32(how.get("q", 0))))
        for i, share in zip(ids, w / w.sum()):
            assert abs(int((tokens == int(i)).sum()) - 4096 * share) <= 1


def test_numbers_outside_their_range():
    """u beyond [0, 1), and settings in tensors that no number may have: the nearest allowed."""
    x, _ = rows_of(8, 3001, "f32", seed=2)
    u = torch.tensor([-1.0, NAN, 0.0, 1.0, 5.0, INF, -INF, 1 - 2.0 ** -24])
    check(x, u)
    check(x, u, k=20)
    v = torch.full((8,), 0.4)
    check(x, v, T=torch.tensor([-1.0, NAN, INF, 1e-30, 1e30, 1e-45, 0.0, 1.0]))
    check(x, v, k=torch.tensor([-3, 0, 1, 3000, 3001, 3002, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32))
    check(x, v, p=torch.tensor([-1.0, 0.0, 1.0, 2.0, INF, 0.3, 1 - 2.0 ** -24, 1e-30]))
    check(x, v, q=torch.tensor([-1.0, 0.0, 1.0, 2.0, INF, 0.3, 1e-30, 0.999]))
    none = dict(p=torch.tensor([NAN]), q=torch.tensor([NAN]))
    assert int(binding.sample(x[:1].cuda(), v[:1].cuda(), 1.0, 0, none["p"].cuda(), none["q"].cuda())) == \
        ref.sample(x[0].double().numpy(), 0.4000000059604645)[0]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_of_their_own_settings(dtype):
    """Every combination of settings in one call; a row alone, in another place and at another stride: the same bits."""
    grid = list(itertools.product([0.0, 0.7, 1.5], [0, 1, 40], [1.0, 0.9], [0.0, 0.05]))
    R, V = len(grid), 20011
    x, u = rows_of(R, V, dtype, seed=21)
    T, k, p, q = (torch.tensor([s[i] for s in grid], dtype=torch.int32 if i == 1 else torch.float32) for i in range(4))
    tokens, logprobs = check(x, u, T, k, p, q)
    for pad in (0, 1, 3, 8, 64):
        wide = torch.full((R, V + pad), 50.0, dtype=x.dtype, device="cuda")
        wide[:, :V] = x.cuda()
        a, b = binding.sample(wide[:, :V], u.cuda(), T.cuda(), k.cuda(), p.cuda(), q.cuda(), logprobs=True)
        assert torch.equal(a.cpu(), tokens) and torch.allclose(b.cpu(), logprobs, rtol=2.0 ** -22, atol=1e-10)
    back = torch.arange(R - 1, -1, -1)
    a, b = binding.sample(x[back].cuda(), u[back].cuda(), T[back].cuda(), k[back].cuda(), p[back].cuda(), q[back].cuda(),
                          logprobs=True)
    assert torch.equal(a.cpu()[back], tokens)


def test_shapes_and_outs():
    x, u = rows_of(34, 999, "bf16", seed=4)
    x, u = x.cuda(), u.cuda()
    want = binding.sample(x, u, 0.9, 10)
    three = binding.sample(x.view(2, 17, 999), u.view(2, 17), 0.9, 10)
    assert three.shape == (2, 17) and torch.equal(three.flatten(), want)
    one = binding.sample(x[3], u[3], 0.9, 10)
    assert one.shape == () and int(one) == int(want[3])
    out = torch.empty(34, dtype=torch.int32, device="cuda"), torch.empty(34, device="cuda")
    got = binding.sample(x, u, 0.9, 10, out=out, logprobs=True)
    assert got[0] is out[0] and torch.equal(out[0], want) and bool((out[1] <= 0).all())
    same_row = binding.sample(x[:1].expand(34, 999), u, 0.9, 10)          # (a stride of 0)
    assert torch.equal(same_row, binding.sample(x[:1].repeat(34, 1), u, 0.9, 10))
    for bad in (dict(u=u[:3]), dict(u=u.double()), dict(logits=x.half()), dict(logits=x.t()), dict(logits=x.cpu()),
                dict(temperature=-1.0), dict(temperature=torch.ones(3, device="cuda")), dict(top_k=torch.ones(34, device="cuda")),
                dict(top_p=-1.0), dict(min_p=2.0), dict(logits=x[:, :0]), dict(logits=x.view(2, 17, 999).transpose(0, 1)),
                dict(out=torch.empty(34, dtype=torch.long, device="cuda")),
                dict(workspace=torch.empty(64, dtype=torch.uint8, device="cuda"))):
        with pytest.raises((ValueError, TypeError, binding.DTError)):
            binding.sample(**dict(dict(logits=x, u=u), **bad))


def test_streams_and_graphs():
    """Captured calls replayed on logits, numbers and settings that change, between eager calls on two streams."""
    R, V = 40, 30011
    x, u = rows_of(R, V, "bf16", seed=30)
    x, u = x.cuda(), u.cuda()
    T = torch.full((R,), 0.8, device="cuda")
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        a = binding.sample(x, u, T, 20, 0.95)
        b, lp = binding.sample(x, u, 1.0, 0, 0.9, 0.01, logprobs=True)
        c = binding.sample(x, u)
    for n in range(4):
        y, v = rows_of(R, V, "bf16", seed=31 + n)
        x.copy_(y)
        u.copy_(v)
        T.fill_(0.5 + n / 4)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (a, b, lp, c)]
        with torch.cuda.stream(side):
            fill = [torch.full((1 << 16,), 7, device="cuda") for _ in range(3)]
        want = [binding.sample(x, u, T, 20, 0.95, stream=side), *binding.sample(x, u, 1.0, 0, 0.9, 0.01, logprobs=True),
                binding.sample(x, u)]
        torch.cuda.synchronize()
        assert all(torch.equal(g, w) for g, w in zip(got, want)) and all(bool((f == 7).all()) for f in fill)
        assert math.isfinite(float(lp.sum()))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [32752, 32753, 32754, 32768, 32769])
def test_where_a_row_takes_another_launch(dtype, V):
    """Sizes about the largest row that one launch reads, also where rows begin inside a 16-byte piece."""
    x, u = rows_of(3, V, dtype, seed=V)
    for how in SETTINGS:
        check(x, u, **how)
    for pad in (1, 7):
        wide = torch.full((3, V + pad), 50.0, dtype=x.dtype, device="cuda")
        wide[:, :V] = x.cuda()
        for how in (dict(), dict(k=20, p=0.95), dict(p=0.9), dict(p=0.999999), dict(T=0.0)):
            check(x, u, dev=wide[:, :V], **how)


@pytest.mark.parametrize("how", [dict(k=1023), dict(k=1024), dict(k=1025), dict(k=2400, p=0.9), dict(k=5000, q=0.01),
                                 dict(k=60000, p=0.99, q=0.001), dict(k=100000)], ids=str)
def test_many_of_a_large_vocabulary(how):
    for spread in (0.7, 2.2):
        x, u = rows_of(3, 100003, "f32", seed=40, spread=spread, high=2)
        check(x, u, **how)


@pytest.mark.parametrize("how", [dict(p=0.9), dict(p=0.3, q=0.5), dict(q=0.9), dict(k=3000), dict(k=3000, p=0.5), dict()], ids=str)
def test_ties_of_a_large_vocabulary(how):
    """Thousands of equal logits at the border, more than a list holds; rows that are and are not so in one call."""
    g = torch.Generator().manual_seed(41)
    x = torch.randn(6, 70001, generator=g)
    x[0] = 1.0
    x[1] = torch.randint(0, 3, (70001,), generator=g).float()
    x[2, 100:60000] = 0.25
    x[3, ::2] = -INF
    x[3, 1::2] = 2.0
    x[4, 5:4000] = INF
    check(x, torch.rand(6, generator=g), **how)


def test_host_threads_on_one_stream():
    """Calls of different sizes by several threads on the same stream: each thread's workspace is its own."""
    import threading
    cases = []
    for n, (R, V, how) in enumerate([(3, 151936, dict(p=0.9)), (40, 2003, dict(k=20)), (1, 60001, dict(k=50, p=0.8)), (17, 40000, dict())]):
        x, u = rows_of(R, V, "bf16", seed=50 + n, spread=0.9, high=3)
        args = x.cuda(), u.cuda(), 1.0, how.get("k", 0), how.get("p", 1.0)
        cases.append((args, binding.sample(*args).cpu()))
    torch.cuda.synchronize()
    wrong = []

    def work(first):
        for n in range(24):
            args, want = cases[(first + n) % 4]
            if not torch.equal(binding.sample(*args).cpu(), want):
                wrong.append((first, n))

    threads = [threading.Thread(target=work, args=(i,)) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong
