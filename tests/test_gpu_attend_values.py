"""Attention whose result follows from the values alone, and values and scores at the ends of their range.

Where a tolerance is needed it is the one of the attention tests (test_gpu_attend.allowed)."""
import numpy as np
import pytest
import torch

import verify_ref as ref
from test_gpu_attend import Attend, allowed
from test_gpu_cache import i32

pytestmark = pytest.mark.gpu


def store(a):
    """The whole sequences of a.k and a.v into the cache again."""
    a.cache.append(a.make([(n, n) for n, _ in a.sizes]), a.k.cuda(), a.v.cuda())


# (length, chunk), heads, kv heads: rows of both kernels, splits of a long sequence, blocks that all see and masked ones
CONSTANT = {"tokens": ([(1, 1), (33, 1), (257, 1), (700, 1)], 8, 2), "chunks": ([(300, 37), (129, 129), (513, 64)], 8, 2),
            "long": ([(6001, 2)], 4, 1)}


@pytest.mark.parametrize("D", [64, 96, 128, 256])
@pytest.mark.parametrize("shape", CONSTANT)
def test_equal_values_give_that_value(D, shape):
    """The weights of a row of a bf16 cache sum to one as they are used: with every value 1.875 the result is 1.875, bit
    for bit.  Products, sums and the division err by (n + 16) 2^-23 of it at most in fp32, and the points
    where the rounding to bf16 turns are 2^-8 / 1.875 of it away."""
    sizes, heads, kv = CONSTANT[shape]
    print(f"[values] equal D={D} {shape}", flush=True)
    a = Attend("bf16", sizes, heads, 64, kv, D, seed=D, sharp=4.0)
    a.v.fill_(1.875)
    store(a)
    got = a.run()
    assert bool((got == 1.875).all()), f"{int((got != 1.875).sum())} of {got.numel()} differ"


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f8"])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("chunk", [1, 64])
def test_values_whose_sum_is_just_finite(dtype, D, chunk):
    """256 values of about 1e36, the later half's scores 7.5 (in powers of two) above the first's: no sum passes
    what the values themselves sum to, 2.6e38."""
    print(f"[values] large {dtype} D={D} chunk={chunk}", flush=True)
    a = Attend(dtype, [(256, chunk)], 8, 64, 2, D, seed=D)
    a.q.fill_(1.0)
    a.k.zero_()
    a.k[128:] = 7.5 / 1.4426950408889634 / D ** 0.5
    a.v.copy_((0.75 + 0.25 * a.v.float().abs().clamp(max=1.0)) * 1e36)
    store(a)
    got = a.run()
    assert bool(torch.isfinite(got).all())
    a.check(got)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f8"])
@pytest.mark.parametrize("scale", [0.0, -0.0])
@pytest.mark.parametrize("chunk", [1, 64])
def test_scale_of_zero(dtype, scale, chunk):
    """Every key alike, however large its product with the query is (1.3e38 of either sign here)."""
    print(f"[values] scale {scale} {dtype} chunk={chunk}", flush=True)
    a = Attend(dtype, [(200, chunk)], 8, 64, 2, 64, seed=7)
    a.q.fill_(1e19)
    a.k.copy_(torch.where(a.k[:, :, :1].float() > 0, 2e17, -2e17).expand(a.k.shape))
    store(a)
    a.check(a.run(scale=scale), scale=0.0)
    for x in (float("inf"), float("-inf")):      # (0 times infinity)
        a.k[5, 1, 3] = x
        store(a)
        got = a.run(scale=scale)
        assert bool(torch.isnan(got[:, 4:]).all()) and bool(torch.isfinite(got[:, :4]).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D,chunk", [(64, 1), (64, 64), (128, 64), (256, 1), (256, 64)])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_one_infinite_element_of_a_key(dtype, D, chunk, sign):
    """Scores of -infinity are weights of 0: the row is what it is without that key.  Those of +infinity make NaN."""
    print(f"[values] infinite key {dtype} D={D} chunk={chunk} sign={sign}", flush=True)
    n, at = 200, 90                                  # (a block that every row sees whole)
    a = Attend(dtype, [(n, chunk)], 8, 64, 2, D, seed=D + chunk)
    a.k[at, :, 7] = sign * float("inf")
    store(a)
    got = a.run().double().cpu()
    keep = [j for j in range(n) if j != at]
    ok = ref.visible(chunk, n - chunk, n, 0, 0)[:, keep]
    k, v = a.k[keep], a.v[keep]
    want = ref.attend(a.q, k, v, D ** -0.5, ok)
    tol = allowed(a.q, k, v, D ** -0.5, ok, a.cache.data_dtype)
    zero = a.q[:, :, 7].double() * sign < 0          # (rows whose score there is -infinity)
    assert bool(zero.any()) and not bool(zero.all())
    assert bool(((got - want).abs() <= tol)[zero].all())
    assert bool(torch.isnan(got[~zero]).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_scores_of_minus_infinity_alone(dtype):
    """No key has a weight: zeros, as where nothing is seen."""
    a = Attend(dtype, [(70, 40)], 8, 64, 2, 64, seed=8)
    a.q[:, :, 7] = a.q[:, :, 7].abs().clamp(min=0.1)
    a.k[:, :, 7] = float("-inf")
    store(a)
    assert not a.run().any()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f8"])
@pytest.mark.parametrize("window", [1, 3])
def test_window_shorter_than_the_tree(dtype, window):
    """A chain of nodes deeper than the window: the mask alone says which nodes are seen; with its far bits cleared the
    result is plain decoding's."""
    N = 12
    a = Attend(dtype, [(90, N + 1), (N + 1, N + 1)], 8, 32, 2, 64, seed=window)
    chain = np.tril(np.ones((N, N), np.uint8))
    near = np.triu(chain, 1 - window)
    depths = [list(range(1, N + 1))] * 2
    for mask in (chain, near):
        got = a.run(mask=torch.from_numpy(np.stack([mask] * 2)).cuda(), depth=i32(depths), window=window, sinks=2)
        a.check(got, window=window, sinks=2, masks=[mask] * 2, depths=depths)
    # (sinks among the nodes are the mask's, too; with one, the root of the second sequence, there are none)
    a.check(a.run(mask=torch.from_numpy(np.stack([near] * 2)).cuda(), depth=i32(depths), window=window, sinks=1),
            window=window, sinks=1)
