"""Attention whose result follows from the values alone, and values and scores at the ends of their range.

Where a tolerance is needed it is the one of the attention tests (test_gpu_attend.allowed)."""
import pytest

from test_gpu_attend import Attend

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
