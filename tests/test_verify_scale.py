"""Scales that the attention call takes and refuses, on the host (no GPU needed)."""
import ctypes

import pytest

from paper_2607_08642_amd import binding as b
from test_verify_abi import SHAPE, cache, chunk, options, ref


@pytest.mark.parametrize("scale,ok", [(0.0, True), (-0.0, True), (1e-45, True), (-2.3e38, True), (2.36e38, False),
                                      (-3.4e38, False)])
def test_scales(scale, ok):
    """Exponents are taken to the base of 2: a scale whose product with log2 e is infinite would give 0 * infinity."""
    n = ctypes.c_size_t()
    L = b.load()
    o = options(scale=scale)
    assert L.dt_attend_workspace_size(ref(cache()), ref(chunk()), 8, ref(o), ref(n)) == (0 if ok else SHAPE)
