"""All verification calls together, as a decoder runs them: trees must not change what is generated."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("window", [0, 48])
@pytest.mark.parametrize("batch", [1, 5])
def test_trees_generate_what_plain_decoding_does(window, batch):
    """fp32: both ways give the same tokens (their scores differ in the last bits of fp32 sums only)."""
    import decode_rounds
    print(f"[rounds] window={window} batch={batch}", flush=True)
    plain, trees = decode_rounds.run("f32", window, batch=batch, seed=3)
    for i, t in enumerate(trees):
        n = min(len(t), plain.shape[1])
        assert n > 24                          # (more than one token a round: paths are accepted)
        assert t[:n] == plain[i, :n].tolist()


@pytest.mark.parametrize("cache", ["bf16", "fp8"])
def test_rounds_run_in_fewer_bits(cache):
    """The same calls with 16- and 8-bit caches: tokens in range, lengths that follow from the paths."""
    import decode_rounds
    plain, trees = decode_rounds.run(cache, 0, batch=2, steps=40, rounds=5, seed=4)
    assert int(plain.min()) >= 0 and int(plain.max()) < decode_rounds.VOCAB
    for i, t in enumerate(trees):
        assert len(t) >= 6 and all(0 <= x < decode_rounds.VOCAB for x in t)
        assert t[0] == int(plain[i, 0])
