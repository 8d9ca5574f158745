"""Samples by speculative rounds over shared pages are those of plain decoding (examples/sampled_rounds.py)."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import sampled_rounds  # noqa: E402

pytestmark = pytest.mark.gpu


def test_rounds_draw_the_samples_of_plain_decoding():
    """fp32: both ways compute the same logits up to their last bits, and draw with the same numbers.  Samples of a prompt differ from
    each other, whole pages of the prompts are shared, and the pages in use are the cache's first ones."""
    (plain, trees), pages = sampled_rounds.run("f32")
    plain = plain.tolist()
    for i, t in enumerate(trees):
        n = min(len(t), len(plain[i]))
        assert len(t) > 8 and t[:n] == plain[i][:n], i
    assert plain[0] != plain[1] and plain[3] != plain[4]
    uses = pages.uses.tolist()
    live = sum(n > 0 for n in uses)
    assert max(uses) == 2 and all(n == 0 for n in uses[live + 6:])     # (at most a page each since they were compacted)
    count = torch.zeros(len(uses), dtype=torch.long)
    for row, held in zip(pages.table.tolist(), pages.held.tolist()):
        for p in row[:held]:
            count[p] += 1
    assert count.tolist() == uses and int(pages.missing) == 0


@pytest.mark.parametrize("cache", ["bf16", "fp8"])
def test_other_caches_run(cache):
    """(Their rounding differs between the two ways, so samples part sooner or later.)"""
    (plain, trees), pages = sampled_rounds.run(cache, samples=2, steps=20, rounds=4)
    assert all(0 <= t < sampled_rounds.VOCAB for row in trees for t in row) and plain.shape == (4, 20)
    assert int(pages.missing) == 0
