"""The Python side of the verification calls: what it keeps alive, shares and refuses (no GPU needed)."""
import gc
import weakref

import pytest
import torch

from paper_2607_08642_amd import binding


@pytest.fixture
def cache():
    return binding.Cache(4, 32, 1, 64, torch.bfloat16, device="cpu")


def test_a_captured_calls_workspace_is_no_other_calls(cache, monkeypatch):
    """A graph comes back to the workspace it was captured with: no call outside may be given it, nor
    replace it, and it is not the one that eager calls have used and may outgrow."""
    capturing = False
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: capturing)
    first = cache._workspace(1000, None, None)
    assert cache._workspace(900, None, None) is first         # (kept, and enough)
    capturing = True
    graph = [cache._workspace(n, None, None) for n in (800, 2000)]
    capturing = False
    assert len({t.data_ptr() for t in (first, *graph)}) == 3
    dead = weakref.ref(graph[1])
    assert cache._workspace(1000, None, None) is first
    assert cache._workspace(5000, None, None).numel() >= 5000
    assert all(cache._workspace(n, None, None) is not t for n in (700, 4000) for t in graph)
    del graph                        # (the graph's memory is the graph's to keep: nothing here holds on to it)
    gc.collect()
    assert dead() is None
