"""The Python side of the verification calls: what it keeps alive, shares and refuses (no GPU needed)."""
import gc
import weakref

import pytest
import torch

from paper_2607_08642_amd import binding


class On:
    """As much of a device tensor as the binding looks at."""

    def __init__(self, shape, dtype=torch.int32, device=0):
        self.shape, self.dtype, self.index = torch.Size(shape), dtype, device
        self.device, self.is_cuda = torch.device("cuda", device), True

    def get_device(self):
        return self.index

    def stride(self):
        return tuple(torch.empty(self.shape, device="meta").stride())

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 1 << 20

    def numel(self):
        return self.shape.numel()


class Calls:
    """A library that notes the names of its calls and does nothing."""

    def __init__(self):
        self.made = []

    def __getattr__(self, name):
        return lambda *args: self.made.append(name) or 0


@pytest.fixture
def on_device(cache, monkeypatch):
    """(cache, library): a cache on device 0, the current one, over a library that does nothing."""
    lib = Calls()
    cache._lib, cache._device = lib, 0
    monkeypatch.setattr(binding, "load", lambda: lib)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda d: 0, raising=False)
    return cache, lib


def chunk(device=0):
    return binding.Chunk(On([3], device=device), On([2], device=device), On([2, 4], device=device), 5, 128)


BF16 = torch.bfloat16


def attend(c, k, **kw):
    return c.attend(k, On([8, 2, 64], BF16), out=On([8, 2, 64], BF16), **kw)


def test_calls_on_one_device_are_made(on_device):
    c, lib = on_device
    x = On([8, 1, 64], BF16)
    c.append(chunk(), x, x)
    c.read(chunk(), out=(x, x))
    attend(c, chunk(), mask=On([2, 4, 4], torch.uint8), depth=On([2, 4]), workspace=On([1 << 20], torch.uint8))
    c.commit(chunk(), On([2, 4]), On([2]))
    assert lib.made == ["dt_cache_append", "dt_cache_read", "dt_cache_attend", "dt_cache_commit"]


def test_tensors_of_another_device_are_refused(on_device):
    """Each tensor of each call: an address of another GPU is not to reach a kernel."""
    c, lib = on_device
    x, good, far = On([8, 1, 64], BF16), chunk(), chunk(1)
    calls = [lambda: binding.Chunk(On([3], device=1), On([2]), On([2, 4]), 5, 128),
             lambda: binding.Chunk(On([3]), On([2], device=1), On([2, 4]), 5, 128),
             lambda: binding.Chunk(On([3]), On([2]), On([2, 4], device=1), 5, 128),
             lambda: c.append(far, x, x), lambda: c.read(far, out=(x, x)), lambda: attend(c, far),
             lambda: c.commit(far, On([2, 4]), On([2])),
             lambda: attend(c, good, mask=On([2, 4, 4], torch.uint8, 1)),
             lambda: attend(c, good, mask=On([2, 4, 4], torch.uint8), depth=On([2, 4], device=1)),
             lambda: attend(c, good, workspace=On([1 << 20], torch.uint8, 1)),
             lambda: attend(c, good, workspace=torch.empty(1 << 20, dtype=torch.uint8)),
             lambda: c.commit(good, On([2, 4], device=1), On([2])),
             lambda: c.commit(good, On([2, 4]), On([2], device=1))]
    for n, call in enumerate(calls):
        with pytest.raises(ValueError):
            call()
            pytest.fail(f"call {n} was made")
    assert set(lib.made) <= {"dt_attend_workspace_size"}


def test_calls_of_several_threads_share_a_chunk(on_device):
    """While one call is under way (its library call lets other threads run) another with other rows is made
    from the same Chunk: the first call's structure stays as it was."""
    c, _ = on_device
    k, rows = chunk(), []

    class Busy(Calls):
        def __getattr__(self, name):
            def call(ref, layer, chunk_ref, *rest):
                if not rows:
                    rows.append(None)
                    for n in range(1, 200):      # (also past what a Chunk keeps)
                        k.as_c(n)
                rows.append(chunk_ref._obj.rows)
                return 0
            return call

    c._lib = Busy()
    c.append(k, On([8, 1, 64], BF16), On([8, 1, 64], BF16))
    assert rows == [None, 8]


def test_a_call_on_another_stream_keeps_all_that_it_uses(on_device, monkeypatch):
    """The cache's own memory too: a Cache that goes while a stream still works on it must not be allocated anew."""
    c, _ = on_device
    kept = []
    monkeypatch.setattr(binding, "_keep", lambda stream, *tensors: kept.append(tensors))
    side = type("Stream", (), dict(device_index=0, cuda_stream=5))()
    k, x, q, path, n = chunk(), On([8, 1, 64], BF16), On([8, 2, 64], BF16), On([2, 4]), On([2])
    mask, depth, ws = On([2, 4, 4], torch.uint8), On([2, 4]), On([1 << 20], torch.uint8)
    calls = [(lambda: c.append(k, x, x, stream=side), [x]), (lambda: c.read(k, out=(x, x), stream=side), [x]),
             (lambda: c.attend(k, q, out=q, mask=mask, depth=depth, workspace=ws, stream=side), [q, mask, depth, ws]),
             (lambda: c.commit(k, path, n, stream=side), [path, n])]
    for call, used in calls:
        kept.clear()
        call()
        assert {id(t) for t in (c.storage, k.starts, k.lens, k.table, *used)} <= {id(t) for ts in kept for t in ts}


def tree(b=2, B=4, device=0):
    shapes = dict(tokens=[b, B], parents=[b, B], depth=[b, B], position_ids=[b, B], mask=[b, B, B], scores=[b, B],
                  n_nodes=[b], status=[b])
    return binding.Tree(**{n: On(s, device=device) for n, s in shapes.items()})


def results(**kw):
    return binding.Accepted(**{**dict(path=On([2, 4]), n_accepted=On([2]), next_token=On([2])), **kw})


def test_accept_looks_at_every_tensor(on_device, monkeypatch):
    """Shapes, types and devices of a tree and of given results, and the current device, before anything is launched."""
    _, lib = on_device
    binding.accept_tree(tree(), On([2, 5]), out=results())
    assert lib.made == ["dt_tree_accept"]
    bad = [(tree(), On([2, 4]), results()), (tree(), On([2, 5], torch.int64), results()),
           (tree(device=1), On([2, 5]), results()), (tree(), On([2, 5]), results(path=On([2, 3]))),
           (tree(), On([2, 5]), results(path=On([2, 4], torch.int64))),
           (tree(), On([2, 5]), results(n_accepted=On([1]))), (tree(), On([2, 5]), results(next_token=On([2], device=1)))]
    for name in ("tokens", "parents", "n_nodes"):
        for x in (On([2, 9]), On(getattr(tree(), name).shape, torch.int64), On(getattr(tree(), name).shape, device=1)):
            t = tree()
            setattr(t, name, x)
            if name != "tokens" or x.shape == (2, 4):     # (tokens' shape is the tree's)
                bad.append((t, On([2, 5]), results()))
    for n, (t, target, out) in enumerate(bad):
        with pytest.raises(ValueError):
            binding.accept_tree(t, target, out=out)
            pytest.fail(f"call {n} was made")
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 1)
    with pytest.raises(ValueError):
        binding.accept_tree(tree(), On([2, 5]), out=results())
    assert lib.made == ["dt_tree_accept"]


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
