"""The pages' calls refuse bad arguments on the host, before anything is launched (no GPU needed)."""
import ctypes

import pytest

from paper_2607_08642_amd import binding as b
from test_verify_abi import ALIGN, AT, CACHE_FAULTS, NULL, SHAPE, UNSUPPORTED, WORKSPACE, cache, ref


def pages(**kw):
    a = dict(pages=64, page_size=32, batch=4, table_width=8, uses=AT, held=AT, lens=AT, table=AT, missing=AT)
    a.update(kw)
    return b.dt_pages(*a.values())


def calls(p, c=None, ws=AT, size=1 << 30, source=AT):
    L, c = b.load(), cache() if c is None else c
    return {"fit": lambda: L.dt_pages_fit(ref(p), ws, size, None),
            "fork": lambda: L.dt_pages_fork(ref(p), ref(c), source, ws, size, None),
            "compact": lambda: L.dt_pages_compact(ref(p), ref(c), ws, size, None)}


@pytest.mark.parametrize("fault,status", [
    (dict(pages=0), SHAPE), (dict(batch=0), SHAPE), (dict(table_width=0), SHAPE), (dict(page_size=48), UNSUPPORTED),
    (dict(page_size=0), UNSUPPORTED), (dict(batch=65536), UNSUPPORTED), (dict(pages=0x7fffffff), UNSUPPORTED),
    (dict(table_width=1 << 25), UNSUPPORTED),
    (dict(batch=1 << 10, table_width=1 << 21), UNSUPPORTED)])
def test_sizes(fault, status):
    n = ctypes.c_size_t(7)
    assert b.load().dt_pages_workspace_size(ref(pages(**fault)), ref(n)) == status and n.value == 7
    for call in calls(pages(**fault)).values():
        assert call() == status


def test_pointers():
    for f in ("uses", "held", "lens", "table", "missing"):
        for x, status in ((None, NULL), (AT + 2, ALIGN)):
            for name, call in calls(pages(**{f: x})).items():
                assert call() == status, (f, name)
    for call in calls(None).values():
        assert call() == NULL
    n = ctypes.c_size_t()
    L = b.load()
    assert L.dt_pages_workspace_size(None, ref(n)) == NULL and L.dt_pages_workspace_size(ref(pages()), None) == NULL
    assert L.dt_pages_workspace_size(ref(pages(uses=None)), ref(n)) == 0 and n.value > 0
    for kw, status in ((dict(ws=None), WORKSPACE), (dict(size=n.value - 1), WORKSPACE), (dict(ws=AT + 128), ALIGN)):
        for call in calls(pages(), **kw).values():
            assert call() == status
    assert calls(pages(), source=None)["fork"]() == NULL and calls(pages(), source=AT + 2)["fork"]() == ALIGN


def test_caches():
    L = b.load()
    for fault, status in CACHE_FAULTS + [(dict(data=None), NULL), (dict(data=AT + 64), ALIGN)]:
        for name in ("fork", "compact"):
            assert calls(pages(), cache(**fault))[name]() == status
        assert L.dt_cache_copy_pages(ref(cache(**fault)), AT, AT, 3, None) == status
    for fault in (dict(pages=65), dict(page_size=64)):      # (not the books' cache)
        for name in ("fork", "compact"):
            assert calls(pages(), cache(**fault))[name]() == SHAPE
    many = cache(layers=1 << 20)
    assert calls(pages(batch=60000), many)["fork"]() == UNSUPPORTED


def test_copies():
    L, c = b.load(), cache()
    for a, status in (((None, AT, 3), NULL), ((AT, None, 3), NULL), ((AT + 2, AT, 3), ALIGN), ((AT, AT + 1, 3), ALIGN),
                      ((AT, AT, 0), SHAPE), ((AT, AT, -1), SHAPE), ((AT, AT, 0x7fffffff), UNSUPPORTED)):
        assert L.dt_cache_copy_pages(ref(c), *a, None) == status
