"""The verification calls refuse bad arguments on the host, before anything is launched (no GPU needed)."""
import ctypes

import pytest

from paper_2607_08642_amd import binding as b

NULL, SHAPE, DTYPE, UNSUPPORTED, WORKSPACE, ALIGN = (
    next(c for c, n in b.STATUS.items() if n.endswith(e))
    for e in ("ERR_NULL", "ERR_SHAPE", "ERR_DTYPE", "ERR_UNSUPPORTED", "ERR_WORKSPACE", "ERR_ALIGN"))
AT = 1 << 20      # an address that is never used


def ref(x):
    return None if x is None else ctypes.byref(x)


def cache(**kw):
    a = dict(data=AT, layers=2, pages=64, page_size=32, kv_heads=2, head_dim=64, dtype=b.DT_BF16)
    a.update(kw)
    return b.dt_cache(*a.values())


def chunk(**kw):
    a = dict(batch=2, rows=12, max_chunk=6, max_len=90, table_width=3, starts=AT, lens=AT, table=AT)
    a.update(kw)
    return b.dt_chunk(*a.values())


def options(**kw):
    a = dict(scale=0.1, window=0, sinks=0, tree_nodes=0, mask=None, depth=None)
    a.update(kw)
    return b.dt_attend_options(*a.values())


ROWS = b.dt_rows(AT, 128, 64)
CACHE_FAULTS = [(dict(dtype=7), DTYPE), (dict(layers=0), SHAPE), (dict(pages=0), SHAPE), (dict(kv_heads=-1), SHAPE),
                (dict(page_size=48), UNSUPPORTED), (dict(page_size=16), UNSUPPORTED),
                (dict(page_size=512), UNSUPPORTED), (dict(head_dim=80), UNSUPPORTED),
                (dict(kv_heads=5000), UNSUPPORTED)]
CHUNK_FAULTS = [(dict(batch=0), SHAPE), (dict(rows=0), SHAPE), (dict(max_chunk=0), SHAPE), (dict(max_len=0), SHAPE),
                (dict(table_width=0), SHAPE), (dict(max_chunk=13), SHAPE), (dict(max_len=97), SHAPE),
                (dict(max_len=5), SHAPE), (dict(batch=70000), UNSUPPORTED), (dict(table_width=1 << 26), UNSUPPORTED),
                (dict(table_width=0x7fffffff), UNSUPPORTED)]


def calls(c, k, rows=ROWS, layer=0):
    """Every call that takes a cache and a chunk."""
    L = b.load()
    n = ctypes.c_size_t()
    return {"append": lambda: L.dt_cache_append(ref(c), layer, ref(k), ref(rows), ref(ROWS), None),
            "read": lambda: L.dt_cache_read(ref(c), layer, ref(k), ref(ROWS), ref(rows), None),
            "size": lambda: L.dt_attend_workspace_size(ref(c), ref(k), 8, ref(options()), ref(n)),
            "attend": lambda: L.dt_cache_attend(ref(c), layer, ref(k), 8, ref(ROWS), ref(rows), ref(options()), None,
                                                0, None),
            "commit": lambda: L.dt_cache_commit(ref(c), ref(k), 4, AT, AT, None)}


@pytest.mark.parametrize("fault,status", CACHE_FAULTS)
def test_caches(fault, status):
    n = ctypes.c_size_t(7)
    assert b.load().dt_cache_size(ref(cache(**fault)), ref(n)) == status and n.value == 7
    for call in calls(cache(**fault), chunk()).values():
        assert call() == status


@pytest.mark.parametrize("fault,status", CHUNK_FAULTS)
def test_chunks(fault, status):
    for call in calls(cache(), chunk(**fault)).values():
        assert call() == status


def test_pointers():
    L = b.load()
    n = ctypes.c_size_t()
    assert L.dt_cache_size(None, ref(n)) == NULL and L.dt_cache_size(ref(cache()), None) == NULL
    for name, call in calls(None, chunk()).items():
        assert call() == NULL, name
    for name, call in calls(cache(), None).items():
        assert call() == NULL, name
    faults = [(dict(data=None), {}, NULL), (dict(data=AT + 64), {}, ALIGN)]
    faults += [({}, {f: x}, s) for f in ("starts", "lens", "table") for x, s in ((None, NULL), (AT + 2, ALIGN))]
    for of_cache, of_chunk, status in faults:
        for name, call in calls(cache(**of_cache), chunk(**of_chunk)).items():
            if name != "size":       # (a size needs no data)
                assert call() == status, (name, of_cache, of_chunk)
    for rows, status in ((None, NULL), (b.dt_rows(None, 128, 64), NULL), (b.dt_rows(AT + 1, 128, 64), ALIGN),
                         (b.dt_rows(AT, -128, 64), SHAPE), (b.dt_rows(AT, 128, -64), SHAPE)):
        for name in ("append", "read", "attend"):
            assert calls(cache(), chunk(), rows)[name]() == status, name
    for layer in (-1, 2):
        for name in ("append", "read", "attend"):
            assert calls(cache(), chunk(), ROWS, layer)[name]() == SHAPE, name


def test_sizes():
    """Bytes of a cache: every layer's, page's and head's keys and values; 8-bit ones have a scale byte each."""
    n = ctypes.c_size_t()
    for dtype, token in ((b.DT_F32, 2 * 96 * 4), (b.DT_BF16, 2 * 96 * 2), (b.DT_F8, 2 * 96 + 2)):
        c = cache(data=None, layers=3, pages=5000, page_size=128, kv_heads=7, head_dim=96, dtype=dtype)
        assert b.load().dt_cache_size(ref(c), ref(n)) == 0
        assert n.value == 3 * 5000 * 7 * 128 * token


@pytest.mark.parametrize("heads,opts,status", [
    (0, {}, SHAPE), (3, {}, SHAPE), (4096, {}, UNSUPPORTED), (8, dict(window=-1), SHAPE), (8, dict(sinks=-1), SHAPE),
    (8, dict(tree_nodes=-1), SHAPE), (8, dict(tree_nodes=7), SHAPE), (8, dict(tree_nodes=5000), UNSUPPORTED),
    (8, dict(scale=float("nan")), SHAPE), (8, dict(scale=float("inf")), SHAPE), (8, None, NULL)])
def test_attention(heads, opts, status):
    n = ctypes.c_size_t()
    o = None if opts is None else options(**opts)
    L = b.load()
    assert L.dt_attend_workspace_size(ref(cache()), ref(chunk()), heads, ref(o), ref(n)) == status
    assert L.dt_cache_attend(ref(cache()), 0, ref(chunk()), heads, ref(ROWS), ref(ROWS), ref(o), None, 0,
                             None) == status


def test_attention_trees_and_workspace():
    L = b.load()

    def status(o, k=None, ws=None, size=0):
        return L.dt_cache_attend(ref(cache()), 0, ref(k or chunk()), 8, ref(ROWS), ref(ROWS), ref(o), ws, size, None)

    assert status(options(tree_nodes=4)) == NULL                                        # no mask
    assert status(options(tree_nodes=4, mask=AT, window=9)) == NULL                     # a window needs depths
    assert status(options(tree_nodes=4, mask=AT, window=9, depth=AT + 1)) == ALIGN
    long = chunk(batch=1, rows=1, max_chunk=1, max_len=1 << 20, table_width=1 << 15)    # (long enough for parts)
    n = ctypes.c_size_t()
    assert L.dt_attend_workspace_size(ref(cache()), ref(long), 8, ref(options()), ref(n)) == 0 and n.value > 0
    assert L.dt_attend_workspace_size(ref(cache()), ref(long), 8, ref(options()), None) == NULL
    assert status(options(), long) == WORKSPACE
    assert status(options(), long, AT, n.value - 1) == WORKSPACE
    assert status(options(), long, AT + 128, n.value) == ALIGN


def test_launches_that_do_not_fit():
    """More workgroups than a launch can count."""
    n = ctypes.c_size_t()
    L = b.load()
    wide = chunk(batch=1, rows=1 << 27, max_chunk=1 << 27, max_len=1 << 27, table_width=1 << 22)
    assert L.dt_cache_append(ref(cache(kv_heads=4)), 0, ref(wide), ref(ROWS), ref(ROWS), None) == UNSUPPORTED
    assert L.dt_cache_read(ref(cache(kv_heads=4)), 0, ref(wide), ref(ROWS), ref(ROWS), None) == UNSUPPORTED
    assert L.dt_attend_workspace_size(ref(cache()), ref(wide), 4, ref(options()), ref(n)) == UNSUPPORTED
    assert L.dt_cache_commit(ref(cache(layers=1 << 23, pages=1)), ref(chunk()), 4, AT, AT, None) == UNSUPPORTED


def test_accept_and_commit():
    L = b.load()
    fields = [f for f, _ in b.dt_tree._fields_]

    def accept(tree=True, batch=2, B=16, **kw):
        t = b.dt_tree(*(AT for _ in fields))
        outs = dict(target=AT, path=AT, n_accepted=AT, next_token=AT)
        for name, x in kw.items():
            if name in outs:
                outs[name] = x
            else:
                setattr(t, name, x)
        return L.dt_tree_accept(ref(t) if tree else None, batch, B, *outs.values(), None)

    assert accept(tree=False) == NULL
    for name in ("tokens", "parents", "n_nodes", "target", "path", "n_accepted", "next_token"):
        assert accept(**{name: None}) == NULL and accept(**{name: AT + 2}) == ALIGN, name
    assert accept(batch=0) == SHAPE and accept(B=0) == SHAPE and accept(B=1 << 14) == UNSUPPORTED
    assert accept(batch=1 << 24) == UNSUPPORTED

    def commit(nodes=4, path=AT, n=AT, k=None):
        return L.dt_cache_commit(ref(cache()), ref(k or chunk()), nodes, path, n, None)

    assert commit(path=None) == NULL and commit(n=None) == NULL
    assert commit(path=AT + 1) == ALIGN and commit(n=AT + 1) == ALIGN
    assert commit(nodes=0) == SHAPE and commit(nodes=7) == SHAPE
    assert commit(nodes=5000, k=chunk(rows=6000, max_chunk=6000, max_len=6000, table_width=200)) == UNSUPPORTED
