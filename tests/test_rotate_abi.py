"""The rotation's calls refuse bad arguments on the host, before anything is launched (no GPU needed)."""
import pytest

from paper_2607_08642_amd import binding as b
from test_verify_abi import ALIGN, AT, CACHE_FAULTS, CHUNK_FAULTS, DTYPE, NULL, ROWS, SHAPE, UNSUPPORTED, cache, chunk, ref


def rotary(**kw):
    a = dict(positions=AT, inv_freq=AT, pairs=32, interleaved=0, q_weight=AT, k_weight=AT, eps=1e-6)
    a.update(kw)
    return b.dt_rotary(*a.values())


def rotate(r=None, q=ROWS, heads=8, k=ROWS, kv=2, rows=12, D=64, dtype=b.DT_BF16, q_out=ROWS, k_out=ROWS, **kw):
    return b.load().dt_rotate(ref(q), heads, ref(k), kv, rows, D, dtype, ref(rotary(**kw) if r is None else r), ref(q_out),
                              ref(k_out), None)


def append(c=None, k=None, layer=0, heads=8, q=ROWS, kk=ROWS, v=ROWS, q_out=ROWS, r=None, **kw):
    return b.load().dt_cache_append_rotated(ref(c or cache()), layer, ref(k or chunk()), heads, ref(q), ref(kk), ref(v),
                                            ref(rotary(**kw) if r is None else r), ref(q_out), None)


ROTARY_FAULTS = [(dict(positions=None), NULL), (dict(inv_freq=None), NULL), (dict(pairs=0), SHAPE), (dict(pairs=-8), SHAPE),
                 (dict(pairs=12), SHAPE), (dict(pairs=40), SHAPE), (dict(eps=-1e-6), SHAPE), (dict(eps=float("nan")), SHAPE),
                 (dict(eps=float("inf")), SHAPE), (dict(positions=AT + 2), ALIGN), (dict(inv_freq=AT + 1), ALIGN),
                 (dict(q_weight=AT + 8), ALIGN), (dict(k_weight=AT + 2), ALIGN)]
ROWS_FAULTS = [(b.dt_rows(None, 128, 64), NULL), (b.dt_rows(AT + 1, 128, 64), ALIGN), (b.dt_rows(AT, -128, 64), SHAPE),
               (b.dt_rows(AT, 128, -64), SHAPE)]


@pytest.mark.parametrize("fault,status", ROTARY_FAULTS)
def test_rotaries(fault, status):
    assert rotate(**fault) == status and append(**fault) == status


@pytest.mark.parametrize("rows,status", ROWS_FAULTS)
def test_rows(rows, status):
    for name in ("q", "k", "q_out", "k_out"):
        assert rotate(**{name: rows}) == status, name
    for name in ("q", "kk", "v", "q_out"):
        assert append(**{name: rows}) == status, name


@pytest.mark.parametrize("sizes,status", [
    (dict(dtype=b.DT_F8), DTYPE), (dict(dtype=9), DTYPE), (dict(rows=0), SHAPE), (dict(heads=0), SHAPE), (dict(kv=-1), SHAPE),
    (dict(kv=0), SHAPE), (dict(k=None, kv=2), SHAPE), (dict(k=None, kv=0), SHAPE), (dict(k_out=None), SHAPE),
    (dict(D=0), UNSUPPORTED), (dict(D=72), UNSUPPORTED), (dict(D=528), UNSUPPORTED), (dict(heads=1 << 20), UNSUPPORTED),
    (dict(kv=(1 << 20) - 8), UNSUPPORTED), (dict(kv=0x7fffffff), UNSUPPORTED), (dict(rows=1 << 26), UNSUPPORTED),
    (dict(rows=0x7fffffff), UNSUPPORTED)])
def test_sizes(sizes, status):
    assert rotate(**sizes) == status


def test_appends():
    for fault, status in CACHE_FAULTS:
        assert append(cache(**fault)) == status
    for fault, status in CHUNK_FAULTS:
        assert append(k=chunk(**fault)) == status
    assert append(cache(data=None)) == NULL and append(cache(data=AT + 64)) == ALIGN
    assert append(layer=2) == SHAPE and append(layer=-1) == SHAPE
    assert append(heads=0) == SHAPE and append(heads=1 << 20) == SHAPE
    wide = chunk(batch=1, rows=1 << 20, max_chunk=1 << 20, max_len=1 << 20, table_width=1 << 16)
    assert append(k=wide, heads=64) == UNSUPPORTED
    for name in ("q", "kk", "v", "q_out"):
        assert append(**{name: None}) == NULL, name
    assert b.load().dt_cache_append_rotated(ref(cache()), 0, ref(chunk()), 8, ref(ROWS), ref(ROWS), ref(ROWS), None,
                                            ref(ROWS), None) == NULL
    assert b.load().dt_rotate(ref(ROWS), 8, None, 0, 12, 64, b.DT_F32, None, ref(ROWS), None, None) == NULL


def test_the_first_sizes_past_the_limits():
    assert rotate(rows=(1 << 26) - 4) == UNSUPPORTED
    n = 621378 * 32                               # n * 3 / 4 + (n / 32 + 3) * 3 = 2^24 - 1
    wide = chunk(batch=1, rows=n, max_chunk=n, max_len=n, table_width=1 << 20)
    assert append(cache(kv_heads=3), k=wide, heads=3) == UNSUPPORTED
