"""Attention where its paths meet: windows, trees, unseen non-finite values and missing pages at every head size and in
calls of few rows (at 256 a head two waves share a block there), and all of them in calls whose axis is split.

Tolerances are those of test_gpu_attend."""
import numpy as np
import pytest
import torch

import verify_ref as ref
from paper_2607_08642_amd import binding
from test_gpu_attend import TYPES, Attend, allowed, trees
from test_gpu_cache import i32, same

pytestmark = pytest.mark.gpu


def splits(a, chunk=None, window=0, nodes=0):
    """In how many parts a call is cut, from the size of its workspace (sums of D, two words and a count a part)."""
    o = binding.dt_attend_options(0.1, window, 0, nodes, None, None)
    size = a.cache.workspace_size(chunk or a.chunk, a.rows, a.heads, o)
    rows = a.rows * a.heads
    up = lambda x: (x + 255) // 256 * 256  # noqa: E731
    return next(s for s in range(1, 65) if size == (up(rows * (s + 1) * 8) + up(rows * s * a.D * 4) if s > 1 else 0))


TOKENS = [(1, 1), (31, 1), (33, 1), (64, 1), (97, 1), (257, 1), (700, 1)]     # (blocks: odd and even numbers of them)
CHUNKS = [(300, 37), (129, 129), (70, 1), (513, 64)]                            # (fp32: calls of 32 rows at a time)


@pytest.mark.parametrize("dtype,sizes", [(t, TOKENS) for t in TYPES] + [(t, CHUNKS) for t in TYPES],
                         ids=[f"{t}-{s}" for s in ("tokens", "chunks") for t in TYPES])
@pytest.mark.parametrize("D", [96, 128, 256])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 3), (33, 1), (50, 32), (64, 40), (5000, 4)])
def test_windows(dtype, sizes, D, window, sinks):
    print(f"[paths] window {dtype} D={D} {window}/{sinks} {len(sizes)}", flush=True)
    a = Attend(dtype, sizes, 8, 32, 2, D, seed=window % 1000 + D)
    a.check(a.run(window=window, sinks=sinks), window=window, sinks=sinks)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D", [96, 128, 256])
@pytest.mark.parametrize("N,lead", [(1, 0), (6, 1), (7, 1), (40, 2)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (20, 5)])
def test_trees_of_few_and_many_rows(dtype, D, N, lead, window, sinks):
    sizes = [(n + N + lead, N + lead) for n in (0, 1, 31, 90, 64)]
    print(f"[paths] tree {dtype} D={D} N={N} lead={lead} window={window}", flush=True)
    a = Attend(dtype, sizes, 8, 64, 2, D, seed=N + D)
    masks, depths = trees(sizes, N, N)
    got = a.run(mask=torch.from_numpy(np.stack(masks)).cuda(), depth=i32(depths), window=window, sinks=sinks)
    a.check(got, window=window, sinks=sinks, masks=masks, depths=depths)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D", [96, 256])
@pytest.mark.parametrize("N", [6, 16])
def test_unseen_nonfinite_nodes(dtype, D, N):
    """A node of NaN keys and infinite values: rows that see it are not finite, the others' bits stay."""
    sizes = [(N + 41, N + 1), (N + 200, N + 1)]
    masks, _ = trees(sizes, N, 4)
    mask = torch.from_numpy(np.stack(masks)).cuda()
    a = Attend(dtype, sizes, 8, 32, 2, D, seed=D)
    clean = a.run(mask=mask)
    bad, k, v = 2, a.k.clone(), a.v.clone()
    for end in np.cumsum([n for n, _ in sizes]):
        k[end - N + bad] = float("nan")
        v[end - N + bad] = float("inf")
    a.cache.append(a.make([(n, n) for n, _ in sizes]), k.cuda(), v.cuda())
    got = a.run(mask=mask)
    hit = 0
    for b in range(2):
        first = a.starts[b + 1] - N
        for i in range(-1, N):
            if i >= 0 and masks[b][i][bad]:
                hit += 1
                assert not bool(torch.isfinite(got[first + i]).any())
            else:
                assert same(got[first + i], clean[first + i]), (b, i)
    assert hit > 0


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D", [96, 256])
@pytest.mark.parametrize("chunk", [1, 40])
def test_missing_pages(dtype, D, chunk):
    """Tokens of pages that are not there are not seen: one in the middle, the first, and all of a sequence's."""
    a = Attend(dtype, [(96, 1), (130, chunk), (64, 1)], 4, 32, 2, D, seed=D + chunk)
    table = a.table.clone()
    table[0, 1], table[1, 0], table[2] = -7, 10 ** 6, -1
    got = a.cache.attend(binding.Chunk(a.chunk.starts, a.chunk.lens, table.cuda(), max(chunk, 1), 130), a.q.cuda())
    hk, hv = (x if dtype != "f8" else ref.quantise(x).bfloat16() for x in (a.k, a.v))
    for b, (first, n, m, gone) in enumerate([(0, 96, 1, range(32, 64)), (96, 130, chunk, range(32)), (226, 64, 1, range(64))]):
        r0 = a.starts[b]
        ok = ref.visible(m, n - m, n, 0, 0)
        keep = [j for j in range(n) if j not in gone]
        k, v = hk[first:first + n][keep], hv[first:first + n][keep]
        want = ref.attend(a.q[r0:r0 + m], k, v, D ** -0.5, ok[:, keep])
        tol = allowed(a.q[r0:r0 + m], k, v, D ** -0.5, ok[:, keep], a.cache.data_dtype) if keep else torch.zeros_like(want)
        assert bool(((got[r0:r0 + m].double().cpu() - want).abs() <= tol).all()), b


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("sizes,N", [([(6000, 17)], 16), ([(6000, 7)], 6), ([(5000, 17), (40, 17)], 16)])
def test_trees_under_windows_in_parts(dtype, D, sizes, N):
    """Trees whose window begins thousands of tokens back: several parts of one window, and the first tokens'."""
    print(f"[paths] parts {dtype} D={D} {sizes} N={N}", flush=True)
    a = Attend(dtype, sizes, 4, 64, 1, D, seed=N + D)
    assert splits(a, window=3000, nodes=N) > 4
    masks, depths = trees(sizes, N, N)
    got = a.run(mask=torch.from_numpy(np.stack(masks)).cuda(), depth=i32(depths), window=3000, sinks=70)
    a.check(got, window=3000, sinks=70, masks=masks, depths=depths)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D", [64, 96, 128, 256])
def test_many_parts(dtype, D):
    """One token over 20,000: more parts than the lanes that a row of 64 is joined by."""
    print(f"[paths] many parts {dtype} D={D}", flush=True)
    a = Attend(dtype, [(20000, 1)], 4, 128, 1, D, seed=D)
    assert splits(a) > 16
    a.check(a.run())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D", [64, 256])
def test_lengths_far_below_their_bound(dtype, D):
    """A plan for 32,768 tokens at lengths of 1 to 3,000, as a captured graph has it: parts without a block."""
    print(f"[paths] bound {dtype} D={D}", flush=True)
    a = Attend(dtype, [(3000, 1), (1, 1), (700, 1)], 4, 64, 1, D, seed=D)
    wide = torch.full((3, 512), -1, dtype=torch.int32)
    wide[:, :a.table.shape[1]] = a.table
    a.chunk = binding.Chunk(a.chunk.starts, a.chunk.lens, wide.cuda(), 1, 32768)
    assert splits(a) > 4
    a.check(a.run())
