"""The paged cache (append, read, commit) and the accepted path, against plain 64-bit forms.

Everything here is exact: rows are copied, the 8-bit codes are defined by a power-of-two scale and a
rounding to nearest even, and the values that they stand for are exact in bf16."""
import random

import numpy as np
import pytest
import torch

import verify_ref as ref
from paper_2607_08642_amd import binding

pytestmark = pytest.mark.gpu
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f8": torch.float8_e4m3fn}


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Setup:
    """A cache full of NaN bytes, a shuffled page table, ragged chunks ending at ragged lengths."""

    def __init__(self, dtype, sizes, page=32, kv=2, D=64, layers=1, seed=0):
        self.sizes, self.page, self.kv, self.D = sizes, page, kv, D
        g = torch.Generator().manual_seed(seed)
        width = max(-(-n // page) for n, _ in sizes)
        pages = len(sizes) * width + 2
        self.cache = binding.Cache(pages, page, kv, D, DTYPES[dtype], layers=layers)
        self.cache.storage.fill_(0xff)
        self.table = torch.randperm(pages, generator=g)[:len(sizes) * width].reshape(len(sizes), width).int()
        self.starts = np.concatenate([[0], np.cumsum([m for _, m in sizes])]).tolist()
        self.rows = self.starts[-1]
        self.chunk = self.make(sizes)
        self.g = g

    def make(self, sizes):
        starts = np.concatenate([[0], np.cumsum([m for _, m in sizes])]).tolist()
        return binding.Chunk(i32(starts), i32([n for n, _ in sizes]), self.table.cuda(),
                             max(max(m for _, m in sizes), 1), max(n for n, _ in sizes))

    def randn(self, rows, heads=None):
        return torch.randn(rows, heads or self.kv, self.D, generator=self.g).to(self.cache.data_dtype)


def held(s, x):
    return ref.quantise(x).to(torch.bfloat16) if s.cache.dtype == torch.float8_e4m3fn else x


def same(a, b):
    a, b = a.float().cpu(), b.float().cpu()
    return torch.equal(torch.nan_to_num(a, nan=12345.0), torch.nan_to_num(b, nan=12345.0))


SIZES = [[(1, 1)], [(33, 1), (32, 1), (31, 1), (64, 1)], [(100, 37), (37, 37), (70, 3), (5, 0), (64, 64)],
         [(300, 257), (129, 128)]]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f8"])
@pytest.mark.parametrize("D,page", [(64, 32), (96, 64), (128, 128), (256, 256)])
@pytest.mark.parametrize("which", range(len(SIZES)))
def test_append_then_read(dtype, D, page, which):
    print(f"[cache] {dtype} D={D} page={page} sizes={SIZES[which]}", flush=True)
    s = Setup(dtype, SIZES[which], page, kv=3, D=D, seed=which)
    k, v = s.randn(s.rows), s.randn(s.rows)
    s.cache.append(s.chunk, k.cuda(), v.cuda())
    gk, gv = s.cache.read(s.chunk, s.rows)
    assert same(gk, held(s, k)) and same(gv, held(s, v))


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f8"])
def test_tokens_one_by_one(dtype):
    """A token's row leaves its neighbours in block and page as they are; the last layer of three."""
    s = Setup(dtype, [(70, 70), (41, 41)], 32, kv=2, D=96, layers=3, seed=5)
    k, v = s.randn(s.rows), s.randn(s.rows)
    for p in range(70):
        sizes = [(p + 1, 1), (min(p, 40) + 1, 1 if p < 41 else 0)]
        rows = [p] + ([70 + p] if p < 41 else [])
        s.cache.append(s.make(sizes), k[rows].cuda(), v[rows].cuda(), layer=2)
    gk, gv = s.cache.read(s.chunk, s.rows, layer=2)
    assert same(gk, held(s, k)) and same(gv, held(s, v))
    other = s.cache.storage.view(3, -1)[:2]
    assert bool((other == 0xff).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f8"])
def test_strided_rows(dtype):
    """Rows of a fused [rows, 3, heads, D] tensor, heads before rows, and addresses one element off."""
    s = Setup(dtype, [(50, 50), (40, 13)], 64, kv=2, D=64, seed=7)
    dt = s.cache.data_dtype
    k, v = s.randn(s.rows), s.randn(s.rows)
    fused = torch.zeros(s.rows, 3, 2, 64, dtype=dt, device="cuda")
    fused[:, 1], fused[:, 2] = k.cuda(), v.cuda()
    turned = torch.zeros(2, s.rows, 64, dtype=dt, device="cuda").transpose(0, 1)
    off = torch.zeros(s.rows * 128 + 1, dtype=dt, device="cuda")[1:].view(s.rows, 2, 64)
    turned.copy_(k)
    off.copy_(v)
    for kk, vv in ((fused[:, 1], fused[:, 2]), (turned, off), (off.clone().copy_(k), turned.clone().copy_(v))):
        s.cache.storage.fill_(0xff)
        s.cache.append(s.chunk, kk, vv)
        ok, ov = torch.zeros_like(fused)[:, 0], torch.zeros(s.rows * 128 + 1, dtype=dt, device="cuda")[1:].view(s.rows, 2, 64)
        s.cache.read(s.chunk, out=(ok, ov))
        assert same(ok, held(s, k)) and same(ov, held(s, v))


def test_codes_of_eight_bits():
    """Ties, the ends of the range, subnormals, zeros, infinities and NaN; every finite code comes back as itself."""
    D = 256
    codes = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float()
    rows = [codes, codes * 2.0 ** 9, torch.zeros(D), torch.full((D,), -0.0),
            torch.linspace(-448, 448, D), torch.linspace(-449, 449, D), torch.linspace(-1e-3, 1e-3, D) ** 3,
            torch.full((D,), 3.3e38), torch.full((D,), 1e-38)]
    ties = torch.arange(D).float() / 16          # halves between codes
    ties[-1] = 448.0
    rows += [ties, ties * 2.0 ** -7]
    bad = torch.randn(D, generator=torch.Generator().manual_seed(1))
    bad[3], bad[77], bad[200] = float("inf"), float("nan"), float("-inf")
    rows.append(bad)
    x = torch.stack(rows)[:, None].to(torch.bfloat16)
    s = Setup("f8", [(len(rows), len(rows))], 32, kv=1, D=D)
    s.cache.append(s.chunk, x.cuda(), x.cuda())
    for got in s.cache.read(s.chunk, len(rows)):
        assert same(got, ref.quantise(x).to(torch.bfloat16))
    assert same(s.cache.read(s.chunk, len(rows))[0][0, 0], codes)


def test_pages_out_of_range():
    """Tokens of a page that is not there: written nowhere, read as zeros."""
    s = Setup("bf16", [(96, 96)], 32, kv=1, D=64)
    s.table[0, 1] = 10 ** 6
    s.chunk = s.make(s.sizes)
    k, v = s.randn(96), s.randn(96)
    s.cache.append(s.chunk, k.cuda(), v.cuda())
    gk, gv = (t.cpu() for t in s.cache.read(s.chunk, 96))
    for got, x in ((gk, k), (gv, v)):
        assert same(got[:32], x[:32]) and same(got[64:], x[64:]) and not got[32:64].any()


def random_tree(rng, N, B, depth=16):
    """Parents first, siblings of distinct tokens; padded to B."""
    par = []
    dep = []
    for i in range(N):
        p = rng.choice([-1, i - 1, rng.randrange(i)]) if i else -1
        if p >= 0 and dep[p] >= depth:
            p = -1
        par.append(p)
        dep.append(1 if p < 0 else dep[p] + 1)
    tok = [5 + 3 * i for i in range(N)]
    pad = B - N
    return tok + [-1] * pad, par + [-1] * pad, dep + [0] * pad


def device_tree(trees, B):
    t = binding.Tree.empty(len(trees), B, "cuda")
    t.tokens.copy_(i32([x[0] for x in trees]))
    t.parents.copy_(i32([x[1] for x in trees]))
    return t


@pytest.mark.parametrize("B", [1, 2, 16, 64, 65, 256])
def test_accept(B):
    rng = random.Random(B)
    trees, counts, targets = [], [], []
    for b in range(9):
        N = [B, B, 0, 1, max(1, B // 2)][b % 5]
        tok, par, dep = random_tree(rng, N, B)
        if b == 1:     # a chain, followed to a depth past the builder's
            par = list(range(-1, N - 1))
        tgt = []
        for at in range(-1, B):
            kids = [i for i in range(N) if par[i] == at]
            # (-1: the padding's token, which must not match it)
            tgt.append(tok[rng.choice(kids)] if kids and (b == 1 or rng.random() < 0.9) else rng.choice([-1, 2]))
        trees.append((tok, par, dep))
        counts.append(N)
        targets.append(tgt)
    tree = device_tree(trees, B)
    tree.n_nodes.copy_(i32(counts))
    a = binding.accept_tree(tree, i32(targets))
    deepest = 0
    for b, (tok, par, _) in enumerate(trees):
        path, nxt = ref.accept(tok, par, counts[b], targets[b])
        assert a.n_accepted[b].item() == len(path) and a.next_token[b].item() == nxt
        assert a.path[b].tolist() == path + [-1] * (B - len(path))
        deepest = max(deepest, len(path))
    assert deepest > 2 or B <= 2


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f8"])
@pytest.mark.parametrize("N,D,page", [(1, 64, 32), (16, 128, 64), (64, 96, 32), (200, 64, 64)])
def test_commit(dtype, N, D, page):
    """Accepted rows in their new places, every other row as it was, in both layers."""
    rng = random.Random(N)
    sizes = [(N + 40, N + 1), (N + 1, N + 1), (N + 77, N + 3), (N + 31, N + 1)]
    s = Setup(dtype, sizes, page, kv=2, D=D, layers=2, seed=N)
    paths = [sorted(rng.sample(range(N), n)) for n in (N // 2, N, 0, min(N, 9))]
    rows = [[s.randn(s.rows), s.randn(s.rows)] for _ in range(2)]
    for n, (k, v) in enumerate(rows):
        s.cache.append(s.chunk, k.cuda(), v.cuda(), layer=n)
    path = i32([p + [-1] * (N - len(p)) for p in paths])
    s.cache.commit(s.chunk, path, i32([len(p) for p in paths]))
    for n in range(2):
        got = s.cache.read(s.chunk, s.rows, layer=n)
        for g, x in zip(got, rows[n]):
            want = held(s, x).clone()
            for b, p in enumerate(paths):
                first = s.starts[b + 1] - N
                want[first:first + len(p)] = held(s, x)[[first + i for i in p]]
            assert same(g, want)


def test_commit_leaves_out_bad_entries():
    """Entries below their index, past the tree or negative move nothing."""
    s = Setup("bf16", [(20, 9)], 32, kv=1, D=64)
    k, v = s.randn(9), s.randn(9)
    s.cache.append(s.chunk, k.cuda(), v.cuda())
    s.cache.commit(s.chunk, i32([[3, 0, 8, 900, -5, 6, 6, 7]]), i32([6]))
    want = k.clone()
    want[1], want[6] = k[4], k[7]      # (row 1 is node 0)
    assert same(s.cache.read(s.chunk, 9)[0], want)


def test_refusals():
    s = Setup("bf16", [(20, 9)], 32, kv=2, D=64)
    x = s.randn(9).cuda()
    with pytest.raises(ValueError):
        s.cache.append(s.chunk, x.float(), x)
    with pytest.raises(ValueError):
        s.cache.append(s.chunk, x[:, :1], x)
    with pytest.raises(ValueError):
        s.cache.append(s.chunk, x, x[:8])
    with pytest.raises(ValueError):
        s.cache.append(s.chunk, x.transpose(1, 2).contiguous().transpose(1, 2), x)
    with pytest.raises(binding.DTError) as e:
        s.cache.append(s.chunk, x, x, layer=1)
    assert e.value.status == -2
    for bad in (dict(page_size=16), dict(page_size=48), dict(head_dim=80)):
        kw = dict(pages=2, page_size=32, kv_heads=1, head_dim=64, dtype=torch.bfloat16)
        kw.update(bad)
        with pytest.raises(binding.DTError) as e:
            binding.Cache(**kw)
        assert e.value.status == -4
    with pytest.raises(TypeError):
        binding.Cache(2, 32, 1, 64, torch.float16)
    with pytest.raises(binding.DTError) as e:   # longer than the table
        binding.Cache.append(s.cache, binding.Chunk(s.chunk.starts, s.chunk.lens, s.chunk.table, 9, 33), x, x)
    assert e.value.status == -2
    with pytest.raises(ValueError):
        binding.Chunk(s.chunk.starts.long(), s.chunk.lens, s.chunk.table, 9, 20)
