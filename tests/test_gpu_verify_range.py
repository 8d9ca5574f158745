"""The verification calls at the ends of their range: offsets beyond 32 bits in the cache and in the rows, one
sequence with enough rows for the widest workgroups, and tensors of another stream.

Tolerances are those of the attention tests; where both sides run the same kernels on the same values the bits have
to be the same."""
import pytest
import torch

from paper_2607_08642_amd import binding
from test_gpu_attend import Attend, trees
from test_gpu_cache import DTYPES, i32, same

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f8"])
def test_pages_beyond_4_gib(dtype):
    """The same rows in a cache's last pages, and in a small cache: the same bits from every call."""
    page, kv, D = 256, 2, 128
    per_page = page * kv * 2 * D * {"f32": 4, "bf16": 2, "f8": 1}[dtype]
    many = (9 << 29) // per_page                 # 4.5 GiB
    g = torch.Generator().manual_seed(5)
    n, m = 700, 40
    k, v = (torch.randn(n, kv, D, generator=g).cuda().to(binding.Cache(1, 32, 1, 64, DTYPES[dtype]).data_dtype)
            for _ in "kv")
    q = torch.randn(m, 8, D, generator=g).cuda().to(k.dtype)
    path, count = i32([[3, 5, 20] + [-1] * 29]), i32([3])
    results = []
    for pages in (4, many):
        print(f"[range] {dtype} pages={pages}", flush=True)
        c = binding.Cache(pages, page, kv, D, DTYPES[dtype])
        table = i32([[pages - 2, pages - 4, pages - 1]])
        every = binding.Chunk(i32([0, n]), i32([n]), table, n, n)
        last = binding.Chunk(i32([0, m]), i32([n]), table, m, n)
        c.append(every, k, v)
        out = [*c.read(every, n), c.attend(last, q), c.attend(last, q[:, :2].contiguous(), window=50, sinks=3)]
        c.commit(last, path, count)
        results.append(out + [*c.read(every, n)])
    for a, b in zip(*results):
        assert same(a, b)
    assert c.storage.numel() > 1 << 32


@pytest.mark.parametrize("dtype", ["bf16", "f8"])
def test_rows_beyond_32_bit_offsets(dtype):
    """Rows 2^27 elements apart: the last lie past 2^31 elements and 2^32 bytes."""
    a = Attend(dtype, [(50, 33)], 2, 32, 1, 64, seed=21)
    k, v = a.randn(33).cuda(), a.randn(33).cuda()
    a.cache.append(a.chunk, k, v)
    held_k, held_v = a.cache.read(a.chunk, 33)
    want = a.run()
    big = torch.empty(33 * (1 << 27), dtype=torch.bfloat16, device="cuda")
    wide = lambda at, heads: big.as_strided((33, heads, 64), (1 << 27, 64, 1), at)  # noqa: E731
    q, out, kk, vv = wide(0, 2), wide(128, 2), wide(256, 1), wide(320, 1)
    q.copy_(a.q.cuda())
    kk.copy_(k)
    vv.copy_(v)
    a.cache.storage.fill_(0xff)
    every = a.make([(50, 50)])
    a.cache.append(every, a.k.cuda(), a.v.cuda())
    a.cache.append(a.chunk, kk, vv)
    a.cache.attend(a.chunk, q, out=out)
    assert same(out, want)
    kk.zero_()
    vv.zero_()
    a.cache.read(a.chunk, out=(kk, vv))
    assert same(kk, held_k) and same(vv, held_v)


@pytest.mark.parametrize("dtype", ["bf16", "f8"])
@pytest.mark.parametrize("D,window,nodes", [(64, 0, 0), (96, 70, 0), (128, 0, 24), (256, 40, 24)])
def test_one_sequence_of_many_rows(dtype, D, window, nodes):
    """512 heads and chunks over 32 rows: workgroups of the largest kind, two tiles, the second one uneven."""
    print(f"[range] many rows {dtype} D={D} window={window} nodes={nodes}", flush=True)
    a = Attend(dtype, [(303, 290)], 512, 64, 512, D, seed=D)
    kw = dict(window=window, sinks=5 if window else 0)
    masks = depths = None
    if nodes:
        masks, depths = trees([0], nodes, D)
        kw["mask"] = torch.from_numpy(masks[0])[None].cuda()
        if window:
            kw["depth"] = i32(depths)
    got = a.run(**kw)
    some = [0, 1, 254, 511]       # (each head has keys of its own: these are compared)
    a.q, a.k, a.v, got = (x[:, some] for x in (a.q, a.k, a.v, got))
    a.check(got, window=window, sinks=kw["sinks"], masks=masks, depths=depths)


def test_streams_of_their_own():
    """Outputs and workspaces made for another stream, in use there while this one reuses its memory."""
    a = Attend("bf16", [(6000, 2)], 8, 64, 2, 128, seed=31)
    q = a.q.cuda()
    want = a.run()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    outs = []
    for n in range(30):
        junk = torch.full((2, 8, 128), float(n), dtype=torch.bfloat16, device="cuda")
        del junk
        outs.append(a.cache.attend(a.chunk, q.clone(), stream=ordered(side)))
    torch.cuda.current_stream().wait_stream(side)
    for o in outs:
        assert same(o, want)


def ordered(side):
    """The side stream after what this one has made so far."""
    side.wait_stream(torch.cuda.current_stream())
    return side
