"""Pages of sequences against the same books as Python lists: everything is whole numbers and copies, so exact."""
import random

import pytest
import torch

from pages_ref import Books
from paper_2607_08642_amd import binding
from test_gpu_cache import i32, same

pytestmark = pytest.mark.gpu


class Both:
    """The calls and the lists side by side."""

    def __init__(self, pages, page_size, batch, width, kv=2, D=64, layers=2, dtype=torch.bfloat16, seed=0):
        self.rng = random.Random(seed)
        self.cache = binding.Cache(pages, page_size, kv, D, dtype, layers=layers)
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.cache.storage.random_(generator=g)
        self.first = self.bytes().clone()
        self.pages = binding.Pages(self.cache, batch, width)
        self.books = Books(pages, page_size, batch, width)

    def bytes(self):
        return self.cache.storage.view(self.cache.layers, self.cache.pages, -1)

    def set(self, lens):
        self.books.lens = list(lens)
        self.pages.lens.copy_(i32(lens))

    def check(self):
        p, k = self.pages, self.books
        assert int(p.missing) == k.missing
        assert p.lens.tolist() == k.lens and p.held.tolist() == [len(r) for r in k.rows]
        assert p.table.tolist() == [r + [-1] * (k.width - len(r)) for r in k.rows]
        assert p.uses.tolist() == k.uses
        live = [i for i, n in enumerate(k.uses) if n]
        if live:
            assert torch.equal(self.bytes()[:, live], self.first[:, [k.data[i] for i in live]])

    def do(self, what, *args):
        getattr(self.books, what)(*args)
        getattr(self.pages, what)(*(i32(a) for a in args))
        self.check()


@pytest.mark.parametrize("page_size,batch,width,pages", [(32, 1, 1, 1), (32, 3, 4, 9), (64, 7, 20, 100), (256, 5, 3, 16),
                                                         (32, 70, 40, 5000), (64, 1500, 3, 2500)])
def test_long_runs(page_size, batch, width, pages):
    """Lengths that rise, fall and end, forks, compactions, in any order, until pages run out now and then."""
    b = Both(pages, page_size, batch, width, kv=1, D=64, layers=1 if pages > 2000 else 2, seed=batch)
    r = b.rng
    for step in range(40 if batch < 100 else 12):
        what = r.choice(["fit", "fit", "fit", "fork", "compact"])
        if what == "fit":
            most = width * page_size
            few = max(1, pages // batch * page_size)        # (that all can have)
            b.set([r.choice([0, n, n + 1, n + 17, n - 17, page_size, r.randint(0, most), r.randint(0, few)]) % (most + 1)
                   for n in b.books.lens])
            b.do("fit")
            if b.books.missing:
                b.set([min(n, few) for n in b.books.lens])
                b.do("fit")
        elif what == "fork":
            b.do("fork", [r.choice([i, i, r.randrange(batch), -1, batch]) for i in range(batch)])
        else:
            b.do("compact")


def test_growth_past_the_pages_changes_nothing_but_what_shrinks():
    b = Both(10, 32, 3, 8)
    b.set([96, 64, 160])
    b.do("fit")
    assert b.books.missing == 0 and not b.books.free()
    before = b.pages.table.clone()
    b.set([97, 64, 160])
    b.do("fit")
    assert int(b.pages.missing) == 1 and torch.equal(b.pages.table, before)
    b.set([160, 64, 128])                        # one gives a page, another wants two
    b.do("fit")
    assert int(b.pages.missing) == 1 and b.pages.held.tolist() == [3, 2, 4]
    b.set([128, 64, 128])
    b.do("fit")
    assert int(b.pages.missing) == 0


def test_forks_without_pages():
    """No free page for the partial ones: nothing changes; whole pages need none."""
    b = Both(4, 32, 4, 4)
    b.set([40, 64, 0, 0])
    b.do("fit")
    b.do("fork", [0, 1, 0, 1])
    assert int(b.pages.missing) == 1 and b.pages.lens.tolist() == [40, 64, 0, 0]
    b.do("fork", [0, 1, 1, 1])
    assert int(b.pages.missing) == 0 and b.pages.uses.tolist() == [1, 1, 3, 3]


def test_forks_of_lengths_that_were_not_fitted():
    """Lengths that changed since pages were given: a source has the pages that it holds, whole or partial."""
    b = Both(40, 32, 5, 6, seed=8)
    b.set([100, 64, 33, 0, 0])
    b.do("fit")
    b.set([130, 20, 33, 0, 5])                   # more than it holds; fewer; as many; none held
    b.do("fork", [4, 0, 1, 2, 2])
    b.do("fork", [1, 1, 1, 1, 0])
    b.do("fit")


def test_beams_change_places():
    b = Both(64, 32, 4, 6)
    b.set([100, 0, 0, 0])
    b.do("fit")
    b.do("fork", [0, 0, 0, 0])
    b.set([101, 102, 130, 131])
    b.do("fit")
    b.do("fork", [1, 0, 3, 2])
    assert b.pages.lens.tolist() == [102, 101, 131, 130]
    b.do("fork", [3, 3, 3, 3])
    b.set([0, 0, 0, 0])
    b.do("fit")
    assert not b.pages.uses.any() and bool((b.pages.table == -1).all())


@pytest.mark.parametrize("dtype,kv,D,page_size", [(torch.float32, 3, 96, 32), (torch.float8_e4m3fn, 1, 64, 32),
                                                  (torch.float8_e4m3fn, 5, 256, 256), (torch.bfloat16, 8, 128, 128)])
def test_every_cache(dtype, kv, D, page_size):
    """Page sizes that are no whole number of a copy's steps; several layers."""
    b = Both(24, page_size, 5, 4, kv, D, 3, dtype, seed=3)
    n = page_size
    b.set([n + 5, 0, 2 * n, 1, 0])
    b.do("fit")
    b.do("fork", [0, 0, 2, 3, 2])
    b.set([0, n + 6, 0, 5, 2 * n + 1])
    b.do("fit")
    b.do("compact")
    free = b.books.free()[-3:]
    b.cache.copy_pages(i32([0, 1, 2, 99, 0, -1]), i32(free + [3, 24, 4]))
    assert torch.equal(b.bytes()[:, free], b.bytes()[:, :3])
    b.check()


def test_books_that_are_not_consistent_stay_within_their_tensors():
    b = Both(16, 32, 3, 4)
    p = b.pages
    guard = b.cache.storage.clone()
    p.lens.copy_(i32([-5, 10 ** 9, 40]))
    p.held.copy_(i32([99, -7, 3]))
    p.table.copy_(i32([[77, -3, 5, 16], [2 ** 31 - 1] * 4, [1, 2, -2 ** 31, 15]]))
    for call in (p.fit, lambda: p.fork(i32([2, 2, 0])), p.compact, p.fit):
        call()
        torch.cuda.synchronize()
    assert b.cache.storage.shape == guard.shape


def test_a_fork_attends_as_its_source():
    """Sequences with common pages through the cache's own calls: each goes its own way after the fork."""
    b = Both(40, 32, 4, 5, kv=2, D=64, layers=1, seed=9)
    p, c = b.pages, b.cache
    g = torch.Generator().manual_seed(1)
    rnd = lambda *s: torch.randn(*s, generator=g).bfloat16().cuda()  # noqa: E731
    k, v = rnd(70, 2, 64), rnd(70, 2, 64)
    p.lens.copy_(i32([70, 0, 0, 0]))
    p.fit()
    c.append(binding.Chunk(i32([0, 70, 70, 70, 70]), p.lens, p.table, 70, 160), k, v)
    p.fork(i32([0, 0, 0, 0]))
    one = binding.Chunk(i32([0, 1, 2, 3, 4]), p.lens, p.table, 1, 160)
    more = []
    for _ in range(40):
        p.lens.add_(1)
        p.fit()
        x, y, q = rnd(4, 2, 64), rnd(4, 2, 64), rnd(4, 4, 64)
        c.append(one, x, y)
        out = c.attend(one, q)
        more.append((x, y))
    p.compact()
    whole = binding.Chunk(i32([0, 110, 220, 330, 440]), p.lens, p.table, 110, 160)
    gk, gv = c.read(whole, 440)
    for i in range(4):
        wk, wv = torch.cat([k] + [m[0][i:i + 1] for m in more]), torch.cat([v] + [m[1][i:i + 1] for m in more])
        assert same(gk[110 * i:110 * i + 110], wk) and same(gv[110 * i:110 * i + 110], wv)
        alone = binding.Cache(5, 32, 2, 64, torch.bfloat16)
        at = binding.Chunk(i32([0, 110]), i32([110]), i32([[4, 2, 0, 1, 3]]), 110, 160)
        alone.append(at, wk, wv)
        last = binding.Chunk(i32([0, 1]), i32([110]), i32([[4, 2, 0, 1, 3]]), 1, 160)
        # (both sides round their probabilities, 2^-8 of sum p |v| <= max |v| each, and their results, 2^-8 of each)
        assert torch.allclose(alone.attend(last, q[i:i + 1]).float(), out[i:i + 1].float(), rtol=2.0 ** -7,
                              atol=2.0 ** -7 * float(wv.abs().max()))


def test_a_cut_into_a_shared_page():
    """Forked on, a sequence that was cut back into a page of another has that page for itself."""
    b = Both(40, 32, 4, 5, kv=2, D=64, layers=1, seed=10)
    p, c = b.pages, b.cache
    g = torch.Generator().manual_seed(2)
    rnd = lambda *s: torch.randn(*s, generator=g).bfloat16().cuda()  # noqa: E731
    k, v, x, y = rnd(100, 2, 64), rnd(100, 2, 64), rnd(1, 2, 64), rnd(1, 2, 64)
    p.lens.copy_(i32([100, 0, 0, 0]))
    p.fit()
    c.append(binding.Chunk(i32([0, 100, 100, 100, 100]), p.lens, p.table, 100, 160), k, v)
    p.fork(i32([-1, 0, -1, -1]))
    p.lens.copy_(i32([100, 70, 0, 0]))
    p.fit()
    p.fork(i32([-1, -1, 1, -1]))
    p.lens.copy_(i32([100, 70, 71, 0]))
    p.fit()
    c.append(binding.Chunk(i32([0, 0, 0, 1, 1]), p.lens, p.table, 1, 160), x, y)
    table = p.table.tolist()
    assert table[0][:3] == table[1][:3] and table[2][:2] == table[0][:2] and table[2][2] != table[0][2]
    gk, gv = c.read(binding.Chunk(i32([0, 100, 170, 241, 241]), p.lens, p.table, 100, 160), 241)
    for got, old, one in ((gk, k, x), (gv, v, y)):
        assert same(got[:100], old) and same(got[100:170], old[:70]) and same(got[170:], torch.cat([old[:70], one]))


def test_streams_and_graphs():
    """A captured round (lengths grow, pages follow, sequences fork) replayed, between calls on another stream."""
    b = Both(300, 32, 6, 12, seed=4)
    source, step = i32([0, 1, 2, 3, 4, 5]), i32([0] * 6)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        b.pages.lens.add_(step)
        b.pages.fit()
        b.pages.fork(source)
    r = b.rng
    for n in range(6):
        s, t = [r.randrange(6) for _ in range(6)], [r.randrange(40) for _ in range(6)]
        source.copy_(i32(s))
        step.copy_(i32(t))
        graph.replay()
        torch.cuda.synchronize()
        b.books.lens = [x + y for x, y in zip(b.books.lens, t)]
        b.books.fit()
        b.books.fork(s)
        b.check()
        b.books.compact()
        b.pages.compact(stream=side)
        torch.cuda.synchronize()
        b.check()


def test_refusals_of_the_binding():
    b = Both(16, 32, 3, 4)
    for bad in (i32([0, 1]), i32([0, 1, 2]).long(), torch.zeros(3, dtype=torch.int32)):
        with pytest.raises(ValueError):
            b.pages.fork(bad)
    with pytest.raises(ValueError):
        b.cache.copy_pages(i32([0, 1]), i32([2]))
    with pytest.raises(binding.DTError):
        b.cache.copy_pages(i32([]), i32([]))
    with pytest.raises(binding.DTError):
        binding.Pages(b.cache, 0, 4)
