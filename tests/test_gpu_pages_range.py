"""Books that are not consistent: no call writes outside the tensors that it is given, whatever they hold.

Every tensor (books, source, lists, workspace, cache) lies between guards of a known value within one allocation, and the
calls' own inputs (source, lists) have to stay as they are too."""
import ctypes
import random

import pytest
import torch

from paper_2607_08642_amd import binding

pytestmark = pytest.mark.gpu
GUARD = 1 << 16                                   # bytes before and after each tensor
FILL = 0x5a
WORST = [-2 ** 31, -2 ** 31 + 1, -77, -2, -1, 2 ** 30, 2 ** 31 - 2, 2 ** 31 - 1]


class Fenced:
    """Tensors of so many bytes each, guards around them."""

    def __init__(self, sizes):
        self.at, n = {}, GUARD
        for name, size in sizes.items():
            self.at[name] = n, size
            n += -(-size // 256) * 256 + GUARD
        self.all = torch.full((n,), FILL, dtype=torch.uint8, device="cuda")
        assert self.all.data_ptr() % 256 == 0

    def __getitem__(self, name):
        at, size = self.at[name]
        return self.all[at:at + size]

    def ints(self, name):
        return self[name].view(torch.int32)

    def whole(self):
        """Whether every guard is as it was made."""
        end = 0
        for at, size in self.at.values():
            if not bool((self.all[end:at] == FILL).all()):
                return False
            end = at + size
        return bool((self.all[end:] == FILL).all())


@pytest.mark.parametrize("dtype", [binding.DT_F32, binding.DT_BF16, binding.DT_F8])
@pytest.mark.parametrize("pages,page_size,batch,width", [(1, 32, 1, 1), (16, 32, 3, 4), (5, 64, 40, 3), (300, 32, 7, 33),
                                                         (5000, 32, 1100, 2)])
def test_nothing_outside_is_written(dtype, pages, page_size, batch, width):
    lib, n = binding.load(), ctypes.c_size_t()
    cache = binding.dt_cache(None, 2, pages, page_size, 1, 64, dtype)
    assert lib.dt_cache_size(ctypes.byref(cache), ctypes.byref(n)) == 0
    storage = n.value
    books = binding.dt_pages(pages, page_size, batch, width)
    assert lib.dt_pages_workspace_size(ctypes.byref(books), ctypes.byref(n)) == 0
    space, copies = n.value, 9
    f = Fenced(dict(uses=4 * pages, held=4 * batch, lens=4 * batch, table=4 * batch * width, missing=4, source=4 * batch,
                    froms=4 * copies, tos=4 * copies, workspace=space, cache=storage))
    cache.data = f["cache"].data_ptr()
    for name in ("uses", "held", "lens", "table", "missing"):
        setattr(books, name, f[name].data_ptr())
    at = {name: f[name].data_ptr() for name in f.at}
    b, c = ctypes.byref(books), ctypes.byref(cache)
    calls = [lambda: lib.dt_pages_fit(b, at["workspace"], space, None),
             lambda: lib.dt_pages_fork(b, c, at["source"], at["workspace"], space, None),
             lambda: lib.dt_pages_compact(b, c, at["workspace"], space, None),
             lambda: lib.dt_cache_copy_pages(c, at["froms"], at["tos"], copies, None)]
    rng, g = random.Random(pages), torch.Generator(device="cuda")
    g.manual_seed(pages)

    def some(n, likely, k):
        """n numbers, of which about one in k is one that no call can use."""
        return torch.tensor([rng.choice(WORST) if rng.random() * k < 1 else rng.randint(*likely) for _ in range(n)],
                            dtype=torch.int32)

    for trial in range(8):
        k = (1, 2, 10)[trial % 3]
        f.ints("uses").copy_(some(pages, (-1, 2), k))
        f.ints("held").copy_(some(batch, (-1, width + 1), k))
        f.ints("lens").copy_(some(batch, (-1, (width + 1) * page_size), k))
        f.ints("table").copy_(some(batch * width, (-1, pages), k))
        f.ints("source").copy_(some(batch, (-1, batch), k))
        f.ints("froms").copy_(some(copies, (-1, pages), k))
        # (no page may be written twice, or written and read: pages that the other list does not hold)
        free = [p for p in range(pages) if p not in f.ints("froms").tolist()]
        to = [rng.choice(WORST + [pages]) for _ in range(copies)]
        for i, p in zip(rng.sample(range(copies), min(copies, len(free)) // 2), rng.sample(free, min(copies, len(free)) // 2)):
            to[i] = p
        f.ints("tos").copy_(torch.tensor(to, dtype=torch.int32))
        f["workspace"].random_(generator=g)                  # (and what a workspace held before means nothing)
        f["cache"].random_(generator=g)
        given = [f.ints(x).clone() for x in ("source", "froms", "tos")]
        for i in rng.sample(range(4), 4) + [0]:
            assert calls[i]() == 0
            torch.cuda.synchronize()
            assert f.whole(), (trial, i)
            assert all(torch.equal(f.ints(x), g) for x, g in zip(("source", "froms", "tos"), given))
