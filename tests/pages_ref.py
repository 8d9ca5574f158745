"""The pages of sequences as plain Python lists, written from their definitions, for the tests."""


class Books:
    """rows: the pages of every sequence; lens; uses.  data: what each page holds (any value)."""

    def __init__(self, pages, page_size, batch, width):
        self.pages, self.page_size, self.width = pages, page_size, width
        self.rows, self.lens = [[] for _ in range(batch)], [0] * batch
        self.data = list(range(pages))
        self.missing = 0

    @property
    def uses(self):
        n = [0] * self.pages
        for row in self.rows:
            for p in row:
                n[p] += 1
        return n

    def free(self):
        return [p for p, n in enumerate(self.uses) if n == 0]

    def fit(self):
        want = [-(-n // self.page_size) for n in self.lens]
        self.rows = [row[:w] for row, w in zip(self.rows, want)]
        free = self.free()
        lacks = sum(w - len(row) for row, w in zip(self.rows, want))
        self.missing = max(0, lacks - len(free))
        if not self.missing:
            for row, w in zip(self.rows, want):
                while len(row) < w:
                    row.append(free.pop(0))

    def fork(self, source):
        moves = [(b, s) for b, s in enumerate(source) if 0 <= s < len(source) and s != b]
        free = self.free()
        parts = [b for b, s in moves if self.lens[s] % self.page_size and len(self.rows[s]) * self.page_size >= self.lens[s]]
        self.missing = max(0, len(parts) - len(free))
        if self.missing:
            return
        new = {}
        for b, s in moves:
            full = self.lens[s] // self.page_size
            row = self.rows[s][:full]
            if b in parts:
                p = free.pop(0)
                self.data[p] = self.data[self.rows[s][full]]
                row.append(p)
            new[b] = row, self.lens[s]
        for b, (row, n) in new.items():
            self.rows[b], self.lens[b] = row, n

    def compact(self):
        uses = self.uses
        n = sum(u > 0 for u in uses)
        to = dict(zip([p for p in range(n, self.pages) if uses[p]], [p for p in range(n) if not uses[p]]))
        for p, q in to.items():
            self.data[q] = self.data[p]
        self.rows = [[to.get(p, p) for p in row] for row in self.rows]
        self.missing = 0
