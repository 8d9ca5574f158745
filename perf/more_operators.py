"""Performance cases of what stands around the attention of a decoding round: rotated heads, sampled tokens, pages.

Three families:

* ``rotate`` -- the norm of every query and key head and the rotation by position, in one pass; alone, or with the
                keys and values written into the pages of a cache (and read back as dense rows);
* ``sample`` -- a token for each row of logits with temperature, top-k, top-p and min-p from given random numbers:
                single tokens of a batch, and the root and nodes of its trees;
* ``pages``  -- which pages the sequences of a batch hold: grown and dropped to their lengths, forked (samples of a
                prompt, beams), compacted.  A pass begins with the saved state of the pages copied back.

Sequences are ragged: ``ragged`` is the share of the length by which they differ.
"""
import math
import random

import torch

own = False

DEV = "cuda"
EPS = 1e-6


def _rotate(name=None, batch=1, chunk=1, length=1024, ragged=0.0, heads=32, kv=8, D=128, pairs=0, interleaved=False,
            norm="both", dtype="bf16", append=True, page=64):
    c = dict(family="rotate", batch=batch, chunk=chunk, length=max(length, chunk), ragged=ragged, heads=heads, kv=kv,
             D=D, pairs=pairs or D // 2, interleaved=interleaved, norm=norm, dtype=dtype, append=append, page=page)
    return c if name is None else dict(c, name=name)


def _sample(name=None, rows=1, V=151936, dtype="bf16", T=1.0, top_k=0, top_p=1.0, min_p=0.0, mixed=False, pad=0,
            sharp=1.0):
    c = dict(family="sample", rows=rows, V=V, dtype=dtype, T=T, top_k=top_k, top_p=top_p, min_p=min_p, mixed=mixed,
             pad=pad, sharp=sharp)
    return c if name is None else dict(c, name=name)


def _pages(name=None, op="fit", batch=64, length=4096, ragged=0.5, page=64, pages=0, samples=1, layers=2, kv=8, D=128,
           step=17):
    width = -(-(length + step) // page) + 1
    c = dict(family="pages", op=op, batch=batch, length=length, ragged=ragged, page=page, width=width, samples=samples,
             pages=max(pages, batch * width + batch), layers=layers, kv=kv, D=D, step=step)
    return c if name is None else dict(c, name=name)


def listed():
    return [
        # the smallest call: one token of a toy fp32 model, all latency
        _rotate("rotate_tiny_fp32", heads=4, kv=2, D=64, dtype="f32", append=False, length=37),
        # one decoding step of a serving batch, far into its texts
        _rotate("rotate_tokens_32", batch=32, length=30000, ragged=0.7),
        # verification of a serving batch: the roots and 16 nodes of 32 trees
        _rotate("rotate_verify_32", batch=32, chunk=17, length=4096, ragged=0.5),
        # long prompts, into the pages
        _rotate("rotate_prompts", batch=4, chunk=8192, length=8192, ragged=0.4),
        # part of wide fp32 heads rotated, neighbours as pairs, an odd number of rows, queries alone normed
        _rotate("rotate_partial_fp32", chunk=999, length=20011, heads=16, kv=2, D=256, pairs=32, interleaved=True,
                norm="q", dtype="f32", append=False),
        # the smallest sampling: one row of a small vocabulary
        _sample("sample_one_fp32", V=2003, dtype="f32", T=0.8, top_p=0.9),
        # one decoding step of a serving batch with a common setting
        _sample("sample_tokens_32", rows=32, T=0.6, top_k=20, top_p=0.95),
        # the root and 16 nodes of 32 trees, requests with settings of their own
        _sample("sample_verify_32", rows=544, mixed=True),
        # a high temperature: thousands of tokens are kept, padded fp32 rows
        _sample("sample_flat_fp32", rows=17, dtype="f32", T=1.3, top_p=0.97, min_p=1e-5, pad=61, sharp=0.0),
        # the pages of a serving batch before a round: most grow, some end, some begin
        _pages("pages_fit_64", batch=64, length=8192, pages=16384),
        # 8 prompts become 8 samples each
        _pages("pages_fork_64", op="fork", batch=64, samples=8),
        # half of the sequences are gone: the pages in use move together
        _pages("pages_compact", op="compact", batch=32, length=4000, page=64, pages=2048),
    ]


def _logint(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    family = rng.choice(["rotate", "rotate", "sample", "sample", "sample", "pages", "pages"])
    if family == "rotate":
        D = rng.choice([64, 96, 128, 128, 256])
        kv = rng.choice([1, 2, 4, 8])
        heads = kv * rng.choice([1, 2, 4, 4, 8, 5])
        dtype = rng.choice(["bf16", "bf16", "f32"])
        rows = min(20000, 160000000 // ((heads + kv) * D * (2 if dtype == "bf16" else 4)))
        batch = _logint(rng, 1, 64)
        chunk = _logint(rng, 1, max(2, rows // batch))
        return _rotate(batch=batch, chunk=chunk, length=chunk + _logint(rng, 1, 8192), ragged=rng.choice([0.0, 0.5, 0.9]),
                       heads=heads, kv=kv, D=D, pairs=rng.choice([D // 2, D // 2, D // 2, 16, 8 * rng.randint(1, D // 16)]),
                       interleaved=rng.random() < 0.3, norm=rng.choice(["both", "both", "both", "q", "none"]),
                       dtype=dtype, append=rng.random() < 0.6, page=rng.choice([32, 64, 128]))
    if family == "sample":
        V = rng.choice([151936, 151936, _logint(rng, 100, 151936)])
        dtype = rng.choice(["bf16", "bf16", "f32"])
        rows = _logint(rng, 1, min(2048, 544 * 151936 // V // (1 if dtype == "bf16" else 2)))
        return _sample(rows=rows, V=V, dtype=dtype, T=rng.choice([0.0, 0.3, 0.6, 0.8, 1.0, 1.0, 1.5, 2.0]),
                       top_k=rng.choice([0, 0, 1, 20, 50, _logint(rng, 1, 5000)]),
                       top_p=rng.choice([1.0, 1.0, 0.5, 0.8, 0.9, 0.95, 0.99]), min_p=rng.choice([0.0, 0.0, 0.02, 0.1]),
                       mixed=rng.random() < 0.25, pad=rng.choice([0, 0, 8, 64, 3]), sharp=rng.choice([1.0, 1.0, 0.5, 0.0]))
    op = rng.choice(["fit", "fork", "fork", "compact"])
    page = rng.choice([32, 64, 128])
    samples = rng.choice([1, 2, 4, 8]) if op == "fork" else 1
    batch = samples * _logint(rng, 1, 128 // samples)
    kv, D, layers = rng.choice([2, 4, 8]), rng.choice([64, 128]), rng.choice([1, 2, 3])
    most = 2 ** 30 // (4 * layers * kv * D)      # tokens in the pages
    length = _logint(rng, 20, min(16384, most // batch // 2))
    return _pages(op=op, batch=batch, length=length, ragged=rng.choice([0.0, 0.5, 0.9]), page=page, samples=samples,
                  pages=rng.choice([0, most // page // 2]), layers=layers, kv=kv, D=D, step=rng.choice([1, 17, 65]))


# ---- what a case holds ------------------------------------------------------------

def _dt(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _sizes(c):
    """(length, chunk) of each sequence."""
    out = []
    for i in range(c["batch"]):
        n = c["chunk"] if c["chunk"] <= 32 else max(1, round(c["chunk"] * (1 - c["ragged"] * (i * 0.7548776662 % 1.0))))
        out.append((max(n, round(c["length"] * (1 - c["ragged"] * (i * 0.6180339887 % 1.0)))), n))
    return out


def _rotate_inputs(c, seed):
    """Queries, keys and values as slices of one projection's rows, a few large channels; weights near one."""
    g, dt, D = _gen(seed), _dt(c["dtype"]), c["D"]
    sizes = _sizes(c)
    T, H, kv = sum(n for _, n in sizes), c["heads"], c["kv"]
    chan = 1.0 + 5.0 * (torch.rand(H + 2 * kv, D, generator=g, device=DEV) < 0.03)
    x = (torch.randn(T, H + 2 * kv, D, generator=g, device=DEV) * chan).to(dt)
    s = dict(q=x[:, :H], k=x[:, H:H + kv], v=x[:, H + kv:], T=T, sizes=sizes)
    for n in ("q", "k"):
        on = c["norm"] == "both" or c["norm"] == n
        s[n + "_weight"] = (1 + 0.3 * torch.randn(D, generator=g, device=DEV)).to(dt) if on else None
    j = torch.arange(c["pairs"], device=DEV, dtype=torch.float64)
    s["inv_freq"] = (1e6 ** (-j / c["pairs"])).float()
    jump = random.Random(seed).randrange(1, 9)    # (a tree's nodes share depths; positions need not rise)
    s["positions"] = _i32([p - (i % jump if n <= 32 else 0) for ln, n in sizes for i, p in enumerate(range(ln - n, ln))])
    if c["append"]:
        width = max(-(-ln // c["page"]) for ln, _ in sizes)
        pages = c["batch"] * width + 3
        order = torch.randperm(pages, generator=g, device=DEV)[:c["batch"] * width]
        starts = [0]
        for _, n in sizes:
            starts.append(starts[-1] + n)
        s.update(pages=pages, table=order.reshape(c["batch"], width).int(), starts=_i32(starts),
                 lens=_i32([ln for ln, _ in sizes]), max_chunk=max(n for _, n in sizes),
                 max_len=max(ln for ln, _ in sizes))
    return s


def _sample_inputs(c, seed):
    """Logits of a language model: a wide bulk and, where a row is sure of something, a few high ones; random
    numbers; settings of each row where requests differ."""
    g, rng, R, V = _gen(seed), random.Random(seed), c["rows"], c["V"]
    x = torch.randn(R, V + c["pad"], generator=g, device=DEV) * 2.2
    n = min(V, 40)
    top = torch.randint(0, V, (R, n), generator=g, device=DEV)
    step = 0.2 + 1.5 * torch.rand(R, 1, generator=g, device=DEV)
    high = 16 - step * torch.arange(n, device=DEV) + 0.3 * torch.randn(R, n, generator=g, device=DEV)
    sure = torch.rand(R, 1, generator=g, device=DEV) < c["sharp"]
    high = torch.where(sure, high, x.gather(1, top))
    x.scatter_(1, top, high)
    s = dict(logits=x.to(_dt(c["dtype"]))[:, :V], u=torch.rand(R, generator=g, device=DEV), T=c["T"], top_k=c["top_k"],
             top_p=c["top_p"], min_p=c["min_p"])
    if c["mixed"]:   # (requests of 17 rows each)
        of = [rng.choice([(0.6, 20, 0.95, 0.0), (1.0, 0, 1.0, 0.0), (0.8, 0, 0.9, 0.0), (0.0, 0, 1.0, 0.0),
                          (1.0, 50, 1.0, 0.0), (1.2, 0, 1.0, 0.05), (0.7, 200, 0.8, 0.01)]) for _ in range(R // 17 + 1)]
        rows = [of[r // 17] for r in range(R)]
        for i, n in enumerate(("T", "top_k", "top_p", "min_p")):
            s[n] = torch.tensor([o[i] for o in rows], dtype=torch.int32 if n == "top_k" else torch.float32, device=DEV)
    return s


def _lengths(c, rng):
    return [max(1, round(c["length"] * (1 - c["ragged"] * rng.random()))) for _ in range(c["batch"])]


def _pages_inputs(c, seed):
    """The state of the pages before the call, as Pages.state holds it: pages missing, uses of every page, pages held
    and tokens of every sequence, the table; the cache's bytes; each sequence's source where they fork."""
    g, rng = _gen(seed), random.Random(seed * 31 + 7)
    b, page, width, P = c["batch"], c["page"], c["width"], c["pages"]
    lens = _lengths(c, rng)
    order = list(range(P))
    rng.shuffle(order)                       # (as after a long run)
    uses, rows, at = [0] * P, [], 0
    for n in lens:
        row = order[at:at + -(-n // page)]
        at += len(row)
        rows.append(row)
    source = list(range(b))
    if c["op"] == "fit":
        for i in range(b):
            what = rng.random()
            if what < 0.1:                   # ends
                lens[i] = 0
            elif what < 0.2:                 # begins
                rows[i] = []
            elif what < 0.8:                 # a root and its nodes
                lens[i] += c["step"]
            else:                            # nodes that were not accepted
                lens[i] = max(1, lens[i] - c["step"])
    elif c["op"] == "fork":
        beams = c["samples"] > 1 and c["batch"] // c["samples"] == 1
        for i in range(b):
            first = i - i % c["samples"]
            if beams and i > first:          # (common first half, then each its own)
                half = len(rows[first]) // 2
                rows[i] = rows[first][:half] + rows[i][:max(0, len(rows[first]) - half)]
                lens[i] = min(lens[first], len(rows[i]) * page)
            elif i > first:
                rows[i], lens[i] = [], 0
            source[i] = rng.randrange(b) if beams else first
            if c["samples"] == 1 and rng.random() < 0.5:
                source[i] = rng.randrange(b)
    else:
        for i in range(b):
            if rng.random() < 0.5:
                rows[i], lens[i] = [], 0
    for row in rows:
        for p in row:
            uses[p] += 1
    table = [row + [-1] * (width - len(row)) for row in rows]
    state = _i32([0] + uses + [len(r) for r in rows] + lens + [p for row in table for p in row])
    n = c["layers"] * P * c["kv"] * page * c["D"]   # words: keys and values of two bytes each
    return dict(state=state, source=_i32(source),
                data=torch.randint(-2 ** 31, 2 ** 31 - 1, (n,), generator=g, device=DEV, dtype=torch.int32))


# ---- the plain form: 32 bits (64 for angles, sums and borders), elementary operations --------------------------

def _plain_heads(c, x, w, cos, sin):
    x = x.float()
    if w is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w.float()
    P = c["pairs"]
    a, b = (x[..., 0:2 * P:2], x[..., 1:2 * P:2]) if c["interleaved"] else (x[..., :P], x[..., P:2 * P])
    y, z = a * cos - b * sin, b * cos + a * sin
    y = torch.stack([y, z], -1).flatten(-2) if c["interleaved"] else torch.cat([y, z], -1)
    return torch.cat([y, x[..., 2 * P:]], -1).to(_dt(c["dtype"]))


def _plain_rotate(c, s):
    angle = s["positions"].double()[:, None] * s["inv_freq"].double()
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    q = _plain_heads(c, s["q"], s["q_weight"], cos, sin)
    k = _plain_heads(c, s["k"], s["k_weight"], cos, sin)
    if not c["append"]:
        return dict(q=q, k=k)
    row = torch.arange(s["T"], device=DEV, dtype=torch.int32)
    seq = torch.bucketize(row, s["starts"][1:], right=True)
    pos = s["lens"][seq] - s["starts"][seq + 1] + row
    at = s["table"][seq, pos // c["page"]].long(), (pos % c["page"]).long()
    s["cache"][0][at] = k
    s["cache"][1][at] = s["v"]
    return dict(q=q, k=s["cache"][0][at], v=s["cache"][1][at])


def _column(x):
    """A setting as a column of 64-bit values, for all rows or of each."""
    if isinstance(x, torch.Tensor):
        return x.double()[:, None]
    return torch.tensor([[x]], dtype=torch.float32, device=DEV).double()


def _plain_sample(c, s):
    x = s["logits"].float()
    T, k, p, q = (_column(s[n]) for n in ("T", "top_k", "top_p", "min_p"))
    y, ids = torch.sort(x, dim=1, descending=True, stable=True)
    m = y[:, :1].double()
    w = torch.exp((y.double() - m) / torch.where(T > 0, T, torch.ones_like(T)))
    w = torch.where(T > 0, w, (torch.arange(c["V"], device=DEV) == 0).double())       # (greedy)
    rank = torch.arange(c["V"], device=DEV)
    keep = ((rank < k) | (k <= 0)).expand(w.shape)
    w = torch.where(keep, w, torch.zeros_like(w))
    before = torch.cumsum(w, 1) - w
    keep = keep & ((before < p * w.sum(1, keepdim=True)) | (p >= 1) | (rank == 0)) & (w >= q)
    w = torch.where(keep, w, torch.zeros_like(w))
    del before, keep, y
    w = torch.zeros_like(w).scatter_(1, ids, w)
    run = torch.cumsum(w, 1)
    z = run[:, -1:]
    hit = (run > s["u"].double()[:, None] * z) & (w > 0)
    token = hit.int().argmax(1)
    return dict(tokens=token.int(), logprobs=torch.log(w.gather(1, token[:, None]) / z)[:, 0].float())


def _parts(c, state):
    P, b = c["pages"], c["batch"]
    return (state[:1], state[1:1 + P], state[1 + P:1 + P + b], state[1 + P + b:1 + P + 2 * b],
            state[1 + P + 2 * b:].view(b, c["width"]))


def _count(c, pages, on, sign, uses):
    """Add or take a use of the pages of a table's entries where `on`."""
    at = torch.where(on, pages, torch.full_like(pages, c["pages"])).flatten().long()
    add = torch.zeros(c["pages"] + 1, dtype=torch.int32, device=DEV)
    add.index_add_(0, at, torch.full_like(at, sign, dtype=torch.int32))
    uses += add[:-1]


def _copy_pages(data, frm, to, on):
    """Pages `to` of every layer from pages `frm` where `on`; the other places repeat the first such copy."""
    first = on.int().argmax()
    some = on.any()
    frm, to = (torch.where(on, x, torch.where(some, x[first], torch.zeros_like(first))) for x in (frm, to))
    data[:, to] = data[:, frm]


def _plain_pages(c, s):
    state, page, width, P = s["book"], c["page"], c["width"], c["pages"]
    state.copy_(s["state"])
    missing, uses, held, lens, table = _parts(c, state)
    col = torch.arange(width, device=DEV, dtype=torch.int32)
    data = s["cache"].view(c["layers"], P, -1)
    if c["op"] == "fit":
        want = (lens + page - 1) // page
        _count(c, table, (col >= want[:, None]) & (col < held[:, None]), -1, uses)
        table.masked_fill_(col >= want[:, None], -1)
        kept = torch.minimum(held, want)
        grow = want - kept
        first = torch.cumsum(grow, 0) - grow
        free = torch.sort(uses > 0, stable=True).indices.int()
        short = (grow.sum() - (uses == 0).sum()).clamp(min=0).int()
        new = (col >= kept[:, None]) & (col < want[:, None]) & (short == 0)
        take = free[(first[:, None] + col - kept[:, None]).clamp(0, P - 1).long()]
        table.copy_(torch.where(new, take, table))
        _count(c, table, new, 1, uses)
        held.copy_(torch.where(short == 0, want, kept))
        missing.copy_(short.view(1))
        return dict(state=state)
    if c["op"] == "fork":
        src = s["source"].long()
        moves = src != torch.arange(len(src), device=DEV)
        ln = lens[src]
        full, part = ln // page, (ln % page > 0) & moves
        free = torch.sort(uses > 0, stable=True).indices
        to = free[(torch.cumsum(part.int(), 0) - 1).clamp(min=0)]
        short = (part.sum() - (uses == 0).sum()).clamp(min=0).int()
        moves &= short == 0
        part &= short == 0
        old = table.clone()
        rows = old[src]
        frm = rows.gather(1, full.clamp(max=width - 1).long()[:, None])[:, 0].long()
        _copy_pages(data, frm, to, part)
        new = torch.where(col < full[:, None], rows, torch.full_like(rows, -1))
        new = torch.where((col == full[:, None]) & part[:, None], to[:, None].int(), new)
        _count(c, old, moves[:, None] & (col < held[:, None]), -1, uses)
        _count(c, new, moves[:, None] & (new >= 0), 1, uses)
        table.copy_(torch.where(moves[:, None], new, old))
        held.copy_(torch.where(moves, full + part.int(), held))
        lens.copy_(torch.where(moves, ln, lens))
        missing.copy_(short.view(1))
        return dict(state=state, data=s["cache"])
    live = uses > 0
    n = live.sum()
    index = torch.arange(P, device=DEV)
    high, hole = live & (index >= n), ~live & (index < n)
    frm = torch.sort(~high, stable=True).indices        # the pages that move, in order, then the others
    to = torch.sort(~hole, stable=True).indices
    on = index < high.sum()
    _copy_pages(data, frm, to, on)
    where = index.clone()                                # (page 0 never moves)
    where.scatter_(0, torch.where(on, frm, index[:1]), torch.where(on, to, index[:1]))
    moved = torch.zeros_like(uses).index_add_(0, where, torch.where(live, uses, torch.zeros_like(uses)))
    uses.copy_(moved)
    table.copy_(torch.where(table >= 0, where[table.clamp(min=0).long()].int(), table))
    missing.zero_()
    return dict(state=state, data=s["cache"])


# ---- the interface ------------------------------------------------------------------

def prepare(case, seed):
    c = case
    if c["family"] == "sample":
        return dict(_sample_inputs(c, seed), case=c, own=own)
    if c["family"] == "rotate":
        s = dict(_rotate_inputs(c, seed), case=c, own=own)
        if c["append"] and own:
            from paper_2607_08642_amd import binding
            s["cache"] = binding.Cache(s["pages"], c["page"], c["kv"], c["D"], _dt(c["dtype"]), device=DEV)
            s["chunk"] = binding.Chunk(s["starts"], s["lens"], s["table"], s["max_chunk"], s["max_len"])
        elif c["append"]:
            s["cache"] = torch.zeros(2, s["pages"], c["page"], c["kv"], c["D"], dtype=_dt(c["dtype"]), device=DEV)
        return s
    s = dict(_pages_inputs(c, seed), case=c, own=own)
    if own:
        from paper_2607_08642_amd import binding
        s["cache"] = binding.Cache(c["pages"], c["page"], c["kv"], c["D"], torch.bfloat16, layers=c["layers"], device=DEV)
        s["book"] = binding.Pages(s["cache"], c["batch"], c["width"])
        s["cache"].storage.view(torch.int32).copy_(s.pop("data"))
    else:
        s["book"], s["cache"] = s["state"].clone(), s.pop("data")
    return s


def run(state):
    s, c = state, state["case"]
    if s["own"]:
        if c["family"] == "sample":
            from paper_2607_08642_amd import binding
            tokens, logprobs = binding.sample(s["logits"], s["u"], s["T"], s["top_k"], s["top_p"], s["min_p"],
                                              logprobs=True)
            return dict(tokens=tokens, logprobs=logprobs)
        if c["family"] == "rotate":
            how = dict(q_weight=s["q_weight"], k_weight=s["k_weight"], eps=EPS, interleaved=c["interleaved"])
            if c["append"]:
                q = s["cache"].append_rotated(s["chunk"], s["q"], s["k"], s["v"], s["positions"], s["inv_freq"], **how)
                k, v = s["cache"].read(s["chunk"], s["T"])
                return dict(q=q, k=k, v=v)
            from paper_2607_08642_amd import binding
            q, k = binding.rotate(s["q"], s["k"], s["positions"], s["inv_freq"], **how)
            return dict(q=q, k=k)
        book = s["book"]
        book.state.copy_(s["state"])
        if c["op"] == "fit":
            book.fit()
            return dict(state=book.state)
        if c["op"] == "fork":
            book.fork(s["source"])
        else:
            book.compact()
        return dict(state=book.state, data=s["cache"].storage.view(torch.int32))
    plain = {"sample": _plain_sample, "rotate": _plain_rotate, "pages": _plain_pages}
    return plain[c["family"]](c, s)


def work(case):
    c = case
    if c["family"] == "sample":
        n = c["rows"] * c["V"]     # a comparison, an exponential and a sum for each logit, a running sum
        return dict(bytes=n * (2 if c["dtype"] == "bf16" else 4) + c["rows"] * 28, flops=4.0 * n)
    if c["family"] == "rotate":
        T, es = sum(n for _, n in _sizes(c)), 2 if c["dtype"] == "bf16" else 4
        q, k = T * c["heads"] * c["D"] * es, T * c["kv"] * c["D"] * es
        flops = T * (c["heads"] + c["kv"]) * (4.0 * c["D"] + 6.0 * c["pairs"]) + 4.0 * T * c["pairs"]
        # q and k in and out; with the cache k and v in, into the pages, out of them, out
        return dict(bytes=2 * q + (8 * k if c["append"] else 2 * k) + 4 * T, flops=flops)
    # the state copied, its uses and lengths read; pages of all layers copied: half of the partial ones of a fork, or
    # those of the live ones that are not among the first
    book = 4 * (1 + c["pages"] + c["batch"] * (2 + c["width"]))
    row = c["layers"] * c["kv"] * c["D"] * 4 * c["page"]
    tokens = c["batch"] * c["length"] * (1 - c["ragged"] / 2)
    moved = 0.0
    if c["op"] == "fork":
        moved = c["batch"] * (1 - 1 / c["samples"] if c["samples"] > 1 else 0.5) * (1 - 1 / c["page"])
    elif c["op"] == "compact":
        live = tokens / 2 / c["page"]
        moved = live * (1 - live / c["pages"])
    return dict(bytes=2 * book + 4 * (c["pages"] + 3 * c["batch"]) + 2 * moved * row, flops=2.0 * c["pages"])


# ---- the definition in 64 bits ---------------------------------------------------------

def _exact_rotate(c, seed):
    s = _rotate_inputs(c, seed)
    P, D = c["pairs"], c["D"]
    out = {}
    first = torch.arange(P, device=DEV) * (2 if c["interleaved"] else 1)
    second = first + (1 if c["interleaved"] else P)
    turn = torch.remainder(s["positions"].double()[:, None] * s["inv_freq"].double()[None], 2 * math.pi)
    e = torch.polar(torch.ones_like(turn), turn)
    for n in ("q", "k"):
        y = s[n].double().clone()
        if s[n + "_weight"] is not None:
            y = y / torch.sqrt(y.square().sum(-1, keepdim=True) / D + EPS) * s[n + "_weight"].double()
        z = torch.complex(y[..., first], y[..., second]) * e[:, None]
        y[..., first], y[..., second] = z.real, z.imag
        out[n] = y
    if c["append"]:
        out["v"] = s["v"].double()
    return out


def _exact_sample(c, seed):
    s = _sample_inputs(c, seed)
    x, out = s["logits"].double(), []
    setting = {n: (s[n].tolist() if isinstance(s[n], torch.Tensor) else
                   [torch.tensor(s[n], dtype=torch.float32).item()] * c["rows"]) for n in ("T", "top_k", "top_p", "min_p")}
    for r in range(c["rows"]):
        T, k, p, q = (setting[n][r] for n in ("T", "top_k", "top_p", "min_p"))
        if T == 0:
            out.append(torch.zeros((), dtype=torch.float64, device=DEV))
            continue
        order = torch.argsort(x[r], descending=True, stable=True)
        prob = torch.softmax(x[r][order][:int(k) if k > 0 else None] / T, 0)
        if p < 1:
            prob = prob[:max(1, int(torch.searchsorted(torch.cumsum(prob, 0), p).item()) + 1)]
        prob = prob[prob >= q * prob[0]]
        ids, at = torch.sort(order[:len(prob)])
        run = torch.cumsum(prob[at], 0)
        i = min(int(torch.searchsorted(run, s["u"][r].double() * run[-1], right=True)), len(run) - 1)
        out.append(torch.log(prob[at][i] / prob.sum()))
    return dict(tokens=None, logprobs=torch.stack(out))


def exact(case, seed):
    c = case
    if c["family"] == "rotate":
        return _exact_rotate(c, seed)
    if c["family"] == "sample" and c["rows"] <= 1024:
        return _exact_sample(c, seed)
    return None
