"""Performance cases of the verification side: the paged cache, the attention that reads it, and the commit of a tree.

A drafted tree is verified by the target model: the keys and values of its nodes are written into the cache, the nodes
attend to the cached context under the tree's ancestor mask, the longest accepted path is taken and its rows kept.
Three families:

* ``store``  -- new tokens' keys and values into pages (as they are, or in 8 bits with a power-of-two scale for each
                token and head) and back out as dense rows;
* ``attend`` -- attention of a chunk of new tokens of each sequence over the pages: single tokens, chunks of a prompt,
                trees; with or without a sliding window and first tokens that stay visible;
* ``commit`` -- the end of a round: a tree's rows written, the accepted path found, its rows moved together, read back.

Sequences are ragged: ``ragged`` is the share of the length (and of the chunk) by which they differ.  The last
``chunk`` tokens of a sequence of ``length`` are the new ones; with ``tree`` nodes the chunk is the root (the last
committed token) and the nodes.  Keys carry a few large channels and queries are spread so that the softmax is neither
flat nor a single key, as in trained models.
"""
import math
import random

import torch

own = False

DEV = "cuda"
DEPTH = 16   # levels of a drafted tree at most (the benchmark's block length)


def _case(name=None, family="attend", batch=1, heads=32, kv=8, D=128, page=64, dtype="bf16", cache="bf16", chunk=1,
          length=1024, ragged=0.0, window=0, sinks=0, tree=0, layers=1):
    c = dict(family=family, batch=batch, heads=heads, kv=kv, D=D, page=page, dtype=dtype, cache=cache,
             chunk=1 + tree if tree else chunk, length=length, ragged=ragged, window=window, sinks=sinks, tree=tree,
             layers=layers)
    return c if name is None else dict(c, name=name)


def listed():
    return [
        # the smallest call: one token of a toy fp32 model, all latency
        _case("token_tiny_fp32", heads=4, kv=2, D=64, page=32, dtype="f32", cache="f32", length=37),
        # plain decoding of a serving batch, ragged lengths
        _case("tokens_32", batch=32, length=8192, ragged=0.7),
        # verification of a serving batch: 32 trees of 16 nodes (the benchmark's concurrent workload)
        _case("verify_32", batch=32, length=4096, ragged=0.5, tree=16),
        # verification of one large tree (budget 64) far into a long text, 8-bit cache: few rows, one long axis
        _case("verify_64_fp8", cache="fp8", page=128, length=30011, tree=64),
        # a prompt's chunk in the middle of a long prompt: the largest, bound by the matrix units
        _case("chunk_4096", chunk=4096, length=16384),
        # a mixed batch of an fp8 cache: chunks of 31 to 509 tokens, heads of 64, one kv head for 8
        _case("chunks_ragged_fp8", batch=8, heads=16, kv=2, D=64, page=32, cache="fp8", chunk=509, length=3001,
              ragged=0.94),
        # decoding with a sliding window and 4 first tokens kept, contexts much longer than the window
        _case("window_tokens", batch=64, heads=16, kv=4, length=20000, ragged=0.5, window=1024, sinks=4),
        # a prompt's chunk under a window
        _case("window_chunk", chunk=2047, heads=16, kv=4, D=64, page=128, length=9001, window=777, sinks=16),
        # what one decoding step of a serving batch writes, and back, in 8 bits
        _case("store_tokens_fp8", family="store", batch=32, cache="fp8", length=4096, ragged=0.9),
        # long prompts written in 8 bits and read back
        _case("store_prompts_fp8", family="store", batch=4, cache="fp8", chunk=16384, length=16384, ragged=0.4),
        # the end of a round for 32 trees, two layers
        _case("commit_32", family="commit", batch=32, length=2048, ragged=0.5, tree=16, layers=2),
        # the same for one large tree of a small fp32 model
        _case("commit_64_fp32", family="commit", heads=8, kv=2, D=96, page=32, dtype="f32", cache="f32", length=777,
              tree=64),
    ]


def _logint(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    cache = "f32" if dtype == "f32" else rng.choice(["bf16", "fp8"])
    D = rng.choice([64, 96, 128, 128, 256])
    kv = rng.choice([1, 2, 4, 8])
    group = rng.choice([1, 2, 4, 4, 8, 5])
    c = dict(heads=kv * group, kv=kv, D=D, page=rng.choice([32, 64, 128]), dtype=dtype, cache=cache,
             ragged=rng.choice([0.0, 0.3, 0.6, 0.9]))
    kind = rng.choice(["token", "token", "verify", "verify", "chunk", "chunk", "store", "store", "commit"])
    batch = _logint(rng, 1, 64)
    keys = int(2 ** 18 * 1024 / (kv * D) / (2 if dtype == "f32" else 1))   # cached tokens of all sequences at most
    if kind == "token":
        c.update(batch=batch, length=_logint(rng, 16, max(17, min(65536, keys // batch))))
    elif kind == "verify":
        tree = rng.choice([8, 16, 16, 32, 64, rng.randint(4, 64)])
        c.update(batch=batch, tree=tree, length=_logint(rng, tree + 2, max(tree + 3, min(32768, keys // batch))))
    elif kind == "chunk":
        batch = _logint(rng, 1, 8)
        n = _logint(rng, 2, 4096 // batch)
        pairs = 2 ** 31 // (4 if dtype == "bf16" else 16)   # (head, row, key) at most
        most = pairs // (batch * n * kv * group * max(1, D // 128))
        c.update(batch=batch, chunk=n, length=n + _logint(rng, 1, max(2, min(16384, most))))
    elif kind == "store":
        n = rng.choice([1, _logint(rng, 1, max(2, min(16384, keys // batch // 4)))])
        return _case(family="store", batch=batch, chunk=n, length=n + _logint(rng, 1, 4096), **c)
    else:
        return _case(family="commit", batch=batch, tree=rng.randint(4, 64), layers=rng.choice([1, 2, 4]),
                     length=_logint(rng, 80, 2048), **c)
    if rng.random() < 0.35:
        c.update(window=_logint(rng, 16, max(17, min(2048, c["length"]))), sinks=rng.choice([0, 1, 4, 16, 64]))
    return _case(**c)


# ---- what a case holds ------------------------------------------------------------

def _sizes(c):
    """(length, chunk) of each sequence."""
    out = []
    for i in range(c["batch"]):
        n = c["chunk"] if c["tree"] else max(1, round(c["chunk"] * (1 - c["ragged"] * (i * 0.7548776662 % 1.0))))
        out.append((max(n, round(c["length"] * (1 - c["ragged"] * (i * 0.6180339887 % 1.0)))), n))
    return out


def _dt(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _trees(c, seed):
    """Trees as the builder emits them (parents first, siblings of distinct tokens), and the target's token at the
    root and at every node: the drafted child's four times out of five."""
    rng = random.Random(seed * 7919 + 17)
    b, N = c["batch"], c["tree"]
    tokens, parents, depth, target = [], [], [], []
    for _ in range(b):
        par, dep = [], []
        for i in range(N):
            while True:
                p = rng.choice([-1, i - 1, rng.randrange(i)] if i else [-1])
                if p < 0 or dep[p] < DEPTH:
                    break
            par.append(p)
            dep.append(1 if p < 0 else dep[p] + 1)
        tok = [3 + 7 * i + rng.randrange(7) for i in range(N)]
        tgt = []
        for at in range(-1, N):
            kids = [i for i in range(N) if par[i] == at]
            tgt.append(tok[rng.choice(kids)] if kids and rng.random() < 0.8 else 1)
        tokens.append(tok)
        parents.append(par)
        depth.append(dep)
        target.append(tgt)
    mask = torch.zeros(b, N, N, dtype=torch.uint8)
    for t in range(b):
        for i in range(N):
            if parents[t][i] >= 0:
                mask[t, i] = mask[t, parents[t][i]]
            mask[t, i, i] = 1
    return dict(tokens=_i32(tokens), parents=_i32(parents), depth=_i32(depth), mask=mask.to(DEV),
                n_nodes=_i32([N] * b), target=_i32(target))


def _inputs(c, seed):
    """Keys and values of the tokens to store (``attend``: of whole sequences), queries, pages' order."""
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    sizes = _sizes(c)
    whole = c["family"] == "attend"
    T = sum(n if whole else m for n, m in sizes)
    dt, kv, D = _dt(c["dtype"]), c["kv"], c["D"]
    chan = 1.0 + 3.0 * (torch.rand(kv, D, generator=g, device=DEV) < 0.03)
    x = dict(sizes=sizes, k=[], v=[])
    for _ in range(c["layers"]):
        x["k"].append((torch.randn(T, kv, D, generator=g, device=DEV) * chan).to(dt))
        x["v"].append(torch.randn(T, kv, D, generator=g, device=DEV).to(dt))
    if whole:
        x["q"] = (torch.randn(sum(m for _, m in sizes), c["heads"], D, generator=g, device=DEV) * 1.5).to(dt)
    width = max(-(-n // c["page"]) for n, _ in sizes)
    pages = c["batch"] * width + 3
    order = torch.randperm(pages, generator=g, device=DEV)[:c["batch"] * width]
    x.update(width=width, pages=pages, table=order.reshape(c["batch"], width).to(torch.int32))
    if c["tree"]:
        x.update(_trees(c, seed))
    return x


def _starts(counts):
    s = [0]
    for n in counts:
        s.append(s[-1] + n)
    return _i32(s)


# ---- the plain form: 32 bits, elementary operations ----------------------------------

def _plain_cache(c, pages):
    shape = (pages, c["page"], c["kv"], c["D"])
    layer = {}
    for n in ("k", "v"):
        layer[n] = torch.zeros(shape, device=DEV, dtype=torch.float8_e4m3fn if c["cache"] == "fp8" else _dt(c["cache"]))
        layer[n + "e"] = torch.zeros(shape[:3], device=DEV, dtype=torch.int32) if c["cache"] == "fp8" else None
    return layer


def _where(starts, lens, table, page, T):
    """Page and slot of each of the chunks' T rows."""
    row = torch.arange(T, device=DEV, dtype=torch.int32)
    seq = torch.bucketize(row, starts[1:], right=True)
    pos = lens[seq] - starts[seq + 1] + row
    return table[seq, pos // page].long(), (pos % page).long()


def _plain_append(layer, at, k, v):
    for n, x in (("k", k), ("v", v)):
        if layer[n + "e"] is None:
            layer[n][at] = x
            continue
        x = x.float()
        m, e = torch.frexp(x.abs().amax(-1))
        e = torch.where(m > 0.875, e - 8, e - 9).clamp(-120, 120)
        layer[n][at] = torch.ldexp(x, -e[..., None]).to(torch.float8_e4m3fn)
        layer[n + "e"][at] = e.to(torch.int32)


def _plain_rows(layer, n, at):
    """Rows of the pages in 32 bits."""
    if layer[n + "e"] is None:
        return layer[n][at].float()
    return torch.ldexp(layer[n].view(torch.uint8)[at].view(torch.float8_e4m3fn).float(), layer[n + "e"][at][..., None])


def _plain_attend(c, s):
    starts, lens, q = s["starts"], s["lens"], s["q"]
    b, H, kv, D, page = c["batch"], c["heads"], c["kv"], c["D"], c["page"]
    g, nq, width = H // kv, s["max_chunk"], s["table"].shape[1]
    L, T = width * page, q.shape[0]
    i = torch.arange(nq, device=DEV)
    j = torch.arange(L, device=DEV)
    rows = starts[:-1, None].long() + i
    rows = torch.where(rows < starts[1:, None], rows, torch.full_like(rows, T))
    base = (lens - starts[1:] + starts[:-1]).long()
    pos = base[:, None] + i                                            # [b, nq]
    seen = j <= pos[..., None]                                          # [b, nq, L]
    if c["tree"]:
        N, lead = c["tree"], nq - c["tree"]
        pos[:, lead:] = (base + lead - 1)[:, None] + s["depth"]
        first = base + lead
        rel = (j - first[:, None]).clamp(0, N - 1)                      # [b, L]
        inside = (j >= first[:, None]) & (j < first[:, None] + N)
        nodes = torch.gather(s["mask"].bool(), 2, rel[:, None].expand(b, N, L)) & inside[:, None]
        before = (j < first[:, None])[:, None].expand(b, N, L)
        seen[:, lead:] = before | nodes
    if c["window"]:
        near = (j > pos[..., None] - c["window"]) | (j < c["sinks"])
        if c["tree"]:
            near[:, lead:] |= nodes
        seen &= near
    at = s["table"].long()
    k = _plain_rows(s["layers"][0], "k", at).reshape(b, L, kv, D)
    v = _plain_rows(s["layers"][0], "v", at).reshape(b, L, kv, D)
    qf = torch.cat([q, q.new_zeros(1, H, D)])[rows].float().reshape(b, nq, kv, g, D)
    out = q.new_zeros(T + 1, kv, g, D)
    step = kv if b * H * nq * L <= 2 ** 30 else 1                       # (kv heads at a time)
    for h in range(0, kv, step):
        qh = qf[:, :, h:h + step].permute(0, 2, 3, 1, 4).reshape(b, step, g * nq, D)
        sc = torch.matmul(qh, k[:, :, h:h + step].permute(0, 2, 3, 1).contiguous()).mul_(s["scale"])
        sc = sc.view(b, step, g, nq, L).masked_fill_(~seen[:, None, None], -math.inf)
        m = sc.amax(-1, keepdim=True).clamp_min(-3e38)
        p = sc.sub_(m).exp_()
        z = p.sum(-1, keepdim=True)
        o = torch.matmul(p.view(b, step, g * nq, L), v[:, :, h:h + step].transpose(1, 2).contiguous())
        o = o.view(b, step, g, nq, D) / torch.where(z > 0, z, torch.ones_like(z))
        out[rows, h:h + step] = o.permute(0, 3, 1, 2, 4).to(q.dtype)
    return out[:T].reshape(T, H, D)


def _plain_accept(c, s):
    b, N = c["batch"], c["tree"]
    idx = torch.arange(N, device=DEV)
    cur = torch.full((b,), -1, device=DEV)
    path = torch.full((b, N), -1, dtype=torch.int32, device=DEV)
    count = torch.zeros(b, dtype=torch.int32, device=DEV)
    on = torch.ones(b, dtype=torch.bool, device=DEV)
    for d in range(min(N, DEPTH)):
        t = s["target"].gather(1, (cur + 1)[:, None])
        hit = (s["parents"] == cur[:, None]) & (s["tokens"] == t) & (idx < s["n_nodes"][:, None]) & on[:, None]
        nxt = torch.where(hit, idx, torch.full_like(idx, N)).amin(1)
        on = nxt < N
        path[:, d] = torch.where(on, nxt, torch.full_like(nxt, -1)).int()
        cur = torch.where(on, nxt, cur)
        count += on.int()
    return path, count, s["target"].gather(1, (cur + 1)[:, None])[:, 0]


def _plain_commit(c, s, layer, path, count):
    N, page = c["tree"], c["page"]
    idx = torch.arange(N, device=DEV)
    first = (s["lens"] - N)[:, None]
    to = first + idx
    frm = torch.where(idx < count[:, None], first + path, to)
    seq = torch.arange(c["batch"], device=DEV)[:, None]
    src = (s["table"][seq, frm // page].long(), (frm % page).long())
    dst = (s["table"][seq, to // page].long(), (to % page).long())
    for n in ("k", "v", "ke", "ve"):
        if layer[n] is not None:
            x = layer[n].view(torch.uint8) if c["cache"] == "fp8" and n in ("k", "v") else layer[n]
            x[dst] = x[src]


# ---- the interface ------------------------------------------------------------------

def _cache_dtype(c):
    return torch.float8_e4m3fn if c["cache"] == "fp8" else _dt(c["cache"])


def prepare(case, seed):
    c, x = case, _inputs(case, seed)
    sizes = x["sizes"]
    chunks, lens = [m for _, m in sizes], _i32([n for n, _ in sizes])
    s = dict(case=c, own=own, starts=_starts(chunks), lens=lens, table=x["table"], max_chunk=max(chunks),
             max_len=max(n for n, _ in sizes), scale=1.0 / math.sqrt(c["D"]))
    for n in ("q", "mask", "depth", "tokens", "parents", "n_nodes", "target"):
        s[n] = x.get(n)
    if own:
        from paper_2607_08642_amd import binding
        s["cache"] = binding.Cache(x["pages"], c["page"], c["kv"], c["D"], _cache_dtype(c), layers=c["layers"],
                                   device=DEV)
        s["chunk"] = binding.Chunk(s["starts"], lens, s["table"], s["max_chunk"], s["max_len"])
        if c["family"] == "attend":
            every = binding.Chunk(_starts([n for n, _ in sizes]), lens, s["table"], s["max_len"], s["max_len"])
            s["cache"].append(every, x["k"][0], x["v"][0])
        if c["family"] == "commit":
            b, N = c["batch"], c["tree"]
            t = binding.Tree.empty(b, N, DEV)
            for f in ("tokens", "parents", "depth", "mask", "n_nodes"):
                getattr(t, f).copy_(x[f])
            s["tree"] = t
    else:
        s["layers"] = [_plain_cache(c, x["pages"]) for _ in range(c["layers"])]
        if c["family"] == "attend":
            at = _where(_starts([n for n, _ in sizes]), lens, s["table"], c["page"], x["k"][0].shape[0])
            _plain_append(s["layers"][0], at, x["k"][0], x["v"][0])
    if c["family"] != "attend":
        s.update(k=x["k"], v=x["v"])
    return s


def run(state):
    s, c = state, state["case"]
    if s["own"]:
        cache, chunk = s["cache"], s["chunk"]
        if c["family"] == "attend":
            return cache.attend(chunk, s["q"], s["scale"], window=c["window"], sinks=c["sinks"], mask=s["mask"],
                                depth=s["depth"])
        for n in range(c["layers"]):
            cache.append(chunk, s["k"][n], s["v"][n], layer=n)
        out = {}
        if c["family"] == "commit":
            from paper_2607_08642_amd import binding
            a = binding.accept_tree(s["tree"], s["target"])
            cache.commit(chunk, a.path, a.n_accepted)
            out.update(path=a.path, count=a.n_accepted, next=a.next_token)
        out["rows"] = [cache.read(chunk, len(k), layer=n) for n, k in enumerate(s["k"])]
        return out
    if c["family"] == "attend":
        return _plain_attend(c, s)
    at = _where(s["starts"], s["lens"], s["table"], c["page"], s["k"][0].shape[0])
    for n in range(c["layers"]):
        _plain_append(s["layers"][n], at, s["k"][n], s["v"][n])
    out = {}
    if c["family"] == "commit":
        path, count, nxt = _plain_accept(c, s)
        for n in range(c["layers"]):
            _plain_commit(c, s, s["layers"][n], path, count)
        out.update(path=path, count=count, next=nxt)
    dt = _dt(c["dtype"])
    out["rows"] = [tuple(_plain_rows(y, n, at).to(dt) for n in ("k", "v")) for y in s["layers"]]
    return out


def _pairs(c):
    """(query, key) pairs of one head that the mask lets through, and the keys that some query sees."""
    pairs = keys = 0
    for n, m in _sizes(c):
        base, W, S = n - m, c["window"], c["sinks"]
        if c["tree"]:   # (the nodes at a depth of one each: their number of ancestors depends on the tree)
            seen = min(n, base + 2)
            pairs += m * (min(seen, W + S) if W else seen)
            keys += min(n, W + m + S) if W else n
            continue
        if not W:
            pairs += m * base + m * (m + 1) // 2
            keys += n
            continue
        for p in range(base, n):
            lo = max(0, p - W + 1)
            pairs += p + 1 - lo + min(S, lo)
        lo = max(0, base - W + 1)
        keys += n - lo + min(S, lo)
    return pairs, keys


def work(case):
    c = case
    es = 2 if c["dtype"] == "bf16" else 4
    row = c["kv"] * c["D"] * es                                   # a token's keys (or values) in the data type
    kept = c["kv"] * (c["D"] + 1 if c["cache"] == "fp8" else c["D"] * es)
    new = sum(m for _, m in _sizes(c))
    if c["family"] == "attend":
        pairs, keys = _pairs(c)
        return dict(bytes=2 * keys * kept + 2 * new * c["heads"] * c["D"] * es,
                    flops=4.0 * c["heads"] * c["D"] * pairs)
    # rows in, into the cache, out of it, out; for 8 bits a maximum, a product and a rounding each, and a product back
    nbytes = c["layers"] * 4 * new * (row + kept)
    flops = c["layers"] * 2.0 * new * c["kv"] * c["D"] * (4 if c["cache"] == "fp8" else 1)
    if c["family"] == "commit":   # the tree's arrays; about five rows of a path moved
        nbytes += c["batch"] * (12 * c["tree"] + c["layers"] * 5 * 4 * kept)
    return dict(bytes=nbytes, flops=flops)


# ---- the definition in 64 bits ---------------------------------------------------------

def _held(c, x):
    """What the cache holds for x, in 64 bits."""
    x = x.double()
    if c["cache"] != "fp8":
        return x
    top = x.abs().amax(-1, keepdim=True)
    scale = torch.exp2(torch.ceil(torch.log2(top.clamp_min(1e-300) / 448.0)).clamp(-120, 120))
    scale = torch.where(top > 448.0 * scale, scale * 2, scale)       # (log2's own rounding, either way)
    scale = torch.where(top <= 224.0 * scale, scale / 2, scale)
    y = x / scale
    grain = torch.exp2(torch.floor(torch.log2(y.abs().clamp_min(2.0 ** -6))) - 3)
    return torch.round(y / grain) * grain * scale                     # (to nearest, ties to even)


def _exact_attend(c, x):
    q, out, tok, row = x["q"].double(), [], 0, 0
    g = c["heads"] // c["kv"]
    for b, (n, m) in enumerate(x["sizes"]):
        base = n - m
        p = torch.arange(base, n, device=DEV)
        key = torch.arange(n, device=DEV)
        if c["tree"]:
            lead = m - c["tree"]
            p[lead:] = base + lead - 1 + x["depth"][b]
        o = torch.empty(m, c["heads"], c["D"], dtype=torch.float64, device=DEV)
        k, v = _held(c, x["k"][0][tok:tok + n]), _held(c, x["v"][0][tok:tok + n])
        for r0 in range(0, m, 1024):
            r1 = min(m, r0 + 1024)
            ok = torch.zeros(r1 - r0, n, dtype=torch.bool, device=DEV)
            for r in range(r0, r1) if c["tree"] else ():
                if r < lead:
                    ok[r - r0, :base + r + 1] = True
                else:
                    ok[r - r0, :base + lead] = True
                if c["window"]:
                    ok[r - r0, c["sinks"]:max(c["sinks"], int(p[r]) - c["window"] + 1)] = False
                if r >= lead:
                    ok[r - r0, base + lead:] = x["mask"][b, r - lead].bool()
            if not c["tree"]:
                gap = p[r0:r1, None] - key
                ok = gap >= 0
                if c["window"]:
                    ok &= (gap < c["window"]) | (key < c["sinks"])
            for h in range(c["heads"]):
                s = (q[row + r0:row + r1, h] @ k[:, h // g].T) / math.sqrt(c["D"])
                w = torch.softmax(s.masked_fill(~ok, -math.inf), -1)
                o[r0:r1, h] = w @ v[:, h // g]
        out.append(o)
        tok, row = tok + n, row + m
    return torch.cat(out)


def exact(case, seed):
    c = case
    if c["tree"] and c["family"] == "attend" and c["batch"] * c["tree"] > 4096:
        return None   # (row by row)
    x = _inputs(c, seed)
    if c["family"] == "attend":
        return _exact_attend(c, x)
    rows = [[_held(c, k), _held(c, v)] for k, v in zip(x["k"], x["v"])]
    if c["family"] == "store":
        return dict(rows=[tuple(r) for r in rows])
    tok, par, tgt = x["tokens"].tolist(), x["parents"].tolist(), x["target"].tolist()
    N = c["tree"]
    for b in range(c["batch"]):
        at, path = -1, []
        while True:
            go = [i for i in range(N) if par[b][i] == at and tok[b][i] == tgt[b][at + 1]]
            if not go:
                break
            at = go[0]
            path.append(at)
        first = b * (N + 1) + 1
        for r in rows:
            for n in (0, 1):
                r[n][first:first + len(path)] = r[n][[first + i for i in path]]
    return dict(path=None, count=None, next=None, rows=[tuple(r) for r in rows])
