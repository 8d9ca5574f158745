"""Speculative decoding rounds with a tree builder, a paged cache and a small target model.

Each round runs what a serving program runs: the drafter's logits become a tree (Plan.build_tree), the root and the
tree's nodes go through the target in one pass, layer by layer (Cache.append, Cache.attend under the tree's mask),
the longest path that the target agrees with is taken (accept_tree) and its rows are kept (Cache.commit).  Nothing in
a round waits for the device.

The target is a few random attention layers; its drafter's logits are made up here: the target's own continuation
(from plain decoding, one token at a time over the same cache) as the likeliest token four times out of five, so
that paths of several tokens are accepted.  Speculation must not change what is generated: the tokens of both ways
are compared.

    python examples/decode_rounds.py [--cache f32|bf16|fp8] [--window 64] [--rounds 12]
"""
import argparse
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

from paper_2607_08642_amd import binding  # noqa: E402

DEV = "cuda"
VOCAB, WIDTH, LAYERS, HEADS, KV_HEADS, HEAD_DIM = 2003, 256, 2, 8, 2, 64
DEPTH, MENU, BUDGET, PAGE = 8, 16, 16, 32     # of the trees: levels, candidates a level, nodes
CACHES = {"f32": torch.float32, "bf16": torch.bfloat16, "fp8": torch.float8_e4m3fn}


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


class Target:
    """A few layers of attention with random weights; positions are added to the embeddings."""

    def __init__(self, cache: binding.Cache, window: int, seed: int):
        g = torch.Generator(device=DEV)
        g.manual_seed(seed)
        w = lambda *s: torch.randn(*s, generator=g, device=DEV) / s[-1] ** 0.5  # noqa: E731
        self.emb, self.pos = w(VOCAB, WIDTH) * 4, w(4096, WIDTH) * 4
        self.layers = [{"q": w(HEADS * HEAD_DIM, WIDTH) * 2, "k": w(KV_HEADS * HEAD_DIM, WIDTH),
                        "v": w(KV_HEADS * HEAD_DIM, WIDTH), "o": w(WIDTH, HEADS * HEAD_DIM), "up": w(WIDTH, WIDTH),
                        "down": w(WIDTH, WIDTH)} for _ in range(LAYERS)]
        self.cache, self.window = cache, window

    def forward(self, chunk, tokens, positions, tree=None):
        """The target's token after each row ([rows] int32); the rows' keys and values are in the cache after it."""
        x = self.emb[tokens.long()] + self.pos[positions.long()]
        opts = {} if tree is None else dict(mask=tree.mask, depth=tree.depth)
        for n, w in enumerate(self.layers):
            y = torch.nn.functional.layer_norm(x, (WIDTH,))
            q, k, v = ((y @ w[m].T).view(len(x), -1, HEAD_DIM).to(self.cache.data_dtype) for m in "qkv")
            self.cache.append(chunk, k, v, layer=n)
            o = self.cache.attend(chunk, q, layer=n, window=self.window, sinks=4, **opts)
            x = x + o.float().view(len(x), -1) @ w["o"].T
            x = x + torch.relu(torch.nn.functional.layer_norm(x, (WIDTH,)) @ w["up"].T) @ w["down"].T
        return (torch.nn.functional.layer_norm(x, (WIDTH,)) @ self.emb.T).argmax(-1).int()


class Sequences:
    """The page table and lengths of a batch; a chunk's lens tensor is written before each pass."""

    def __init__(self, batch, max_len):
        width = -(-max_len // PAGE)
        self.table = torch.randperm(batch * width, device=DEV).view(batch, width).int()
        self.lens = torch.zeros(batch, dtype=torch.int32, device=DEV)   # tokens kept in the cache
        self.batch, self.max_len = batch, max_len

    def chunk(self, counts, max_chunk):
        starts = i32([0] + list(torch.tensor(counts).cumsum(0)))
        return binding.Chunk(starts, torch.empty_like(self.lens), self.table, max_chunk, self.max_len)


def prompts_pass(target, seqs, prompts):
    """All prompts in one ragged chunk; the token after each."""
    counts = [len(p) for p in prompts]
    chunk = seqs.chunk(counts, max(counts))
    chunk.lens.copy_(i32(counts))
    tokens = i32([t for p in prompts for t in p])
    positions = i32([i for p in prompts for i in range(len(p))])
    out = target.forward(chunk, tokens, positions)
    seqs.lens.copy_(chunk.lens)
    return out[chunk.starts[1:].long() - 1]


def decode_plain(target, seqs, token, steps):
    """One token at a time: [batch, steps] tokens after the first."""
    chunk = seqs.chunk([1] * seqs.batch, 1)
    out = []
    for _ in range(steps):
        torch.add(seqs.lens, 1, out=chunk.lens)
        token = target.forward(chunk, token, seqs.lens)
        seqs.lens += 1
        out.append(token)
    return torch.stack(out, 1)


def decode_trees(target, seqs, plan, token, rounds, ahead, seed):
    """Rounds of trees; `ahead` [batch, n] is the continuation that the made-up drafter peeks at.

    Returns the rounds' results: accepted node tokens (-1: none) and the token after them."""
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    b = seqs.batch
    chunk = seqs.chunk([BUDGET + 1] * b, BUDGET + 1)
    at = torch.zeros(b, dtype=torch.long, device=DEV)       # tokens generated so far
    levels = torch.arange(DEPTH, device=DEV)
    results = []
    for _ in range(rounds):
        logits = torch.randn(b, DEPTH, VOCAB, generator=g, device=DEV)
        peek = ahead.gather(1, (at[:, None] + levels).clamp(max=ahead.shape[1] - 1)).long()
        right = torch.rand(b, DEPTH, generator=g, device=DEV) < 0.8
        logits.scatter_add_(2, peek[..., None], torch.where(right, 9.0, 0.0)[..., None])
        tree = plan.build_tree(logits, 1.0)
        tokens = torch.cat([token[:, None], tree.tokens.clamp(min=0)], 1).flatten()
        positions = torch.cat([seqs.lens[:, None], seqs.lens[:, None] + tree.depth], 1).flatten()
        torch.add(seqs.lens, BUDGET + 1, out=chunk.lens)
        own = target.forward(chunk, tokens, positions, tree).view(b, BUDGET + 1)
        a = binding.accept_tree(tree, own)
        target.cache.commit(chunk, a.path, a.n_accepted)
        kept = tree.tokens.gather(1, a.path.clamp(min=0).long())
        results.append((torch.where(a.path >= 0, kept, -1), a.next_token))
        token = a.next_token
        seqs.lens += 1 + a.n_accepted
        at += 1 + a.n_accepted
    return results


def run(cache="f32", window=0, batch=3, steps=96, rounds=12, seed=0):
    """(tokens of plain decoding [batch, steps], tokens of the rounds: a list for each sequence)."""
    gen = torch.Generator().manual_seed(seed)
    prompts = [torch.randint(0, VOCAB, (n,), generator=gen).tolist() for n in (41, 7, 130, 1, 64)[:batch]]
    max_len = max(len(p) for p in prompts) + max(steps, rounds * (DEPTH + 1)) + BUDGET + 2
    plan_w = [torch.zeros(s, device=DEV) for s in ((VOCAB, 32), (96, 32), (96, 32))]
    plan = binding.Plan(*plan_w, None, None, torch.zeros(32, 32, device=DEV), None, L=DEPTH, M=MENU, B=BUDGET,
                        logits_dtype=binding.DT_F32, max_batch=batch)
    pages = batch * -(-max_len // PAGE)
    outs = []
    for way in ("plain", "trees"):
        c = binding.Cache(pages, PAGE, KV_HEADS, HEAD_DIM, CACHES[cache], layers=LAYERS)
        target, seqs = Target(c, window, seed), Sequences(batch, max_len)
        first = prompts_pass(target, seqs, prompts)
        if way == "plain":
            outs.append(torch.cat([first[:, None], decode_plain(target, seqs, first, steps - 1)], 1))
        else:
            # (the drafter looks at what comes after the root)
            results = decode_trees(target, seqs, plan, first, rounds, outs[0][:, 1:], seed + 1)
            tokens = [[int(first[i])] for i in range(batch)]
            for kept, nxt in results:
                for i in range(batch):
                    tokens[i] += [t for t in kept[i].tolist() if t >= 0] + [int(nxt[i])]
            outs.append(tokens)
    plan.close()
    return outs


def main():
    p = argparse.ArgumentParser()
    p.add_argument("--cache", choices=sorted(CACHES), default="f32")
    p.add_argument("--window", type=int, default=0)
    p.add_argument("--rounds", type=int, default=12)
    a = p.parse_args()
    plain, trees = run(a.cache, a.window, rounds=a.rounds)
    for i, t in enumerate(trees):
        n = min(len(t), plain.shape[1])
        same = next((j for j in range(n) if t[j] != int(plain[i, j])), n)
        print(f"sequence {i}: {len(t)} tokens in {a.rounds} rounds ({len(t) / a.rounds:.1f} a round), "
              f"{same} of {n} compared as in plain decoding")


if __name__ == "__main__":
    main()
