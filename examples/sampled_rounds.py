"""Samples of prompts by speculative rounds: pages, rotated heads, trees, sampled tokens.

Each prompt becomes several samples.  The prompts go through the target once; Pages.fork makes their samples, which
share the whole pages of the prompt.  Then rounds as a serving program runs them: Pages.fit gives every sequence pages
for the root and the tree, Cache.append_rotated norms and rotates the heads by position and writes the keys and values,
Cache.attend reads them under the tree's mask, sample draws the target's token at the root and at every node,
accept_tree and Cache.commit keep the path that agrees.  Half way some samples end: their pages go free, and Pages.compact
moves the rest together.  Nothing waits for the device.

The random number of a token belongs to its sequence and position, whichever way it is drawn, so speculation must not
change the samples: they are compared with plain decoding, one token at a time.  The drafter is made up: it peeks at
that continuation four times out of five.

    python examples/sampled_rounds.py [--cache f32|bf16|fp8] [--samples 3] [--rounds 10]
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
SETTINGS = dict(temperature=0.8, top_k=40, top_p=0.95, min_p=0.01)


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


class Target:
    """A few layers of attention with random weights."""

    def __init__(self, cache: binding.Cache, seed: int):
        g = torch.Generator(device=DEV)
        g.manual_seed(seed)
        w = lambda *s: torch.randn(*s, generator=g, device=DEV) / s[-1] ** 0.5  # noqa: E731
        norm = lambda: (1 + 0.2 * torch.randn(HEAD_DIM, generator=g, device=DEV)).to(cache.data_dtype)  # noqa: E731
        self.emb = w(VOCAB, WIDTH) * 4
        rows = (HEADS + 2 * KV_HEADS) * HEAD_DIM
        self.layers = [{"qkv": w(rows, WIDTH), "q_norm": norm(), "k_norm": norm(), "o": w(WIDTH, HEADS * HEAD_DIM),
                        "up": w(WIDTH, WIDTH), "down": w(WIDTH, WIDTH)} for _ in range(LAYERS)]
        self.inv_freq = 1e4 ** (-torch.arange(0, HEAD_DIM, 2, device=DEV) / HEAD_DIM)
        self.cache = cache

    def logits(self, chunk, tokens, positions, tree=None):
        """[rows, VOCAB] after each row; the rows' keys and values are in the cache after it."""
        x, dt = self.emb[tokens.long()], self.cache.data_dtype
        opts = {} if tree is None else dict(mask=tree.mask, depth=tree.depth)
        for n, w in enumerate(self.layers):
            y = torch.nn.functional.layer_norm(x, (WIDTH,)) @ w["qkv"].T
            y = y.to(dt).view(len(x), -1, HEAD_DIM)
            q, k, v = y.split((HEADS, KV_HEADS, KV_HEADS), 1)
            q = self.cache.append_rotated(chunk, q, k, v, positions, self.inv_freq, w["q_norm"], w["k_norm"], layer=n)
            o = self.cache.attend(chunk, q, layer=n, **opts)
            x = x + o.float().view(len(x), -1) @ w["o"].T
            x = x + torch.relu(torch.nn.functional.layer_norm(x, (WIDTH,)) @ w["up"].T) @ w["down"].T
        return torch.nn.functional.layer_norm(x, (WIDTH,)) @ self.emb.T * 0.25


def start(target, pages, prompts, samples, numbers):
    """The prompts through the target, their samples forked; the first token of each [batch]."""
    batch = len(prompts) * samples
    counts = [len(prompts[b // samples]) if b % samples == 0 else 0 for b in range(batch)]
    starts = i32([0] + list(torch.tensor(counts).cumsum(0)))
    leader = torch.arange(batch, device=DEV, dtype=torch.int32) // samples * samples
    pages.lens.copy_(i32(counts))
    pages.fit()
    chunk = binding.Chunk(starts, pages.lens, pages.table, max(counts), pages.width * PAGE)
    out = target.logits(chunk, i32([t for p in prompts for t in p]), i32([i for p in prompts for i in range(len(p))]))
    pages.fork(leader)
    last = starts[1:].long()[leader.long()] - 1
    at = (pages.lens - 1).long()
    return binding.sample(out[last], numbers.gather(1, at[:, None])[:, 0].contiguous(), **SETTINGS)


def decode_plain(target, pages, token, steps, numbers):
    """One token at a time: [batch, steps] tokens after the first."""
    chunk = binding.Chunk(torch.arange(pages.batch + 1, dtype=torch.int32, device=DEV), pages.lens, pages.table, 1,
                          pages.width * PAGE)
    out = []
    for _ in range(steps):
        position = pages.lens.clone()
        pages.lens += 1
        pages.fit()
        u = numbers.gather(1, position[:, None].long())[:, 0].contiguous()
        token = binding.sample(target.logits(chunk, token, position), u, **SETTINGS)
        out.append(token)
    return torch.stack(out, 1)


def decode_trees(target, pages, plan, token, rounds, ahead, numbers, seed, ends):
    """Rounds of trees; sequences `ends` end half way.  Accepted node tokens (-1: none) and the token after them, of
    every round."""
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    b = pages.batch
    chunk = binding.Chunk(torch.arange(b + 1, dtype=torch.int32, device=DEV) * (BUDGET + 1), pages.lens, pages.table,
                          BUDGET + 1, pages.width * PAGE)
    at = torch.zeros(b, dtype=torch.long, device=DEV)       # tokens generated so far
    levels = torch.arange(DEPTH, device=DEV)
    going = torch.ones(b, dtype=torch.int32, device=DEV)
    results = []
    for n in range(rounds):
        if n == rounds // 2:
            going[ends] = 0
            pages.lens *= going
            pages.fit()
            pages.compact()
        draft = torch.randn(b, DEPTH, VOCAB, generator=g, device=DEV)
        peek = ahead.gather(1, (at[:, None] + levels).clamp(max=ahead.shape[1] - 1)).long()
        right = torch.rand(b, DEPTH, generator=g, device=DEV) < 0.8
        draft.scatter_add_(2, peek[..., None], torch.where(right, 9.0, 0.0)[..., None])
        tree = plan.build_tree(draft, 1.0)
        tokens = torch.cat([token[:, None], tree.tokens.clamp(min=0)], 1).flatten()
        depth = torch.cat([torch.zeros_like(tree.depth[:, :1]), tree.depth], 1)
        positions = pages.lens[:, None] + depth
        kept = pages.lens.clone()
        pages.lens += BUDGET + 1      # (ended sequences go on with a round of their own: the batch keeps its shape)
        pages.fit()
        u = numbers.gather(1, positions.long().clamp(max=numbers.shape[1] - 1))
        own = binding.sample(target.logits(chunk, tokens, positions.flatten(), tree).view(b, BUDGET + 1, VOCAB), u, **SETTINGS)
        a = binding.accept_tree(tree, own)
        target.cache.commit(chunk, a.path, a.n_accepted)
        path = tree.tokens.gather(1, a.path.clamp(min=0).long())
        results.append((torch.where(a.path >= 0, path, -1), a.next_token))
        token = a.next_token
        pages.lens.copy_((kept + 1 + a.n_accepted) * going)
        at += 1 + a.n_accepted
    return results


def run(cache="f32", samples=3, steps=80, rounds=10, seed=0):
    """(tokens of plain decoding [batch, steps], tokens of the rounds: a list for each sequence, pages in use before and
    after the samples ended)."""
    gen = torch.Generator().manual_seed(seed)
    prompts = [torch.randint(0, VOCAB, (n,), generator=gen).tolist() for n in (75, 33)]
    batch = len(prompts) * samples
    ends = [b for b in range(batch) if b % samples == samples - 1]
    width = -(-(max(len(p) for p in prompts) + max(steps, rounds * (DEPTH + 1)) + BUDGET + 2) // PAGE)
    numbers = torch.rand(batch, width * PAGE, generator=torch.Generator().manual_seed(seed + 1)).to(DEV)
    plan_w = [torch.zeros(s, device=DEV) for s in ((VOCAB, 32), (96, 32), (96, 32))]
    plan = binding.Plan(*plan_w, None, None, torch.zeros(32, 32, device=DEV), None, L=DEPTH, M=MENU, B=BUDGET,
                        logits_dtype=binding.DT_F32, max_batch=batch)
    outs, books = [], None
    for way in ("plain", "trees"):
        c = binding.Cache(batch * width, PAGE, KV_HEADS, HEAD_DIM, CACHES[cache], layers=LAYERS)
        target, pages = Target(c, seed), binding.Pages(c, batch, width)
        first = start(target, pages, prompts, samples, numbers)
        if way == "plain":
            outs.append(torch.cat([first[:, None], decode_plain(target, pages, first, steps - 1, numbers)], 1))
        else:
            results = decode_trees(target, pages, plan, first, rounds, outs[0][:, 1:], numbers, seed + 2, ends)
            tokens = [[int(first[i])] for i in range(batch)]
            for n, (kept, nxt) in enumerate(results):
                for i in range(batch):
                    if n < rounds // 2 or i not in ends:
                        tokens[i] += [t for t in kept[i].tolist() if t >= 0] + [int(nxt[i])]
            outs.append(tokens)
            books = pages
    plan.close()
    return outs, books


def main():
    p = argparse.ArgumentParser()
    p.add_argument("--cache", choices=sorted(CACHES), default="f32")
    p.add_argument("--samples", type=int, default=3)
    p.add_argument("--rounds", type=int, default=10)
    a = p.parse_args()
    (plain, trees), pages = run(a.cache, a.samples, rounds=a.rounds)
    for i, t in enumerate(trees):
        n = min(len(t), plain.shape[1])
        same = next((j for j in range(n) if t[j] != int(plain[i, j])), n)
        print(f"sample {i}: {len(t)} tokens, {same} of {n} compared as in plain decoding")
    print(f"{int((pages.uses > 0).sum())} pages in use, {int((pages.uses > 1).sum())} of them by several samples")


if __name__ == "__main__":
    main()
