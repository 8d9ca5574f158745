"""Decoding rounds over 16- and 8-bit caches, looked at call by call: the attention of every layer against the 64-bit form
on what the cache holds, accepted paths against the definition, and the cache before and after a commit."""
import os
import sys

import numpy as np
import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

import verify_ref as ref  # noqa: E402
from paper_2607_08642_amd import binding  # noqa: E402
from test_gpu_attend import allowed  # noqa: E402
from test_gpu_cache import i32, same  # noqa: E402

pytestmark = pytest.mark.gpu


class Watch:
    """The calls of decode_rounds.decode_trees, each checked as it is made."""

    def __init__(self, monkeypatch, window):
        self.window, self.attends, self.accepted, self.moved, self.tokens = window, 0, 0, 0, []
        attend, commit, accept = binding.Cache.attend, binding.Cache.commit, binding.accept_tree
        build = binding.Plan.build_tree

        def build_with_rivals(plan, logits, T):
            """Every other level's likeliest token has one that is a little likelier: the path that the target agrees
            with is not the tree's first nodes then, and its rows have to move."""
            logits = logits.clone()
            top, at = logits[:, ::2].max(-1, keepdim=True)
            logits[:, ::2].scatter_(2, (at + 1) % logits.shape[-1], top + 0.5)
            return build(plan, logits, T)

        def watched_attend(cache, chunk, q, layer=0, **kw):
            out = attend(cache, chunk, q, layer=layer, **kw)
            if kw.get("mask") is not None:
                self.check_attend(cache, chunk, q, layer, kw, out)
            return out

        def watched_commit(cache, chunk, path, n_accepted):
            rows = int(chunk.starts[-1])
            before = [cache.read(chunk, rows, layer=n) for n in range(cache.layers)]
            commit(cache, chunk, path, n_accepted)
            for n in range(cache.layers):
                for was, now in zip(before[n], cache.read(chunk, rows, layer=n)):
                    self.check_rows(chunk, path, n_accepted, was, now)

        def watched_accept(tree, target):
            a = accept(tree, target)
            self.check_accept(tree, target, a)
            return a

        monkeypatch.setattr(binding.Plan, "build_tree", build_with_rivals)
        monkeypatch.setattr(binding.Cache, "attend", watched_attend)
        monkeypatch.setattr(binding.Cache, "commit", watched_commit)
        monkeypatch.setattr(binding, "accept_tree", watched_accept)

    def check_attend(self, cache, chunk, q, layer, kw, out):
        starts, lens = chunk.starts.tolist(), chunk.lens.tolist()
        ends = np.cumsum([0] + lens).tolist()
        every = binding.Chunk(i32(ends), chunk.lens.clone(), chunk.table, max(lens), max(lens))
        k, v = (x.cpu() for x in cache.read(every, ends[-1], layer=layer))
        mask, depth = kw["mask"].cpu().numpy(), kw["depth"].cpu().numpy()
        for b, n in enumerate(lens):
            rows, keys = slice(starts[b], starts[b + 1]), slice(ends[b], ends[b + 1])
            m = starts[b + 1] - starts[b]
            ok = ref.visible(m, n - m, n, self.window, kw["sinks"], mask[b], depth[b])
            scale = cache.head_dim ** -0.5
            want = ref.attend(q[rows].cpu(), k[keys], v[keys], scale, ok)
            tol = allowed(q[rows].cpu(), k[keys], v[keys], scale, ok, cache.data_dtype)
            assert bool(((out[rows].double().cpu() - want).abs() <= tol).all()), (layer, b)
        self.attends += 1

    def check_accept(self, tree, target, a):
        for b, n in enumerate(tree.n_nodes.tolist()):
            tokens, parents = tree.tokens[b].tolist(), tree.parents[b].tolist()
            path, nxt = ref.accept(tokens, parents, n, target[b].tolist())
            assert a.path[b].tolist() == path + [-1] * (len(tokens) - len(path))
            assert (int(a.n_accepted[b]), int(a.next_token[b])) == (len(path), nxt)
            self.accepted += len(path)
            self.tokens.append([tokens[i] for i in path] + [nxt])

    def check_rows(self, chunk, path, n_accepted, was, now):
        want, N = was.clone(), path.shape[1]
        for b, n in enumerate(n_accepted.tolist()):
            first = int(chunk.starts[b + 1]) - N
            at = path[b, :n].tolist()
            want[first:first + n] = was[[first + i for i in at]]
            self.moved += sum(i != j for j, i in enumerate(at))
        assert same(now, want)


@pytest.mark.parametrize("cache", ["bf16", "fp8"])
@pytest.mark.parametrize("window", [0, 48])
def test_rounds_call_by_call(cache, window, monkeypatch):
    import decode_rounds
    print(f"[rounds] {cache} window={window}", flush=True)
    watch, rounds, batch = Watch(monkeypatch, window), 5, 2
    plain, trees = decode_rounds.run(cache, window, batch=batch, steps=40, rounds=rounds, seed=4)
    assert watch.attends == rounds * decode_rounds.LAYERS
    for i, t in enumerate(trees):
        assert t[1:] == sum(watch.tokens[i::batch], [])     # (after the prompt's token: the rounds' in order)
    # the drafter is right four times out of five, so paths are accepted and rows move
    assert watch.accepted > rounds and watch.moved > 0
