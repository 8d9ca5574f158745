"""The paged cache's calls in 64 bits on the CPU, written from their definitions, for the tests."""
from __future__ import annotations

import math

import numpy as np
import torch


def quantise(x: torch.Tensor):
    """DT_F8's codes' values and scale of rows [..., D]: 448 2^e >= max|x| over the finite x, e least."""
    x = x.double()
    top = torch.where(torch.isfinite(x), x.abs(), torch.zeros_like(x)).amax(-1, keepdim=True)
    e = torch.full_like(top, -120.0)
    while bool((small := (top > 448.0 * torch.exp2(e)) & (e < 120)).any()):
        e = torch.where(small, e + 1, e)
    y = x / torch.exp2(e)
    # e4m3: 3 bits after the leading one, the smallest normal 2^-6, so a grain of 2^-9 below it
    grain = torch.exp2(torch.floor(torch.log2(y.abs().clamp_min(2.0 ** -6))) - 3)
    q = torch.round(y / grain) * grain       # (round: to nearest, ties to even)
    q = torch.where(torch.isfinite(y), q, torch.full_like(q, math.nan))
    return q * torch.exp2(e)


def visible(n, base, length, window, sinks, mask=None, depth=None):
    """[n, length] bool: which keys the rows of one chunk see."""
    ok = np.zeros((n, length), bool)
    N = 0 if mask is None else mask.shape[0]
    lead = n - N
    for i in range(n):
        node = i >= lead and N > 0
        pos = base + lead - 1 + (int(depth[i - lead]) if window else 0) if node else base + i
        for j in range(length):
            before = j < base + lead if node else j <= base + i
            near = not window or j > pos - window or j < sinks
            ok[i, j] = (before and near) or (node and j >= base + lead and bool(mask[i - lead, j - base - lead]))
    return ok


def attend(q, k, v, scale, ok):
    """One sequence: q [n, H, D], k, v [len, Hk, D] in 64 bits, ok [n, len].  A row takes from the keys it
    sees only (nothing: zeros)."""
    n, H, D = q.shape
    g = H // k.shape[1]
    out = torch.zeros(n, H, D, dtype=torch.float64)
    q, k, v = q.double(), k.double(), v.double()
    for i in range(n):
        idx = torch.from_numpy(np.nonzero(ok[i])[0])
        if not len(idx):
            continue
        kk, vv = k[idx].repeat_interleave(g, 1), v[idx].repeat_interleave(g, 1)
        w = torch.softmax((q[i][None] * kk).sum(-1) * scale, 0)
        out[i] = (w[..., None] * vv).sum(0)
    return out


def accept(tokens, parents, n_nodes, target):
    """One tree: the accepted nodes and the token after them."""
    cur, path = -1, []
    while True:
        kids = [i for i in range(n_nodes) if parents[i] == cur and tokens[i] == target[cur + 1]]
        if not kids:
            return path, target[cur + 1]
        cur = kids[0]
        path.append(cur)
