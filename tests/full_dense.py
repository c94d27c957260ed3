"""Softmax attention over the pairs that an 8-bit full-context cache holds, in 64 bits, a stream at a time: for caches that are too long for the
pair-by-pair oracle.  The pairs are taken as the cache has them (codes times scales); what append and evict put there is checked elsewhere."""
from __future__ import annotations

import math

import torch


def pairs(c, b, h):
    """Keys, values and token indices of a stream, in 64 bits."""
    n = int(c.count[b, h])
    at = torch.arange(n, device=c.device) // 64
    return (c.k[b, h, :n].double() * c.k_scale[b, h].double()[at][:, None], c.v[b, h, :n].double() * c.v_scale[b, h].double()[at][:, None],
            c.idx[b, h, :n].long())


def attend(c, q, lens=None, scale=None):
    """q [B, Hq, T, d] -> y [B, Hq, T, d] and the weight that the call adds to every slot [B, Hkv, capacity]."""
    B, Hq, T, d = q.shape
    g = Hq // c.Hkv
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    y = torch.zeros((B, Hq, T, d), dtype=torch.float64, device=c.device)
    w = torch.zeros((B, c.Hkv, c.capacity), dtype=torch.float64, device=c.device)
    for b in range(B):
        n = T if lens is None else min(max(int(lens[b]), 0), T)
        for h in range(c.Hkv):
            K, V, idx = pairs(c, b, h)
            if not n or not len(idx):
                continue
            pos = int(c.n_tokens[b, h]) - n + torch.arange(n, device=c.device)
            hidden = idx[None] > pos[:, None]
            none = hidden.all(1)
            for r in range(h * g, (h + 1) * g):
                s = (q[b, r, :n].double() @ K.t() * scale).masked_fill_(hidden, float("-inf"))
                p = torch.softmax(s, -1)
                p[none] = 0.0
                y[b, r, :n] = p @ V
                w[b, h, :len(idx)] += torch.where(torch.isfinite(p).all(1, keepdim=True), p, 0.0).sum(0)
    return y, w


def distance(x, want):
    """2-norm of the difference relative to the 2-norm of `want`."""
    return float((x.double() - want).norm() / want.norm())
