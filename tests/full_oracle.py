"""Plain implementation of the 8-bit full-context cache (include/lola.h, lola_full_*) in 64 bits on the host, stream by stream and
pair by pair, and the distance that a result computed in fewer bits may have from it."""
from __future__ import annotations

import math

import numpy as np

BLK = 64
TOP = 448.0


def exponent(a: float) -> int:
    """Least integer e >= -100 with a <= 448 * 2^e."""
    e = -100
    if a > 0:
        e = max(e, math.frexp(a)[1] - 10)
        while a > math.ldexp(TOP, e):
            e += 1
    return e


def e4m3(x):
    """x (|x| <= 448) rounded to the nearest e4m3 number, ties to even; NaN stays."""
    x = np.asarray(x, np.float64)
    e = np.maximum(np.frexp(np.where(np.isfinite(x), x, 0.0))[1] - 1, -6)
    step = np.ldexp(1.0, e - 3)
    return np.where(np.isnan(x), np.nan, np.rint(x / step) * step)


class Stream:
    def __init__(self, cap, d):
        self.cap, self.d = cap, d
        self.k, self.v = np.zeros((cap, d)), np.zeros((cap, d))            # codes as values
        self.ek, self.ev = np.full(cap // BLK, -100), np.full(cap // BLK, -100)
        self.idx, self.weight = np.full(cap, -1, np.int64), np.zeros(cap)
        self.count = self.n = 0

    def append(self, k, v):
        k, v = np.array(k, np.float64), np.array(v, np.float64)
        bad = ~(np.isfinite(k).all(1) & np.isfinite(v).all(1))
        v[~np.isfinite(v)] = 0.0
        told, k, v = len(k), k[:self.cap - self.count], v[:self.cap - self.count]
        bad = bad[:len(k)]
        a, n = self.count, len(k)
        for J in range(a // BLK, (a + n + BLK - 1) // BLK) if n else ():
            lo, hi = max(a, J * BLK), min(a + n, J * BLK + BLK)
            for codes, es, x, nan in ((self.k, self.ek, k, bad), (self.v, self.ev, v, None)):
                x = x[lo - a:hi - a]
                fine = x if nan is None else x[~nan[lo - a:hi - a]]
                e = exponent(float(np.abs(fine).max())) if fine.size else -100
                if lo > J * BLK:
                    e = max(e, int(es[J]))
                    codes[J * BLK:lo] = e4m3(np.ldexp(codes[J * BLK:lo], int(es[J]) - e))
                es[J] = e
                y = np.zeros_like(x)
                ok = np.ones(len(x), bool) if nan is None else ~nan[lo - a:hi - a]
                y[ok] = e4m3(np.ldexp(x[ok], -e))
                y[~ok] = np.nan
                codes[lo:hi] = y
        self.idx[a:a + n] = self.n + np.arange(n)
        self.weight[a:a + n] = 0.0
        self.count, self.n = a + n, self.n + told

    def pairs(self):
        s = np.arange(self.count) // BLK
        return np.ldexp(self.k[:self.count], self.ek[s][:, None]), np.ldexp(self.v[:self.count], self.ev[s][:, None])

    def attend(self, q, scale, gather):
        """q [g, n, d] of the newest n tokens -> y [g, n, d] and, per row, how far y may be off (relative to the largest |v|)."""
        g, n, d = q.shape
        K, V = self.pairs()
        y, off, woff = np.zeros((g, n, d)), np.zeros((g, n)), np.zeros(self.count)
        add = np.zeros(self.count)
        for i in range(n):
            seen = np.nonzero(self.idx[:self.count] <= self.n - n + i)[0]
            if not len(seen):
                continue
            for r in range(g):
                with np.errstate(invalid="ignore"):
                    s = scale * (K[seen] @ q[r, i])
                    size = scale * (np.abs(K[seen]) @ np.abs(q[r, i]))
                    p = np.exp(s - s.max())
                    p /= p.sum()
                    y[r, i] = p @ V[seen]
                # A dot product of d terms in 32 bits is off by at most d half steps of the sum of magnitudes, the exponent's own
                # roundings by 4 more of it, sums over n pairs and the exponential by n + 16 half steps.
                e = 2.0 ** -24 * ((d + 4) * (np.nanmax(size) if np.isfinite(size).any() else 0.0) + len(seen) + 16)
                off[r, i] = 2 * e
                if not np.isnan(y[r, i]).any():
                    add[seen] += p
                    woff[seen] += 2 * e * p
        if gather:
            self.weight[:self.count] += add
        return y, off, woff

    def evict(self, keep, first, recent):
        if self.count <= keep:
            return
        i, w = self.idx[:self.count], self.weight[:self.count]
        order = sorted(range(self.count), key=lambda s: (0 if i[s] < first or i[s] >= self.n - recent else 1, 0 if np.isnan(w[s]) else 1,
                                                         -w[s] if not np.isnan(w[s]) else 0.0, s))
        kept = set(order[:keep])
        holes = [s for s in range(keep) if s not in kept]
        moves = [s for s in range(keep, self.count) if s in kept]
        assert len(holes) == len(moves)
        K, V = self.pairs()
        for codes, es, X in ((self.k, self.ek, K), (self.v, self.ev, V)):
            need = {}
            for t, s in zip(holes, moves):
                x = np.nan_to_num(np.abs(X[s]))
                need[t // BLK] = max(need.get(t // BLK, -100), exponent(float(x.max())))
            for J, e in need.items():
                if e > es[J]:
                    end = min(J * BLK + BLK, keep)
                    codes[J * BLK:end] = e4m3(np.ldexp(codes[J * BLK:end], int(es[J]) - e))
                    es[J] = e
            for t, s in zip(holes, moves):
                codes[t] = e4m3(np.ldexp(X[s], -int(es[t // BLK])))
        for x in (self.idx, self.weight):
            x[holes] = x[moves]
        self.count = keep


class FullOracle:
    def __init__(self, B, Hq, Hkv, d, cap, scale=0.0):
        self.B, self.Hq, self.Hkv, self.d, self.g = B, Hq, Hkv, d, Hq // Hkv
        self.scale = scale if scale > 0 else 1.0 / math.sqrt(d)
        self.s = [[Stream(cap, d) for _ in range(Hkv)] for _ in range(B)]

    def each(self):
        for b in range(self.B):
            for h in range(self.Hkv):
                yield b, h, self.s[b][h]

    def append(self, k, v, lens=None):
        """k, v [B, Hkv, T, d]."""
        for b, h, s in self.each():
            n = k.shape[2] if lens is None else min(max(int(lens[b]), 0), k.shape[2])
            s.append(k[b, h, :n], v[b, h, :n])

    def attend(self, q, lens=None, gather=False):
        """q [B, Hq, T, d] -> y, the rows' allowed distance in units of the stream's largest |v|, that largest |v| per row, and the
        weights' allowed distance per stream."""
        T = q.shape[2]
        y, off, top, woff = np.zeros(q.shape), np.zeros(q.shape[:3]), np.zeros(q.shape[:3]), {}
        for b, h, s in self.each():
            n = T if lens is None else min(max(int(lens[b]), 0), T)
            r = slice(h * self.g, (h + 1) * self.g)
            y[b, r, :n], off[b, r, :n], woff[b, h] = s.attend(np.asarray(q[b, r, :n], np.float64), self.scale, gather)
            top[b, r] = np.abs(s.pairs()[1]).max() if s.count else 0.0
        return y, off, top, woff

    def evict(self, keep, first=0, recent=0):
        for _, _, s in self.each():
            s.evict(keep, first, recent)
