"""The 8-bit cache by its definition, in numpy and 64 bits (tests only): e4m3 pages with power-of-two scales, the
sequences' tokens as the values they are held as, attention, accumulated weights and eviction over them.  Shares
nothing with the library."""
from __future__ import annotations

import numpy as np


def e4m3(y):
    """|y| <= 448, to the nearest e4m3 number, ties to even."""
    _, x = np.frexp(y)
    step = np.ldexp(1.0, np.maximum(x - 4, -9))
    return np.round(y / step) * step


def exponent(a):
    """The least e in [-126, 119] with a <= 448 * 2^e; -126 for a = 0."""
    m, x = np.frexp(np.asarray(a, dtype=np.float64))
    e = x - 9 + (m > 0.875)
    return np.where(m == 0, -126, np.clip(e, -126, 119)).astype(np.int64)


def quantise(k, v):
    """One page: k, v fp64 [rows][Hkv][d] -> the values held, and (exponents of K, of V), each [Hkv]."""
    bad = ~(np.isfinite(k).all(-1) & np.isfinite(v).all(-1))  # [rows][Hkv]
    k, v = np.where(bad[..., None], 0.0, k), np.where(bad[..., None], 0.0, v)
    out, exps = [], []
    for x in (k, v):
        e = exponent(np.abs(x).max(axis=(0, 2)) if x.shape[0] else np.zeros(x.shape[1]))
        s = np.ldexp(1.0, e)[None, :, None]
        out.append(e4m3(np.clip(x / s, -448, 448)) * s)
        exps.append(e)
    for x in out:
        x[bad] = np.nan
    return out[0], out[1], np.stack(exps, -1)


class Seq:
    """One sequence: K, V fp64 [L][T][Hkv][d] as held."""

    def __init__(self, L, hkv, d, ps, bits=8):
        self.ps, self.bits = ps, bits
        self.K, self.V = np.zeros((L, 0, hkv, d)), np.zeros((L, 0, hkv, d))
        self.E = np.zeros((L, 0, hkv, 2), dtype=np.int64)  # per page

    def fork(self):
        s = Seq(1, 1, 1, self.ps, self.bits)
        s.K, s.V, s.E = self.K.copy(), self.V.copy(), self.E.copy()
        return s

    def __len__(self):
        return self.K.shape[1]

    def _hold(self, first):
        """Quantises the pages from logical page `first` on."""
        if self.bits != 8:
            return
        n = -(-len(self) // self.ps)
        E = np.zeros(self.E.shape[:1] + (n,) + self.E.shape[2:], dtype=np.int64)
        E[:, :min(first, n)] = self.E[:, :min(first, n)]
        for layer in range(self.K.shape[0]):
            for p in range(first, n):
                at = slice(p * self.ps, (p + 1) * self.ps)
                self.K[layer, at], self.V[layer, at], E[layer, p] = quantise(self.K[layer, at], self.V[layer, at])
        self.E = E

    def append(self, k, v):
        if k.shape[1] == 0:
            return
        first = len(self) // self.ps
        self.K, self.V = np.concatenate([self.K, k], 1), np.concatenate([self.V, v], 1)
        self._hold(first)

    def crop(self, tau):
        self.K, self.V = self.K[:, : tau - 1], self.V[:, : tau - 1]
        self.E = self.E[:, : -(-(tau - 1) // self.ps)]

    def evict(self, keep, weights, sinks, recent):
        T = len(self)
        if keep >= T:
            return np.arange(T), weights.copy()
        kept = keep_positions(weights[:T], keep, sinks, recent)
        first = sinks // self.ps
        self.K, self.V = self.K[:, kept], self.V[:, kept]
        self.E = self.E[:, :first]
        self._hold(first)
        w = weights.copy()
        w[:T] = 0
        w[:keep] = weights[kept]
        return kept, w


def keep_positions(w, keep, sinks, recent):
    T = len(w)
    middle = range(sinks, T - recent)
    rank = sorted(middle, key=lambda j: (1, 0, j) if np.isnan(w[j]) else (0, -float(w[j]), j))
    return np.array(sorted(list(range(sinks)) + rank[: keep - sinks - recent] + list(range(T - recent, T))), dtype=np.int64)


def attend(K, V, Q, scale):
    """out fp64 [n][Hq][d], the keys' weights [T], and sum_j w_j |v_j| per output; K, V [T][Hkv][d].  A NaN key makes
    the rows that see it NaN."""
    n, hq, _ = Q.shape
    T, hkv, _ = K.shape
    out, size, w = np.zeros(Q.shape), np.zeros(Q.shape), np.zeros(T)
    for i in range(n):
        t = T - n + i + 1
        for h in range(hq):
            k, v = K[:t, h // (hq // hkv)], V[:t, h // (hq // hkv)]
            s = scale * (k @ Q[i, h])
            p = np.exp(s - s.max())
            p /= p.sum()
            out[i, h] = p @ v
            size[i, h] = p @ np.abs(v)
            w[:t] += p
    return out, w, size
