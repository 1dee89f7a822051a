"""Definitions in 64 bits of the operators of long contexts on a compressed cache, on the CPU: 4-bit values, attention over cached tokens, eviction."""
import numpy as np
import torch

GRID = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=np.float64)


def encode(x):
    """float64 [..., 32 m] -> codes [..., 32 m] (0..15) and scale bytes [..., m]: the nearest value, ties to the even code."""
    g = np.asarray(x, dtype=np.float64).reshape(*x.shape[:-1], -1, 32)
    top = np.abs(g).max(axis=-1)
    bad = ~np.isfinite(top)
    e = np.frexp(np.where(bad | (top == 0), 2.0**-140, top))[1] - 3                  # floor(log2 top) - 2
    e = np.clip(e + (np.where(bad, 0, top) > 7.0 * np.ldexp(1.0, e)), -124, 125)
    y = np.abs(np.where(bad[..., None], 0.0, g)) / np.ldexp(1.0, e)[..., None]
    d = np.abs(y[..., None] - GRID) + np.array([0, 1] * 4) * 1e-12                   # an odd code loses a tie (steps are 0.5 and more)
    code = d.argmin(axis=-1) + 8 * (np.signbit(g) & ~bad[..., None])
    return code.reshape(x.shape), np.where(bad, 255, e + 127).astype(np.uint8)


def decode(code, scale):
    """codes [..., hd] and scale bytes [..., hd / 32] -> float64 [..., hd]"""
    s = np.where(scale == 255, np.nan, np.ldexp(1.0, scale.astype(np.int64) - 127))
    return np.where(code & 8, -1.0, 1.0) * GRID[code & 7] * np.repeat(s, 32, axis=-1)


def unpack(bytes_):
    return np.stack([bytes_ & 15, bytes_ >> 4], axis=-1).reshape(*bytes_.shape[:-1], 2 * bytes_.shape[-1])


class Cache:
    """A pool whose blocks are full of what must never be used: NaN scales, NaN weights, positions from nowhere."""

    def __init__(self, B, blocks, hkv, size, hd, seed, book=True, wide=False):
        r = self.rng = np.random.default_rng(seed)
        shape = (blocks, hkv, size)
        self.hkv, self.size, self.hd, self.blocks = hkv, size, hd, blocks
        self.k, self.v = (r.integers(0, 256, (*shape, hd // 2), dtype=np.uint8) for _ in range(2))
        self.k_scale, self.v_scale = (np.full((*shape, hd // 32), 255, dtype=np.uint8) for _ in range(2))
        self.weight = np.full(shape, np.nan, dtype=np.float32) if book else None
        self.position = np.full(shape, -7, dtype=np.int32) if book else None
        self.free, self.spread = list(r.permutation(blocks)), (110, 135) if wide else (123, 127)

    def request(self, tokens, width, heads=None):
        """A block table [width] whose first `tokens` tokens (of head h only heads[h]) hold something; -1 behind it."""
        need = -(-tokens // self.size)
        table = np.full(width, -1, dtype=np.int32)
        table[:need] = [self.free.pop() for _ in range(need)]
        for h in range(self.hkv):
            t = np.arange(tokens if heads is None else heads[h])
            at = (table[t // self.size], h, t % self.size)
            for s in (self.k_scale, self.v_scale):
                s[at] = self.rng.integers(*self.spread, (len(t), self.hd // 32))
            if self.weight is not None:
                self.weight[at], self.position[at] = self.rng.random(len(t)), t
        return table

    def upload(self, B):
        names = ("k", "v", "k_scale", "v_scale", "weight", "position")
        self.dev = {n: torch.from_numpy(getattr(self, n)).cuda() if getattr(self, n) is not None else None for n in names}
        self.struct = B.kv4_cache_struct(*(self.dev[n] for n in names))
        return self.struct

    def rows(self, which, table, h, t):
        """float64 values of tokens t (array) of head h."""
        at = (table[t // self.size], h, t % self.size)
        return decode(unpack(getattr(self, which)[at]), getattr(self, which + "_scale")[at])


def attention(cache, tables, lens, rows, q, scale):
    """out, lse, and for bounds: sum p |v|, the sums of |q k| of the largest row, the largest |x|; weights per request and head [tokens].
    q float64 [n, hq, hd]; lens [requests][hkv]; rows: (first, count) of each request."""
    hq, hd = q.shape[1:]
    group = hq // cache.hkv
    out, absv, lse = np.zeros(q.shape), np.zeros(q.shape), np.full(q.shape[:2], -np.inf)
    bound, weight = np.zeros((q.shape[0], hq, 2)), []
    for table, ln, (first, count) in zip(tables, lens, rows):
        got = []
        for h in range(cache.hkv):
            total = ln[h] + count
            w = np.zeros(total)
            t = np.arange(total)
            there = (table[t // cache.size] >= 0) & (table[t // cache.size] < cache.blocks) if total else np.zeros(0, bool)
            k, v = np.zeros((total, hd)), np.zeros((total, hd))
            k[there], v[there] = cache.rows("k", table, h, t[there]), cache.rows("v", table, h, t[there])
            for i in range(count):
                seen = there & (t <= ln[h] + i)
                for a in range(group):
                    row = q[first + i, h * group + a]
                    x = np.where(seen, scale * (k @ row), -np.inf)
                    if not seen.any():
                        continue
                    top = x.max()
                    p = np.exp(x - top)
                    norm = p.sum()
                    p = p / norm
                    out[first + i, h * group + a], absv[first + i, h * group + a] = p @ np.where(seen[:, None], v, 0), p @ np.where(seen[:, None], np.abs(v), 0)
                    lse[first + i, h * group + a] = top + np.log(norm)
                    bound[first + i, h * group + a] = abs(scale) * (np.abs(k) @ np.abs(row))[seen].max(), np.abs(x[seen]).max()
                    w += p
            got.append(w)
        weight.append(got)
    return out, lse, absv, bound, weight


def kept(weight, position, exists, budget, n_sink, newest):
    """Token numbers that stay, ascending: first positions, newest, weight; the lower token on ties."""
    def rank(i):
        p = min(max(int(position[i]), 0), 2**30 - 1)
        if not exists[i]:
            return (0, 0.0)
        if position[i] < n_sink:
            return (3, -p)
        if newest is not None and position[i] >= newest:
            return (2, p)
        return (1, float(weight[i]) if weight[i] > 0 else 0.0)
    order = sorted(range(len(weight)), key=lambda i: (*rank(i), -i), reverse=True)
    return sorted(order[:budget])
