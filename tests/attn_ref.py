"""Plain 64-bit forms of rotary positions, the 4-bit cache and attention, and the pages' tables as
Python lists, with bounds on what float32 arithmetic and one rounding may change."""
import math

import numpy as np

from token_ref import U32, np64, within  # noqa: F401

GRID = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


def quantised(x):
    """The values that a cache holds for x (..., D): blocks of 32 channels, NaN where one has a
    value that is not finite."""
    out = np.zeros(x.shape)
    D = x.shape[-1]
    for lo in range(0, D, 32):
        v = np.asarray(x[..., lo:lo + 32], dtype=np.float64)
        top = np.abs(v).max(-1, keepdims=True)
        fine = np.isfinite(top)
        _, k = np.frexp(np.where(fine, top, 1.0) / 7)       # top / 7 = m 2^k, m in [0.5, 1)
        e = np.where(np.where(fine, top, 1.0) <= 7 * np.ldexp(1.0, k - 1), k - 1, k)
        e = np.clip(np.where(top == 0, -120, e), -120, 125)
        s = np.where(fine, v, 0) / np.ldexp(1.0, e)
        far = np.abs(np.abs(s)[..., None] - GRID)
        # of two as near, the even code
        code = (far + (np.arange(8) % 2) * 1e-9).argmin(-1)
        out[..., lo:lo + 32] = np.where(fine, np.copysign(GRID[code], s) * np.ldexp(1.0, e), np.nan)
    return out


def frequencies(R, base=10000.0, scaling=None):
    how = scaling or {}
    kind = how.get("kind")
    if kind == "base":
        base = base * how["factor"] ** (R / (R - 2))
    f = np.array([base ** (-2 * i / R) for i in range(R // 2)])
    if kind == "linear":
        f = f / how["factor"]
    if kind == "parts":
        k = (how["original"] * f / (2 * math.pi) - how["low"]) / (how["high"] - how["low"])
        k = np.clip(k, 0, 1)
        f = k * f + (1 - k) * f / how["factor"]
    return f


def rotary(x, pos, f, layout, m=1.0):
    """x (B, T, H, D), pos (B, T) -> (value, size of its terms)."""
    R = 2 * len(f)
    y, size = x.copy(), np.zeros(x.shape)
    a = pos[:, :, None, None] * f
    c, s = m * np.cos(a), m * np.sin(a)
    u, w = ((slice(0, R // 2), slice(R // 2, R)) if layout == "half" else
            (slice(0, R, 2), slice(1, R, 2)))
    y[..., u] = x[..., u] * c - x[..., w] * s
    y[..., w] = x[..., w] * c + x[..., u] * s
    size[..., u] = size[..., w] = np.abs(m) * (np.abs(x[..., u]) + np.abs(x[..., w]))
    return y, size


def attend(q, k, v, pos, lo, window, scale):
    """One stream: q (T, H, D) at positions pos (T,), k and v (L, K, D) at 0..L-1 (NaN where the
    stream holds nothing) -> values; their sizes, the largest sum of a score's magnitudes and the
    sum of the values' magnitudes."""
    T, H, D = q.shape
    g = H // k.shape[1]
    y, size, worst, reach = (np.zeros(q.shape) for _ in range(4))
    for t in range(T):
        a = max(lo, pos[t] - window + 1 if window else 0, 0)
        if pos[t] < a:
            continue
        kk, vv = (np.repeat(x[a:pos[t] + 1], g, 1) for x in (k, v))       # (n, H, D)
        s = scale * (kk * q[t]).sum(-1)                                   # (n, H)
        worst[t] = abs(scale) * np.abs(kk * q[t]).sum(-1).max(0)[:, None]
        reach[t] = np.abs(vv).sum(0)
        p = np.exp(s - s.max(0))
        p = p / p.sum(0)
        y[t] = (p[..., None] * vv).sum(0)
        size[t] = (p[..., None] * np.abs(vv)).sum(0)
    return y, (size, worst, reach)


def attend_bound(y, sizes, n, D, u, weights):
    """What may be between an attention's output over n keys and y: its rounding, u; a weight's, `weights`
    (its own and the sum's); the sum of n terms in float32; in a weight the error of
    its score, D + 16 roundings of a sum of magnitudes `worst`, twice (numerator and sum);
    and weights that are multiples of 2^-35 of the largest at most, off by half of that: they are
    16-bit floats, whose least step is 2^-24, and a row's reference, which its largest
    weight is not below, is 2^11."""
    size, worst, reach = sizes
    score = np.minimum((D + 16) * U32 * worst, 300.0)      # past that a weight says nothing
    return (u * np.abs(y) + size * (2 * weights + (n + 64) * U32 + 2 * np.expm1(2 * score))
            + 2.0 ** -36 * reach)


class Streams:
    """Pages and their tables, in Python: what CoPages' calls do, by the same choices."""

    def __init__(self, batch, pages, W, P):
        self.B, self.N, self.W, self.P = batch, pages, W, P
        self.table = [[-1] * W for _ in range(batch)]
        self.tokens, self.first = [0] * batch, [0] * batch
        self.base, self.granted, self.refused = [0] * batch, [0] * batch, [0] * batch

    def refs(self):
        n = [0] * self.N
        for row in self.table:
            for p in row:
                if p >= 0:
                    n[p] += 1
        return n

    def reserve(self, lengths, keep=0):
        P, W = self.P, self.W
        for b in range(self.B):
            to = self.tokens[b] + 1 - keep
            if keep and to > self.first[b]:
                for lp in range(self.first[b] // P, to // P):
                    self.table[b][lp % W] = -1
                self.first[b] = to
        refs = self.refs()
        free = [p for p in range(self.N) if refs[p] == 0]
        asked = 0
        self.base = list(self.tokens)
        plans = []
        for b in range(self.B):
            base, n = self.base[b], lengths[b]
            if n and (base + n - 1) // P - self.first[b] // P >= W:
                self.refused[b] += n
                n = 0
            new = []
            for lp in range(base // P, (base + n - 1) // P + 1) if n else ():
                p = self.table[b][lp % W]
                if p < 0 or refs[p] > 1:
                    new.append((lp % W, asked))
                    asked += 1
            if new and asked > len(free):
                self.refused[b] += n
                n, new = 0, []
            self.granted[b] = n
            plans.append(new)
        for b, new in enumerate(plans):
            for slot, rank in new:
                self.table[b][slot] = free[rank]
            self.tokens[b] = self.base[b] + self.granted[b]

    def truncate(self, lengths):
        P, W = self.P, self.W
        for b in range(self.B):
            to = min(self.tokens[b], max(lengths[b], 0))
            oldest = self.first[b] // P
            for k in range(W):
                if to <= self.first[b] or (oldest + k) * P >= to:
                    self.table[b][(oldest + k) % W] = -1
            self.first[b] = min(self.first[b], to)
            self.tokens[b] = to
        self.base, self.granted = list(self.tokens), [0] * self.B

    def select(self, source):
        self.truncate(self.tokens)                  # what lies past the ends
        pick = [s if 0 <= s < self.B else None for s in source]
        rows, tokens, first = self.table, self.tokens, self.first
        self.table = [[-1] * self.W if s is None else list(rows[s]) for s in pick]
        self.tokens = [0 if s is None else tokens[s] for s in pick]
        self.first = [0 if s is None else first[s] for s in pick]
        self.base, self.granted = list(self.tokens), [0] * self.B

    def compact(self):
        refs = self.refs()
        used = sum(r > 0 for r in refs)
        to = [p for p in range(used) if refs[p] == 0]
        name = dict(zip([p for p in range(used, self.N) if refs[p] > 0], to))
        self.table = [[name.get(p, p) for p in row] for row in self.table]
