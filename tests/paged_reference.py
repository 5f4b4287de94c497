"""The paged 8-bit cache in numpy and 64 bits, written from its definition: one token at a time, one page at a time, explicit
softmax.  Test infrastructure; shares nothing with the library."""
import math

import numpy as np

MIN_EXP = -120


def _e4m3_values():
    v = np.empty(127)
    for c in range(127):
        e, m = c >> 3, c & 7
        v[c] = m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
    return v


E4M3 = _e4m3_values()                       # magnitudes of codes 0 .. 126; 127 is NaN


def decode_e4m3(codes):
    table = np.concatenate([E4M3, [np.nan]])
    return np.where(codes & 128, -1.0, 1.0) * table[codes & 127]


def encode_e4m3(x):
    """Nearest code, ties to the even one; beyond the largest the largest, NaN to NaN."""
    a = np.abs(x)
    hi = np.clip(np.searchsorted(E4M3, a), 1, 126)
    lo = hi - 1
    with np.errstate(invalid="ignore"):
        up = a - E4M3[lo] > E4M3[hi] - a
        tie = a - E4M3[lo] == E4M3[hi] - a
    code = np.where(up | (tie & (hi % 2 == 0)), hi, lo)
    code = np.where(a >= E4M3[126], 126, code)
    code = np.where(np.isnan(x), 127, code)
    return (code | np.where(np.signbit(x), 128, 0)).astype(np.uint8)


def scale_for(x):
    """The smallest power of two under which the largest finite magnitude of x fits."""
    a = np.abs(x[np.isfinite(x)])
    top = a.max() if a.size else 0.0
    if top == 0:
        return 1.0
    e = MIN_EXP
    while top > 448.0 * 2.0 ** e:
        e += 1
    return 2.0 ** e


def slot_of(j, sink, window):
    return j if j < sink else sink + (j - sink) % window


def ring(n, sink, window):
    """{slot: position} after n tokens, one at a time (positions that cannot survive are skipped)."""
    held = {}
    for j in list(range(min(n, sink))) + list(range(max(sink, n - window), n)):
        held[slot_of(j, sink, window)] = j
    return held


def pages_of(n, sink, window, P):
    return -(-min(max(n, 0), sink + window) // P)


class Cache:
    """Pools, scales and table as numpy copies of what the library was given."""

    def __init__(self, sink, window, P, k_codes, v_codes, k_scale, v_scale, table):
        self.sink, self.window, self.P = sink, window, P
        self.codes = [k_codes.copy(), v_codes.copy()]
        self.scale = [k_scale.astype(np.float64), v_scale.astype(np.float64)]
        self.table = table

    def page(self, b, slot):
        p = int(self.table[b, slot // self.P])
        return p if 0 <= p < self.codes[0].shape[0] else -1

    def append(self, b, n0, k, v):
        """k, v [Hkv, t, D]: appended to sequence b behind its n0 tokens."""
        t = k.shape[1]
        if n0 < 0 or t == 0:
            return
        held = ring(n0 + t, self.sink, self.window)
        touched = sorted({s // self.P for s, j in held.items() if j >= n0})
        for lp in touched:
            page = self.page(b, lp * self.P)
            if page < 0:
                continue
            mine = {s - lp * self.P: j for s, j in held.items() if s // self.P == lp}
            at = np.array(sorted(mine))
            pos = np.array([mine[a] for a in at])
            for x, new in enumerate((k, v)):
                for h in range(new.shape[0]):
                    val = decode_e4m3(self.codes[x][page, h, at]) * self.scale[x][page, h]
                    fresh = pos >= n0
                    val[fresh] = new[h, pos[fresh] - n0]
                    s = scale_for(val)
                    self.codes[x][page, h, at] = encode_e4m3(val / s)
                    self.scale[x][page, h] = s

    def rows(self, b, h, n):
        """(positions, K, V) that the cache of sequence b holds after n tokens, in time order, absent pages left out."""
        held = sorted((j, s) for s, j in ring(max(n, 0), self.sink, self.window).items() if self.page(b, s) >= 0)
        pos = np.array([j for j, _ in held], dtype=np.int64)
        out = []
        for x in range(2):
            pg = np.array([self.page(b, s) for _, s in held], dtype=np.int64)
            off = np.array([s % self.P for _, s in held], dtype=np.int64)
            out.append(decode_e4m3(self.codes[x][pg, h, off]) * self.scale[x][pg, h][:, None])
        return pos, out[0], out[1]


def visible(i, pos, sink, window, block):
    near = i // block - pos // block < window // block if block else i - pos < window
    return (pos <= i) & (near | (pos < sink))


def attend(q, k, v, see, scale, weight_round, extra_abs=0.0):
    """One row: (o, lse, tolerance of o, tolerance of lse).

    Tolerances.  A score is a sum of D products in fp32, D / 16 tensor-core steps of which each is off by a few units in the last
    place: |ds| <= 2^-19 scale sum |q k|.  A weight is off by weight_round (half a step of the type it is rounded to), the error
    of its exponential (2^-20) and ds; the sums of n weights or products run in fp32, n / 16 steps and the merges:
    (n / 16 + 64) 2^-23.  o is rounded to bf16 (2^-8).  extra_abs: an absolute error of o."""
    if not see.any():
        return np.zeros(v.shape[1]), -math.inf, np.zeros(v.shape[1]), 0.0
    k, v = k[see], v[see]
    s = (k @ q) * scale
    ds = 2.0 ** -19 * (np.abs(k) @ np.abs(q)) * scale
    m = s.max()
    p = np.exp(s - m)
    l = p.sum()
    o = p @ v / l
    n = len(s)
    chain = (n / 16 + 64) * 2.0 ** -23
    lse = m + math.log(l)
    tol_l = float((p * ds).sum() / l + ds.max()) + chain + 2.0 ** -20 + 2.0 ** -22 * abs(lse)
    tol_o = 2.0 ** -8 * np.abs(o) + (p[:, None] * np.abs(v) * (weight_round + 2.0 ** -20 + chain + 2 * ds.max())).sum(0) / l \
        + np.abs(o) * tol_l + extra_abs
    return o, lse, tol_o, tol_l
