"""The 8-bit cache in float64 on the CPU, from its definition: every e4m3 number is tabulated, rounding picks the nearest of them."""
import math

import numpy as np

E_MIN, E_MAX = -117, 119


def _table():
    v = np.full(256, np.nan)
    for code in range(256):
        s, e, m = -1.0 if code & 128 else 1.0, (code >> 3) & 15, code & 7
        if (code & 127) != 127:
            v[code] = s * (m * 2.0 ** -9 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7))
    return v


VALUES = _table()
_POS = VALUES[:127]                                     # ascending
_MID = (_POS[1:] + _POS[:-1]) / 2


def encode(y):
    """Nearest code (ties to the even one), at most 448 in magnitude; what is not finite is NaN (code 127)."""
    y = np.asarray(y, dtype=np.float64)
    a = np.minimum(np.abs(np.where(np.isfinite(y), y, 0.0)), 448.0)
    lo = np.searchsorted(_MID, a, side="left")          # a midpoint itself stays below
    tie = (lo < 126) & (a == _MID[np.minimum(lo, 125)]) & (lo % 2 == 1)
    code = (lo + tie).astype(np.uint8) | np.where(np.signbit(y), 128, 0).astype(np.uint8)
    return np.where(np.isfinite(y), code, 127).astype(np.uint8)


def decode(codes):
    return VALUES[np.asarray(codes)]


def exponent(amax):
    if not amax > 0:
        return E_MIN
    f, x = math.frexp(amax)
    return min(max(x - 9 + (1 if f > 0.875 else 0), E_MIN), E_MAX)


def norm_rotate(x, weight, eps, positions, theta):
    """x [rows][heads][d] float64."""
    d = x.shape[-1]
    if weight is not None:
        x = x / np.sqrt((x ** 2).mean(-1, keepdims=True) + eps) * weight
    if theta:
        a = np.asarray(positions, dtype=np.float64)[:, None] * theta ** (-2.0 * np.arange(d // 2) / d)
        c, s = np.cos(a)[:, None], np.sin(a)[:, None]
        h = d // 2
        x = np.concatenate([x[..., :h] * c - x[..., h:] * s, x[..., h:] * c + x[..., :h] * s], -1)
    return x


class Cache:
    """codes uint8 [pages][heads][2][page][d], exponents int [pages][heads][2], bounds uint8 [pages][heads][2][d]."""

    def __init__(self, n_pages, heads, d, page):
        self.page, self.heads, self.d = page, heads, d
        self.codes = np.zeros((n_pages, heads, 2, page, d), np.uint8)
        self.exps = np.zeros((n_pages, heads, 2), np.int64)
        self.bounds = np.zeros((n_pages, heads, 2, d), np.uint8)

    def append(self, table, start, k, v):
        """Rows k, v [rows][heads][d] (float64, in cache form) into slots start, start + 1, ... of one sequence."""
        n = start + len(k)
        for lp in range(start // self.page, -(-n // self.page) if len(k) else 0):
            a, z = max(start, lp * self.page), min(n, (lp + 1) * self.page)
            pid, kept = table[lp], a - lp * self.page
            for h in range(self.heads):
                for w, src in enumerate((k, v)):
                    x = src[a - start:z - start, h]
                    fin = np.abs(x[np.isfinite(x)])
                    e = exponent(fin.max() if fin.size else 0.0)
                    if kept:
                        old = int(self.exps[pid, h, w])
                        e = max(e, old)
                        if e != old:
                            self.codes[pid, h, w, :kept] = encode(decode(self.codes[pid, h, w, :kept]) * 2.0 ** (old - e))
                    self.exps[pid, h, w] = e
                    self.codes[pid, h, w, kept:kept + z - a] = encode(np.ldexp(x, -e))
                held = np.nan_to_num(decode(self.codes[pid, h, 0, :kept + z - a]), nan=0.0)
                self.bounds[pid, h, 0], self.bounds[pid, h, 1] = encode(held.min(0)), encode(held.max(0))

    def rows(self, table, h, n):
        """Held keys and values [n][d] of a sequence; rows of pages that are not there (id out of range) are left out (mask)."""
        slots = np.arange(n)
        ids = np.asarray(table)[slots // self.page]
        ok = (ids >= 0) & (ids < len(self.codes))
        ids = np.where(ok, ids, 0)
        both = [np.ldexp(decode(self.codes[ids, h, w, slots % self.page]), self.exps[ids, h, w][:, None]) for w in (0, 1)]
        return both[0], both[1], ok

    def attend(self, table, h, q, seen):
        """q [d], seen: slots (ascending).  Returns out [d] and the largest sum of |q_c k_c| (for error bounds), largest |v|."""
        n = int(max(seen)) + 1 if len(seen) else 0
        if n == 0:
            return np.zeros(self.d), 0.0, 0.0
        k, v, ok = self.rows(table, h, n)
        pick = np.zeros(n, bool)
        pick[np.asarray(seen)] = True
        pick &= ok
        if not pick.any():
            return np.zeros(self.d), 0.0, 0.0
        k, v = k[pick], v[pick]
        x = k @ q / math.sqrt(self.d)
        w = np.exp(x - x.max())
        return w @ v / w.sum(), float((np.abs(k) @ np.abs(q)).max()) / math.sqrt(self.d), float(np.abs(v).max())

    def scores(self, table, h, q, m):
        """q [group][d]; scores of the first m pages."""
        plus, minus = np.maximum(q, 0).sum(0), np.minimum(q, 0).sum(0)
        out = []
        for lp in range(m):
            pid = table[lp]
            if not 0 <= pid < len(self.codes):
                out.append(-math.inf)
                continue
            lo, hi = decode(self.bounds[pid, h, 0]), decode(self.bounds[pid, h, 1])
            out.append(math.ldexp(math.fsum(np.concatenate([plus * hi, minus * lo]).tolist()), int(self.exps[pid, h, 0])))
        return out

    def select(self, table, h, q, n_seen, keep, first, recent):
        m = -(-n_seen // self.page) if n_seen > 0 else 0
        if m <= keep:
            return list(range(m)) + [-1] * (keep - m)
        score = self.scores(table, h, q, m)
        must = list(range(first)) + list(range(m - recent, m))
        rest = sorted(range(first, m - recent), key=lambda j: (-score[j], j))[:keep - first - recent]
        return sorted(must + rest)
