"""Plain float64 NumPy forms of the 8-bit cache, the attention over it and the
page pool, written from their definitions (test infrastructure only)."""
from __future__ import annotations

import numpy as np


# ---- e4m3 -----------------------------------------------------------------
def code_values() -> np.ndarray:
    """The value of every e4m3 code 0..255 (0x7F and 0xFF: NaN)."""
    c = np.arange(256)
    e, m = (c >> 3) & 15, c & 7
    v = np.where(e == 0, m * 2.0 ** -9, (1 + m / 8.0) * 2.0 ** (e - 7.0))
    v = np.where(c & 128, -v, v)
    v[[127, 255]] = np.nan
    return v


VALUES = code_values()


def to_codes(x) -> np.ndarray:
    """Nearest code, ties to even; what is not finite is NaN.  |x| <= 448."""
    x = np.asarray(x, np.float64)
    a = np.abs(x)
    fin = np.isfinite(x)
    pos = VALUES[:127]
    i = np.clip(np.searchsorted(pos, np.where(fin, a, 0)), 1, 126)
    lo, hi = pos[i - 1], pos[i]
    mid = (lo + hi) / 2
    a0 = np.where(fin, a, 0)
    up = (a0 > mid) | ((a0 == mid) & (i % 2 == 0))
    c = np.where(up, i, i - 1)
    c = np.where(np.signbit(x), c + 128, c)
    return np.where(fin, c, 127).astype(np.uint8)


def exponent(x, new) -> int:
    """The least e >= -126 with |x| <= 448 * 2^e over finite new values."""
    v = np.abs(np.asarray(x, np.float64)[new])
    v = v[np.isfinite(v)]
    top = v.max() if v.size else 0.0
    e = -126
    while top > 448.0 * 2.0 ** e:
        e += 1
    return e


def store_block(x, codes, ebyte, t0, t1):
    """One page and head: x, codes [16][hd]; slots t0..t1-1 of x are stored,
    slots below t0 are held.  Returns (codes, scale byte)."""
    x = np.asarray(x, np.float64)
    new = np.zeros(x.shape, bool)
    new[t0:t1] = True
    e = exponent(x, new)
    out = codes.copy()
    if t0 > 0:
        was = int(ebyte) - 127
        if was > e:
            e = was
        if e > was:
            out[:t0] = to_codes(VALUES[codes[:t0]] * 2.0 ** (was - e))
    out[t0:t1] = to_codes(x[t0:t1] * 2.0 ** -e)
    return out, e + 127


# ---- layouts --------------------------------------------------------------
def v_to_page(v):
    """[16][hd] -> the stored order of a V page [4][16][hd/16][4]."""
    hd = v.shape[1]
    return v.reshape(4, 4, hd // 16, 16).transpose(0, 3, 2, 1).reshape(-1)


def v_from_page(p, hd):
    return p.reshape(4, 16, hd // 16, 4).transpose(0, 3, 2, 1).reshape(16, hd)


def page_values(codes, ebyte, hd, is_v):
    """[16][hd] values of a stored page and head."""
    c = v_from_page(codes, hd) if is_v else codes.reshape(16, hd)
    return VALUES[c] * 2.0 ** (int(ebyte) - 127.0)


def entries(codes, exps, table, n, hd, is_v):
    """Entries 0..n-1 of a sequence, [n][Hkv][hd]: codes [pages][Hkv][16 hd],
    exps [pages][Hkv], table the sequence's page-table row."""
    hkv = codes.shape[1]
    out = np.zeros((n, hkv, hd))
    for p in range((n + 15) // 16):
        pg = int(table[p])
        m = min(16, n - 16 * p)
        for h in range(hkv):
            out[16 * p:16 * p + m, h] = page_values(codes[pg, h], exps[pg, h], hd,
                                                    is_v)[:m]
    return out


# ---- attention ------------------------------------------------------------
def attend_row(q, k, v, see):
    """One query head over keys/values [n][hd] under a mask: the output, the
    mean of |v| under the same weights, and the largest sum |q_i k_i|."""
    hd = q.shape[0]
    idx = np.nonzero(see)[0]
    if idx.size == 0:
        return np.zeros(hd), np.zeros(hd), 0.0
    with np.errstate(invalid="ignore", over="ignore"):
        k, v = k[idx], v[idx]
        z = k @ q / np.sqrt(hd)
        p = np.exp(z - z.max())
        p /= p.sum()
        return p @ v, p @ np.abs(v), (np.abs(k) @ np.abs(q)).max() / np.sqrt(hd)


# ---- page pool ------------------------------------------------------------
class PoolRef:
    """The pool's state and calls, one step at a time."""

    def __init__(self, max_seqs, max_pages, n_pages):
        self.table = np.zeros((max_seqs, max_pages), np.int64)
        self.held = np.zeros(max_seqs, np.int64)
        self.refs = np.zeros(n_pages, np.int64)
        self.refused = 0

    def _take(self):
        free = np.nonzero(self.refs == 0)[0]
        if free.size == 0:
            return None
        self.refs[free[0]] = 1
        return int(free[0])

    def grow(self, length, extra=0):
        for s, n in enumerate(length):
            want = (max(0, int(n) + extra) + 15) // 16
            short = want > self.table.shape[1]
            want = min(want, self.table.shape[1])
            while self.held[s] < want:
                p = self._take()
                if p is None:
                    short = True
                    break
                self.table[s, self.held[s]] = p
                self.held[s] += 1
            self.refused += short

    def release(self, seqs):
        for s in seqs:
            for j in range(self.held[s]):
                self.refs[self.table[s, j]] -= 1
            self.held[s] = 0

    def fork(self, parents, children, length):
        """Returns the copies [(source page, target page)]."""
        self.release(children)
        cuts = [min(max(int(length[a]), 0), int(self.held[a]) * 16) for a in parents]
        copies = []
        for a, b, n in zip(parents, children, cuts):
            for j in range(n // 16):
                self.table[b, j] = self.table[a, j]
                self.refs[self.table[a, j]] += 1
            self.held[b] = n // 16
            if n % 16:
                p = self._take()
                if p is None:
                    self.refused += 1
                    continue
                self.table[b, n // 16] = p
                self.held[b] += 1
                copies.append((int(self.table[a, n // 16]), p))
        return copies

    def compact(self):
        live = np.nonzero(self.refs > 0)[0]
        n = live.size
        src = live[live >= n]
        dst = np.nonzero(self.refs[:n] == 0)[0]
        to = np.arange(self.refs.size)
        to[src] = dst
        for s in range(self.table.shape[0]):
            h = self.held[s]
            self.table[s, :h] = to[self.table[s, :h]]
        self.refs[dst] = self.refs[src]
        self.refs[src] = 0
        return list(zip(src.tolist(), dst.tolist()))
