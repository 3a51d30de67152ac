"""The 4-bit paged cache in 64 bits, from its definitions (test infrastructure).

Values: 16 neighbours along the head share a scale s = e4m3(a / (6 * 2^e)), a their largest
magnitude, to the nearest (ties to even), at least 2^-9 and at most 448; each is the nearest
of +-(0, 0.5, 1, 1.5, 2, 3, 4, 6) to x / (s * 2^e), ties to the even code, saturating. NaN is
held as 0, an infinity as the block's largest code, counted as the largest finite bf16.

Pages: plain lists; new pages are the free ones of the lowest number, in list order.
"""
from __future__ import annotations

import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
E4M3 = np.array(sorted({m * 2.0 ** -9 for m in range(8)} |
                       {(1 + m / 8) * 2.0 ** e for e in range(-6, 9) for m in range(8) if not (e == 8 and m == 7)}))
BF16_MAX = 255 / 128 * 2.0 ** 127


def nearest(x: np.ndarray, values: np.ndarray) -> np.ndarray:
    """Index of the nearest of the ascending values (x at most the last); ties to the even index."""
    up = np.clip(np.searchsorted(values, x), 0, len(values) - 1)
    down = np.maximum(up - 1, 0)
    a, b = x - values[down], values[up] - x
    return np.where((b < a) | ((a == b) & (up % 2 == 0)), up, down)


def quantise(x: np.ndarray, exponent: int = 0):
    """Values held for x [..., D], their codes and their blocks' scales."""
    x = np.asarray(x, dtype=np.float64)
    x = np.clip(np.where(np.isnan(x), 0.0, x), -BF16_MAX, BF16_MAX)
    b = x.reshape(*x.shape[:-1], -1, 16) * 2.0 ** -exponent
    want = np.minimum(np.abs(b).max(-1, keepdims=True) / 6, 448.0)
    s = np.maximum(E4M3[nearest(want, E4M3)], 2.0 ** -9)
    code = nearest(np.minimum(np.abs(b) / s, 6.0), GRID)
    v = np.sign(b) * GRID[code] * s * 2.0 ** exponent
    return v.reshape(x.shape), code.reshape(x.shape), s[..., 0]


def attend(q, k, v, causal=False, scale=None, base=None, base_lse=None):
    """One sequence and key head: q [queries, group, D], k, v [tokens, D]. Returns out [queries, group, D],
    lse [group, queries], and for error bounds sum_j p_j |v_j| (as out) and max_j scale sum_d |q_d k_jd|."""
    nq, r, D = q.shape
    n = k.shape[0]
    scale = 1 / np.sqrt(D) if scale is None else scale
    out, mag = np.zeros((nq, r, D)), np.zeros((nq, r, D))
    lse = np.full((r, nq), -np.inf)
    big = 0.0
    for i in range(nq):
        m = max(0, n - nq + 1 + i) if causal else n
        if m:
            z = scale * (q[i] @ k[:m].T)
            big = max(big, scale * (np.abs(q[i]) @ np.abs(k[:m]).T).max())
            top = z.max(-1, keepdims=True)
            p = np.exp(z - top)
            total = p.sum(-1, keepdims=True)
            out[i], mag[i] = p / total @ v[:m], p / total @ np.abs(v[:m])
            lse[:, i] = (top + np.log(total))[:, 0]
    if base is not None:
        with np.errstate(invalid="ignore"):
            both = np.logaddexp(lse, base_lse)
            a, b = (np.where(np.isneginf(both), 0.0, np.exp(x - both)).T[..., None] for x in (lse, base_lse))
        out, mag, lse = a * out + b * base, a * mag + b * np.abs(base), both
    return out, lse, mag, big


class Full(Exception):
    """No page left, or a table is too short."""


class Pages:
    """Tables, lengths and the pages' data (one value a page and layer stands for its bytes)."""

    def __init__(self, pages, sequences, page_tokens, sequence_pages, data=None):
        self.n, self.P, self.W = pages, page_tokens, sequence_pages
        self.table = [[] for _ in range(sequences)]
        self.lengths = [0] * sequences
        self.data = list(range(pages)) if data is None else data  # data[page]: where its bytes came from

    def refs(self):
        r = [0] * self.n
        for row in self.table:
            for p in row:
                r[p] += 1
        return r

    def free(self):
        return [p for p, x in enumerate(self.refs()) if x == 0]

    def need(self, tokens):
        return -(-tokens // self.P)

    def grow(self, seqs, counts):
        refs, free = self.refs(), self.free()
        plan = []
        for s, c in zip(seqs, counts):
            n = self.lengths[s]
            if self.need(n + c) > self.W:
                raise Full
            copied = c > 0 and n % self.P > 0 and refs[self.table[s][-1]] > 1
            k = self.need(n + c) - self.need(n) + copied
            if k > len(free):
                raise Full
            plan.append((s, c, copied, free[:k]))
            free = free[k:]
        for s, c, copied, new in plan:
            if copied:
                self.data[new[0]] = self.data[self.table[s][-1]]
                self.table[s][-1] = new[0]
                new = new[1:]
            self.table[s] += new
            self.lengths[s] += c

    def fork(self, src, dst, lengths=None, copy=False):
        free, plan = self.free(), []
        for i, (s, d) in enumerate(zip(src, dst)):
            n = self.lengths[s] if lengths is None else min(self.lengths[s], lengths[i])
            row = self.table[s][:self.need(n)]
            if copy:
                if len(row) > len(free):
                    raise Full
                for a, b in zip(row, free):
                    plan.append(("data", b, self.data[a]))
                row, free = free[:len(row)], free[len(row):]
            plan.append(("row", d, (list(row), n)))
        for what, at, x in plan:
            if what == "data":
                self.data[at] = x
            else:
                self.table[at], self.lengths[at] = x

    def truncate(self, seqs, lengths=None):
        for i, s in enumerate(seqs):
            self.lengths[s] = min(self.lengths[s], lengths[i] if lengths is not None else 0)
            self.table[s] = self.table[s][:self.need(self.lengths[s])]

    def compact(self):
        refs = self.refs()
        live = sum(x > 0 for x in refs)
        to = dict(zip((p for p in range(live, self.n) if refs[p]), (p for p in range(live) if not refs[p])))
        for a, b in to.items():
            self.data[b] = self.data[a]
        self.table = [[to.get(p, p) for p in row] for row in self.table]

    def table_array(self):
        t = np.full((len(self.table), self.W), -1, dtype=np.int32)
        for s, row in enumerate(self.table):
            t[s, :len(row)] = row
        return t
