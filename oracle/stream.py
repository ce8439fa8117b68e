"""The operators of long-running streams in float64 numpy, from their definitions.

Window attention with sinks, rotary positions with several axes, products with 4-bit weights, and the book-keeping of
pages (tables, forks, growth, trimming, compaction) as plain dictionaries and sorted lists.
"""
from __future__ import annotations

import numpy as np

PAGE = 16


def visible(p: int, t: int, window: int, sinks: int) -> bool:
    """Whether a row at position p sees token t."""
    return t <= p and (t > p - window or t < sinks)


def window_attention(q, K, V, first: int, window: int, sinks: int):
    """q [n, Hq, dh] of one sequence, row j at position first + j; K, V [L, Hkv, dh], L = first + n.

    Returns (out, weight): out [n, Hq, dh], zeros where a row sees nothing, and weight [n, Hq, dh], the same sum over
    |V|, which bounds what rounding the probabilities can change.  Values that no row sees take no part (they may be NaN).
    """
    q = np.asarray(q, dtype=np.float64)
    n, hq, dh = q.shape
    grp = hq // K.shape[1]
    out, weight = np.zeros((n, hq, dh)), np.zeros((n, hq, dh))
    p, t = first + np.arange(n)[:, None], np.arange(len(K))[None, :]
    see = (t <= p) & ((t > p - window) | (t < sinks))
    some, rows = see.any(axis=0), see.any(axis=1)
    K, V, see = K[some].astype(np.float64), V[some].astype(np.float64), see[:, some]
    for h in range(hq if rows.any() else 0):
        s = np.where(see, q[:, h] @ K[:, h // grp].T / np.sqrt(dh), -np.inf)[rows]
        e = np.exp(s - s.max(axis=1, keepdims=True))
        e /= e.sum(axis=1, keepdims=True)
        out[rows, h] = e @ V[:, h // grp]
        weight[rows, h] = e @ np.abs(V[:, h // grp])
    return out, weight


def rope_axes(v, positions, axis_of_pair, theta: float):
    """v [n, heads, dh]; positions [n_axes, n]; pair (i, i + dh/2) turned by positions[axis_of_pair[i]] theta^(-2i/dh)."""
    v = np.asarray(v, dtype=np.float64)
    half = v.shape[-1] // 2
    freq = float(theta) ** (-2.0 * np.arange(half) / v.shape[-1])
    angle = np.asarray(positions, dtype=np.float64)[np.asarray(axis_of_pair)].T * freq        # [n, half]
    z = (v[..., :half] + 1j * v[..., half:]) * np.exp(1j * angle)[:, None, :]
    return np.concatenate([z.real, z.imag], axis=-1)


def w4_linear(x, w, scales, zeros=None):
    """x [m, k], w [n, k] in 0 .. 15, scales and zeros [n, groups] -> [m, n]."""
    group = w.shape[1] // max(1, scales.shape[1])
    z = np.full(scales.shape, 8.0) if zeros is None else np.asarray(zeros, dtype=np.float64)
    full = (w - np.repeat(z, group, axis=1)) * np.repeat(np.asarray(scales, dtype=np.float64), group, axis=1)
    return np.asarray(x, dtype=np.float64) @ full.T


class Pages:
    """Tables as lists, references counted anew whenever they are asked for."""

    def __init__(self, n_pages: int):
        self.n_pages = n_pages
        self.seqs = {}                       # id -> [tokens, table]

    def refs(self, page):
        return sum(t.count(page) for _, t in self.seqs.values())

    def free_pages(self):
        named = {p for _, t in self.seqs.values() for p in t}
        return [p for p in range(self.n_pages) if p not in named]

    def _ids(self, n):
        out, i = [], 0
        while len(out) < n:
            if i not in self.seqs:
                out.append(i)
            i += 1
        return out

    def open(self, n):
        ids = self._ids(n)
        for i in ids:
            self.seqs[i] = [0, []]
        return ids

    def fork(self, parents, children):
        ids = self._ids(len(parents) * children)
        for k, i in enumerate(ids):
            tokens, table = self.seqs[parents[k // children]]
            self.seqs[i] = [tokens, list(table)]
        return ids

    def extend(self, ids, tokens):
        """(src, dst) pairs, or None where there are too few pages (and nothing is changed)."""
        before = {i: [t, list(table)] for i, (t, table) in self.seqs.items()}
        pairs = []
        for i, more in zip(ids, tokens):
            s = self.seqs[i]
            if more and s[0] % PAGE and self.refs(s[1][-1]) > 1:
                free = self.free_pages()
                if not free:
                    self.seqs = before
                    return None
                pairs.append((s[1][-1], free[0]))
                s[1][-1] = free[0]
            s[0] += more
            while len(s[1]) * PAGE < s[0]:
                free = self.free_pages()
                if not free:
                    self.seqs = before
                    return None
                s[1].append(free[0])
        return pairs

    def trim(self, ids, window, sinks):
        for i in ids:
            tokens, table = self.seqs[i]
            for k in range(len(table)):
                inside = range(PAGE * k, PAGE * k + PAGE)
                if PAGE * k + PAGE <= tokens and not any(visible(p, t, window, sinks) for t in inside for p in (tokens, tokens + 1, tokens + window + PAGE)):
                    table[k] = -1

    def free(self, ids):
        for i in ids:
            del self.seqs[i]

    def compact(self):
        live = sorted({p for _, t in self.seqs.values() for p in t if p >= 0})
        holes = [p for p in range(len(live)) if p not in live]
        moves = list(zip([p for p in live if p >= len(live)], holes))
        to = dict(moves)
        for s in self.seqs.values():
            s[1] = [to.get(p, p) for p in s[1]]
        return moves, len(live)
