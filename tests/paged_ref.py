"""Plain references of the paged cache: attention in 64 bits from the
definition, with bounds on what fp32 / bf16 arithmetic may add, and the books
(references, table, lengths) as python lists."""
from __future__ import annotations

import numpy as np


def visible(pos: int, n: int, window: int, sinks: int) -> np.ndarray:
    """which of n keys a query at position pos sees"""
    j = np.arange(n)
    ok = j <= pos
    if window:
        ok &= (j > pos - window) | (j < sinks)
    return ok


def gather(pool: np.ndarray, row, n: int) -> np.ndarray:
    """the first n cached rows of a sequence (fp64); pages that are not there
    read as NaN, so that a key that should not be seen shows"""
    page = pool.shape[1]
    out = np.full((n,) + pool.shape[2:], np.nan)
    for j in range(n):
        p = int(row[j // page]) if j // page < len(row) else -1
        if 0 <= p < pool.shape[0]:
            out[j] = pool[p, j % page]
    return out


def attention(q, k, v, pos0, window=0, sinks=0, scale=None, dtype="bf16"):
    """q [n, hq, d] at positions pos0 .. over k, v [L, hkv, d] (fp64): the
    output and a bound on the error of each element.

    With probabilities off by a factor 1 + e_j each, |e_j| <= e, the quotient
    of the sums is off by at most e / (1 - e) * sum_j p_j |v_j - o| <=
    e (1 + 2 e) (A + |o|), A = sum_j p_j |v_j|.  e holds the rounding of
    p to bf16 (2^-8, bf16 inputs only), the fp32 score (d + 3 roundings of at
    most the sum of the products' magnitudes), the exponent's argument and the
    exponential (2^-20 of the terms that matter: an argument below 64 rounds
    by 2^-18 ln 2 at most), and the accumulation of L terms (L 2^-24).  The
    output's own rounding adds half a step."""
    n, hq, d = q.shape
    L, hkv = k.shape[:2]
    G = hq // hkv
    scale = d ** -0.5 if scale is None else scale
    out, bound = np.zeros((n, hq, d)), np.zeros((n, hq, d))
    half = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    for i in range(n):
        ok = visible(pos0 + i, L, window, sinks)
        if not ok.any():
            continue
        for h in range(hq):
            kk, vv = k[ok, h // G], v[ok, h // G]
            s = kk @ q[i, h] * scale
            p = np.exp(s - s.max())
            p /= p.sum()
            o = p @ vv
            A = p @ np.abs(vv)
            mag = (np.abs(kk) @ np.abs(q[i, h])).max() * scale
            e = (half if dtype == "bf16" else 0.0) + 2 * (d + 3) * 2.0 ** -24 * mag + 2.0 ** -18 + (ok.sum() + 64) * 2.0 ** -24
            out[i, h] = o
            bound[i, h] = e * (1 + 2 * e) * (A + np.abs(o)) + half * (np.abs(o) * (1 + 2 * e) + 2 * e * A) + 1e-30
    return out, bound


class Books:
    """refs, table and ctx, and what the calls do to them"""

    def __init__(self, refs, table, ctx, page):
        self.refs, self.table, self.ctx, self.page = list(refs), [list(r) for r in table], list(ctx), page
        self.flags = 0

    def cols(self, n):
        return -(-n // self.page)

    def free_list(self):
        return [p for p, r in enumerate(self.refs) if r <= 0]

    def reserve(self, add, extra):
        free, at, out, stopped = self.free_list(), 0, [], False
        for b, c in enumerate(self.ctx):
            n = c + (add[b] if add is not None else 0) + extra
            if c < 0 or (add is not None and add[b] < 0) or n > len(self.table[b]) * self.page:
                self.flags |= 256
                out.append(c)
                continue
            need = [x for x in range(self.cols(c), self.cols(n)) if self.table[b][x] < 0]
            if need and (stopped or at + len(need) > len(free)):
                stopped = True
                self.flags |= 128
                out.append(c)
                continue
            for x in need:
                self.table[b][x] = free[at]
                self.refs[free[at]] = 1
                at += 1
            out.append(n)
        return out

    def fork(self, parents, children):
        """returns the page moves (src, dst, rows)"""
        free, at, moves = self.free_list(), 0, []
        table, ctx, refs = [list(r) for r in self.table], list(self.ctx), list(self.refs)
        seen = set()
        for p, c in zip(parents, children):
            first, ok = c not in seen, True
            seen.add(c)
            B = len(ctx)
            if not (0 <= p < B and 0 <= c < B and p != c and first):
                ok = False
            elif not (0 <= ctx[p] <= len(table[p]) * self.page) or ctx[c] != 0 or any(e >= 0 for e in table[c]):
                ok = False
            else:
                used, part = self.cols(ctx[p]), ctx[p] % self.page
                for x in range(used):
                    e = table[p][x]
                    if e >= 0:
                        ok &= e < len(refs) and refs[e] > 0
                    elif x == used - 1 and part:
                        ok = False
            if not ok:
                self.flags |= 256
                continue
            full, part = ctx[p] // self.page, ctx[p] % self.page
            if part and at >= len(free):
                self.flags |= 128
                continue
            for x in range(full):
                self.table[c][x] = table[p][x]
                if table[p][x] >= 0:
                    self.refs[table[p][x]] += 1
            if part:
                self.table[c][full] = free[at]
                self.refs[free[at]] = 1
                moves.append((table[p][full], free[at], part))
                at += 1
            self.ctx[c] = ctx[p]
        return moves

    def _drop(self, b, x):
        e = self.table[b][x]
        if e < 0:
            return
        self.table[b][x] = -1
        if e >= len(self.refs) or self.refs[e] <= 0:
            self.flags |= 64
        else:
            self.refs[e] -= 1

    def free(self, rows):
        for b in rows:
            if not 0 <= b < len(self.ctx):
                self.flags |= 256
                continue
            for x in range(len(self.table[b])):
                self._drop(b, x)
            self.ctx[b] = 0

    def trim(self, window, sinks):
        for b, c in enumerate(self.ctx):
            for x in range(len(self.table[b])):
                last = x * self.page + self.page - 1
                if x * self.page >= sinks and last < c - window:
                    self._drop(b, x)

    def compact(self):
        """returns the page moves and the map"""
        L = sum(r > 0 for r in self.refs)
        holes = [p for p in range(L) if self.refs[p] <= 0]
        late = [p for p in range(L, len(self.refs)) if self.refs[p] > 0]
        to = {p: p for p in range(L) if self.refs[p] > 0}
        to.update(zip(late, holes))
        refs = [0] * len(self.refs)
        for p, q in to.items():
            refs[q] = self.refs[p]
        for row in self.table:
            for x, e in enumerate(row):
                if e >= 0:
                    row[x] = to.get(e, -1)
                    if row[x] < 0:
                        self.flags |= 64
        self.refs = refs
        return [(s, d, self.page) for s, d in zip(late, holes)], [to.get(p, -1) for p in range(len(refs))], L
