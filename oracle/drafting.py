"""Drafted tokens, 4-bit products and cache pages, oracle side (test infrastructure only).

* :func:`verify_row` -- verification of a row's drafted tokens (the rejection rule of
  speculative sampling): d_k is accepted if u_k q(d_k) < p(d_k), the first rejected
  position draws from max(0, p - q), a row whose drafts are all accepted draws from p.
  p and q are the truncated softmax of :mod:`oracle.sampling` (same cutoff, fp64 weights).
* :func:`w4_product` -- x W^T with W = (q - z) s unpacked from 4 bits, in fp64.
* :class:`Pages` -- a paged cache's tables and counts, one page at a time: a page is free
  if its count is 0, and an allocation takes the free page of the lowest number.

Pinned by ``tests/test_oracle_drafting.py`` against closed forms, hand cases, the
identity that emitted tokens are distributed as p whatever the draft, and the invariant
that counts equal the tables' entries.
"""
from __future__ import annotations

import dataclasses
from typing import Optional

import numpy as np

from . import sampling


def probabilities(row32: np.ndarray, temperature: float, min_p: float) -> np.ndarray:
    """softmax(l / T) over the kept set {l >= c}; NaN logits have no weight."""
    row = np.asarray(row32, np.float32)
    top = np.nanmax(row)
    kept = row >= sampling.cutoff32(np.float32(top), temperature, min_p)  # (NaN compares false)
    z = np.where(kept, (np.where(kept, row, 0).astype(np.float64) - float(top)) / float(np.float32(temperature)), -np.inf)
    w = np.exp(z)
    return w / w.sum()


@dataclasses.dataclass
class Verified:
    accepted: int
    token: int
    accept_prob: np.ndarray  # of every drafted position
    near: bool               # a decision was closer than `band` to its threshold


def draw(mass: np.ndarray, u: float, band: float):
    """The smallest index whose cumulative mass exceeds u times the total, and whether rounding may decide it."""
    c = np.cumsum(mass)
    t = float(np.float32(u)) * c[-1]
    i = int(np.argmax(c > t))
    edges = np.abs(c[mass > 0] - t)
    return i, bool(edges.min() <= band * c[-1] or t <= band * c[-1])


def verify_row(target, draft, tokens, greedy: bool, temperature: float, min_p: float, accept_u, draw_u: float,
               band: float = 0.0) -> Verified:
    """``target`` [n + 1, V], ``draft`` [n, V] or None (certain drafts), ``tokens`` [n].  ``band``: how far
    another implementation's probabilities may be off, relative to each."""
    n, vocab = len(tokens), target.shape[1]
    if greedy:
        best = [sampling.greedy_token(np.where(np.isnan(t), -np.inf, t)) for t in target]
        prob = np.array([float(best[k] == tokens[k]) for k in range(n)])
        a = next((k for k in range(n) if not prob[k]), n)
        return Verified(a, best[a], prob, False)
    prob, accepted, near, last = np.zeros(n), n, False, None
    for k in range(n):
        p = probabilities(target[k], temperature, min_p)
        d = int(tokens[k])
        if not 0 <= d < vocab:
            q = np.zeros(vocab)
        elif draft is None:
            q = np.zeros(vocab)
            q[d] = 1.0
        else:
            q = probabilities(draft[k], temperature, min_p)
        pd, qd = (p[d], q[d]) if 0 <= d < vocab else (0.0, 0.0)
        prob[k] = min(1.0, pd / qd) if qd > 0 else float(pd > 0)
        if last is not None:
            continue
        u = float(np.float32(accept_u[k]))
        near = near or (qd > 0 and abs(u * qd - pd) <= 2 * band * max(pd, u * qd) and pd > 0)
        if 0 <= d < vocab and u * qd < pd:
            continue
        accepted = k
        rest = np.maximum(p - q, 0.0) if 0 <= d < vocab else p
        last = rest if rest.sum() > 0 else p
    if last is None:
        last = probabilities(target[n], temperature, min_p)
    token, close = draw(last, draw_u, 4 * band / min(1.0, last.sum()))
    return Verified(accepted, token, prob, near or close)


def w4_unpack(weights: np.ndarray, k: int) -> np.ndarray:
    """uint8 [n, ceil(k / 2)] -> [n, k] whole numbers 0 to 15, the even k in the low half of its byte."""
    out = np.empty((weights.shape[0], 2 * weights.shape[1]), np.int64)
    out[:, 0::2] = weights & 15
    out[:, 1::2] = weights >> 4
    return out[:, :k]


def w4_matrix(weights, scales, zeros, group: int, k: int) -> np.ndarray:
    of = np.arange(k) // group
    z = 8 if zeros is None else np.asarray(zeros, np.int64)[:, of]
    return (w4_unpack(weights, k) - z) * np.asarray(scales, np.float64)[:, of]


def w4_product(x, weights, scales, zeros, group: int) -> np.ndarray:
    x = np.asarray(x, np.float64)
    return x @ w4_matrix(weights, scales, zeros, group, x.shape[1]).T


class Pages:
    """Tables, lengths and counts of a paged cache; ``data`` (any array whose first axis is pages and whose second
    is the 16 slots) stands for the pools."""

    PAGE = 16

    def __init__(self, table, length, refs, data: Optional[np.ndarray] = None):
        self.table, self.length, self.refs = np.array(table), np.array(length), np.array(refs)
        self.data = None if data is None else np.array(data)

    def _take(self):
        for i, c in enumerate(self.refs):
            if c == 0:
                return i
        return -1

    def reserve(self, n_new, active=None):
        """Returns row_ok.  Pages are counted for all rows first, by the counts as they are before the call."""
        rows, cols = self.table.shape
        before, free = self.refs.copy(), int((self.refs == 0).sum())
        wants = []
        for r in range(rows):
            n = int(n_new[r]) if active is None or active[r] else 0
            first, last = int(self.length[r]) // self.PAGE, -(-(int(self.length[r]) + n) // self.PAGE)
            wants.append([j for j in range(first, last if n else first)
                          if self.table[r, j] < 0 or before[self.table[r, j]] > 1])
        ok, used, gone = np.zeros(rows, np.uint8), 0, []
        for r in range(rows):
            used += len(wants[r])
            if (active is not None and not active[r]) or used > free:
                continue
            ok[r] = 1
            for j in wants[r]:
                old, new = int(self.table[r, j]), self._take()
                if old >= 0:
                    keep = int(self.length[r]) % self.PAGE if j == int(self.length[r]) // self.PAGE else 0
                    if self.data is not None:
                        self.data[new, :keep] = self.data[old, :keep]
                    gone.append(old)
                self.table[r, j], self.refs[new] = new, 1
        for old in gone:
            self.refs[old] -= 1
        return ok

    def write(self, values, n_new, rows):
        for r in range(len(rows)):
            for i in range(int(n_new[r]) if rows[r] else 0):
                at = int(self.length[r]) + i
                self.data[self.table[r, at // self.PAGE], at % self.PAGE] = values[r, i]

    def trim(self, length, active=None):
        for r in range(len(self.table)):
            if active is not None and not active[r]:
                continue
            for j in range(-(-int(length[r]) // self.PAGE), self.table.shape[1]):
                if self.table[r, j] >= 0:
                    self.refs[self.table[r, j]] -= 1
                    self.table[r, j] = -1

    def fork(self, parent, child):
        for a, b in zip(parent, child):
            held = -(-int(self.length[a]) // self.PAGE)
            self.table[b] = -1
            self.table[b, :held] = self.table[a, :held]
            self.length[b] = self.length[a]
            for page in self.table[b, :held]:
                self.refs[page] += 1

    def compact(self):
        live = int((self.refs > 0).sum())
        place = {}
        holes = [i for i in range(live) if self.refs[i] == 0]
        for i in range(live, len(self.refs)):
            if self.refs[i] > 0:
                to = holes.pop(0)
                place[i] = to
                self.refs[to], self.refs[i] = self.refs[i], 0
                if self.data is not None:
                    self.data[to] = self.data[i]
        for r, j in np.argwhere(self.table >= live):
            self.table[r, j] = place[int(self.table[r, j])]
        return live
