"""Reference of the operators around a paged key/value cache.

TEST INFRASTRUCTURE ONLY: plain numpy in fp64, written from the definitions in
include/wq4_attn.h; the library never calls it and shares no code with it.

Sequence b owns rows [starts[b], starts[b + 1]) of a batch of prompts, the last
ones of its lens[b] tokens; a decode step is one row a sequence.  The row at
position i sees token t when

    t <= i  and  (window == 0 or t > i - window or t < sinks),

and o = sum_t softmax(scale q.K_t) V_t over what it sees, 0 where that is nothing.
"""
from __future__ import annotations

import numpy as np

from . import double_to_half, half_to_double, rope


def ulp16(v) -> np.ndarray:
    """Distance of fp16 values of v's size (normal and subnormal)."""
    v = np.maximum(np.abs(np.asarray(v, np.float64)), 2.0 ** -14)
    return np.where(np.isfinite(v), 2.0 ** (np.floor(np.log2(np.where(np.isfinite(v), v, 1.0))) - 10), 0.0)


def attention_tolerance(o, A) -> np.ndarray:
    """The contract of the attention calls: 2e-3 * sum_t p_t |V_t| + ulp16(|o|)."""
    return 2e-3 * np.asarray(A) + ulp16(o)


def seen(pos: int, T: int, window: int, sinks: int) -> np.ndarray:
    """Which of the tokens 0 .. T-1 the row at `pos` sees."""
    t = np.arange(T)
    ok = t <= pos
    if window:
        ok &= (t > pos - window) | (t < sinks)
    return ok


def attention(q, k, v, table, starts, lens, scale: float, n_q_heads: int, window: int = 0, sinks: int = 0):
    """fp16 bits q [rows][>= n_q_heads * D], caches [pages][n_kv][P][D], table [batch][stride]; returns
    (o, A) fp64 [rows][n_q_heads][D], A = sum_t p_t |V_t|, and which rows a sequence owns."""
    _, n_kv, P, D = k.shape
    G, rows = n_q_heads // n_kv, q.shape[0]
    o, A = np.zeros((rows, n_q_heads, D)), np.zeros((rows, n_q_heads, D))
    owned = np.zeros(rows, bool)
    for b, T in enumerate(lens):
        n = starts[b + 1] - starts[b]
        for r in range(starts[b], starts[b + 1]):
            owned[r] = True
            pos = T - n + r - starts[b]
            t = np.flatnonzero(seen(pos, max(T, 0), window, sinks))
            if t.size == 0:
                continue
            page = table[b][t // P]
            assert np.all((page >= 0) & (page < k.shape[0])), "a seen token without a page"
            for h in range(n_kv):
                K, V = half_to_double(k[page, h, t % P]), half_to_double(v[page, h, t % P])
                Q = half_to_double(np.ascontiguousarray(q[r, h * G * D:(h + 1) * G * D])).reshape(G, D)
                with np.errstate(invalid="ignore"):
                    s = scale * (Q @ K.T)
                    e = np.exp(s - s.max(1, keepdims=True))
                    p = e / e.sum(1, keepdims=True)
                    o[r, h * G:(h + 1) * G] = p @ V
                    A[r, h * G:(h + 1) * G] = p @ np.abs(V)
    return o, A, owned


def append(qkv, k, v, table, starts, lens, n_q_heads: int, theta: float):
    """Rotated queries in fp64 [rows][n_q_heads * D], and the caches as fp64 copies with the rows'
    rotated keys and (unrotated) values at their places; rows without a place write nothing."""
    _, n_kv, P, D = k.shape
    H, K = n_q_heads * D, n_kv * D
    q_out = np.zeros((qkv.shape[0], H))
    k64, v64 = half_to_double(k), half_to_double(v)
    for b, T in enumerate(lens):
        n = starts[b + 1] - starts[b]
        for r in range(starts[b], starts[b + 1]):
            pos = T - n + r - starts[b]
            row = np.ascontiguousarray(qkv[r:r + 1, :H + K])
            turned = rope(row, [max(pos, 0)], D, theta)[0][0] if theta else half_to_double(row)[0]
            q_out[r] = turned[:H]
            page = table[b][pos // P] if 0 <= pos < table.shape[1] * P else -1
            if 0 <= page < k.shape[0]:
                k64[page, :, pos % P] = turned[H:].reshape(n_kv, D)
                v64[page, :, pos % P] = half_to_double(np.ascontiguousarray(qkv[r, H + K:H + 2 * K])).reshape(n_kv, D)
    return q_out, k64, v64


class Pool:
    """The bookkeeping of a page pool, one page and one sequence at a time.  caches: arrays whose first
    axis is the page (a layer's keys or values, [pages][heads][P][D]).  `refused` counts what a call
    left undone."""

    def __init__(self, num_pages, max_seqs, stride, P, caches=()):
        self.table = np.full((max_seqs, stride), -1, np.int32)
        self.lens = np.zeros(max_seqs, np.int32)
        self.refs = np.zeros(num_pages, np.int32)
        self.P, self.caches, self.refused = P, list(caches), 0

    def pages(self, T):
        return -(-T // self.P)

    def _take(self):
        free = np.flatnonzero(self.refs == 0)
        return int(free[0]) if free.size else -1

    def _drop(self, s, j):
        e = int(self.table[s, j])
        if e >= 0:
            self.table[s, j] = -1
            self.refs[e] -= 1

    def _in(self, s):
        return 0 <= s < len(self.lens)

    def reserve(self, seqs, new_lens):
        done, stuck = set(), False
        for s, L in zip(seqs, new_lens):
            if not self._in(s) or s in done or not self.lens[s] <= L <= self.table.shape[1] * self.P:
                self.refused += 1
                if self._in(s):
                    done.add(s)
                continue
            done.add(s)
            old, new = self.pages(int(self.lens[s])), self.pages(int(L))
            if new > old and (stuck or new - old > np.count_nonzero(self.refs == 0)):
                stuck = True
                self.refused += 1
                continue
            for j in range(old, new):
                p = self._take()
                self.table[s, j], self.refs[p] = p, 1
            self.lens[s] = L

    def free(self, seqs):
        for s in seqs:
            if not self._in(s):
                self.refused += 1
                continue
            for j in range(self.table.shape[1]):
                self._drop(s, j)
            self.lens[s] = 0

    def trim(self, seqs, window, sinks):
        for s in seqs:
            if not self._in(s):
                self.refused += 1
                continue
            T = int(self.lens[s])
            for j in range(self.table.shape[1]):
                tokens = range(j * self.P, (j + 1) * self.P)
                if not any(t < sinks or t > T - window for t in tokens):
                    self._drop(s, j)

    def fork(self, parents, children):
        pairs = [(p, c) for p, c in zip(parents, children)]
        ranged = [self._in(p) and self._in(c) for p, c in pairs]
        are_parents = {p for (p, _), ok in zip(pairs, ranged) if ok}
        done, todo = set(), []
        for (p, c), ok in zip(pairs, ranged):
            if not ok or c in done or c in are_parents:
                self.refused += 1
            else:
                todo.append((p, c))
            if ok:
                done.add(c)
        for _, c in todo:
            for j in range(self.table.shape[1]):
                self._drop(c, j)
        taken = []
        for p, c in todo:                      # the pages of their own first, lowest free ones in order
            T = int(self.lens[p])
            last = T // self.P
            own = None
            if T % self.P and self.table[p, last] >= 0:
                own = self._take()
                if own >= 0:
                    self.refs[own] = 1
            taken.append(own)
        for (p, c), own in zip(todo, taken):
            T = int(self.lens[p])
            if own is not None and own < 0:
                self.refused += 1
                self.lens[c] = 0
                continue
            for j in range(self.pages(T)):
                e = int(self.table[p, j])
                if own is not None and j == T // self.P:
                    for a in self.caches:
                        a[own, :, :T % self.P] = a[e, :, :T % self.P]
                    e = own
                elif e >= 0:
                    self.refs[e] += 1
                self.table[c, j] = e
            self.lens[c] = T

    def compact(self):
        m = int(np.count_nonzero(self.refs > 0))
        movers = [p for p in range(m, len(self.refs)) if self.refs[p] > 0]
        holes = [p for p in range(m) if self.refs[p] == 0]
        for s, d in zip(movers, holes):
            for a in self.caches:
                a[d] = a[s]
            self.refs[d], self.refs[s] = self.refs[s], 0
            self.table[self.table == s] = d

    def copy_pages(self, src, dst):
        n = len(self.refs)
        good = [(s, d) for s, d in zip(src, dst) if 0 <= s < n and 0 <= d < n]
        for s, d in zip(src, dst):
            twice = sum(1 for _, e in good if e == d) > 1
            read = any(0 <= s < n and e == s for _, e in good)
            if (s, d) not in good or twice or read:
                self.refused += 1
        ok = [(s, d) for s, d in good if sum(1 for _, e in good if e == d) == 1 and not any(e == s for _, e in good)]
        for a in self.caches:
            for s, d in ok:
                a[d] = a[s]
