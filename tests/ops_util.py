"""Plain 64-bit forms of the rotate-and-store and page operators, shared by their tests."""

from __future__ import annotations

import numpy as np

FP8_MAX = 448.0


def pages_of(tokens, page):
    return -(-int(tokens) // page)


def rotated(x, weight, eps, cos_sin, positions, interleaved):
    """x [rows, heads, d] float64 -> (z, bound): the normalised and rotated heads, and the sum of the magnitudes that
    each element is made of (|y_a c| + |y_b s|, or |y|)."""
    x = np.asarray(x, dtype=np.float64)
    rows, _, d = x.shape
    if weight is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * np.asarray(weight, dtype=np.float64)
    z, size = x.copy(), np.abs(x)
    rot = cos_sin.shape[1]
    if rot == 0:
        return z, size
    at = np.asarray(cos_sin, dtype=np.float64)[np.clip(positions, 0, cos_sin.shape[0] - 1)]
    for r in range(rows):
        c, s = at[r, :rot // 2], at[r, rot // 2:]
        for j in range(rot // 2):
            a, b = (2 * j, 2 * j + 1) if interleaved else (j, j + rot // 2)
            z[r, :, a] = x[r, :, a] * c[j] - x[r, :, b] * s[j]
            z[r, :, b] = x[r, :, b] * c[j] + x[r, :, a] * s[j]
            size[r, :, a] = np.abs(x[r, :, a] * c[j]) + np.abs(x[r, :, b] * s[j])
            size[r, :, b] = np.abs(x[r, :, b] * c[j]) + np.abs(x[r, :, a] * s[j])
    return z, size


class PagesModel:
    """The page operators on host lists, one page at a time; pools are numpy arrays [layers, P, page, heads, d]."""

    def __init__(self, rows, width, num_pages, page, max_ctx, k=None, v=None):
        self.table = [[-1] * width for _ in range(rows)]
        self.ctx = [0] * rows
        self.counts = [0] * num_pages
        self.page, self.max_ctx, self.k, self.v = page, max_ctx, k, v

    def _take(self, need):
        free = [p for p, c in enumerate(self.counts) if c == 0]
        if need > len(free):
            return None, need - len(free)
        return free[:need], 0

    def _drop(self, page):
        if 0 <= page < len(self.counts):
            self.counts[page] -= 1

    def reserve(self, add):
        need, plan = 0, []
        for r, a in enumerate(add):
            if a < 0 or not 0 <= self.ctx[r] <= self.max_ctx or self.ctx[r] + a > self.max_ctx:
                continue
            first, last = pages_of(self.ctx[r], self.page), pages_of(self.ctx[r] + a, self.page)
            plan.append((r, a, first, last))
            need += last - first
        got, missing = self._take(need)
        if missing:
            return missing
        for r, a, first, last in plan:
            for i in range(first, last):
                self.table[r][i] = got.pop(0)
                self.counts[self.table[r][i]] = 1
            self.ctx[r] += a
        return 0

    def fork(self, parents, children):
        plan = []
        for i, (f, c) in enumerate(zip(parents, children)):
            if not (0 <= f < len(self.ctx) and 0 <= c < len(self.ctx)) or f == c or self.ctx[c] != 0:
                continue
            if c in children[:i]:
                continue
            if 0 <= self.ctx[f] <= self.max_ctx:
                plan.append((f, c))
        got, missing = self._take(sum(self.ctx[f] % self.page != 0 for f, _ in plan))
        if missing:
            return missing
        lens = {f: self.ctx[f] for f, _ in plan}
        for f, c in plan:
            n = lens[f]
            whole, rest = divmod(n, self.page)
            for i in range(whole):
                self.table[c][i] = self.table[f][i]
                self.counts[self.table[f][i]] += 1
            if rest:
                new, old = got.pop(0), self.table[f][whole]
                self.table[c][whole] = new
                self.counts[new] = 1
                for pool in (self.k, self.v):
                    if pool is not None:
                        pool[:, new, :rest] = pool[:, old, :rest]
            self.ctx[c] = n
        return 0

    def compact(self, rows, keeps):
        plan, need = [], 0
        for i, (r, keep) in enumerate(zip(rows, keeps)):
            if not 0 <= r < len(self.ctx) or len(keep) > self.ctx[r] or r in rows[:i]:
                continue
            same = 0
            while same < len(keep) and keep[same] == same:
                same += 1
            first = same // self.page
            plan.append((r, [min(max(p, 0), self.ctx[r] - 1) for p in keep], first))
            need += pages_of(len(keep), self.page) - first
        got, missing = self._take(need)
        if missing:
            return missing
        dropped = []
        for r, keep, first in plan:
            old, held = list(self.table[r]), pages_of(self.ctx[r], self.page)
            for i in range(first, held):
                dropped.append(old[i])
                self.table[r][i] = -1
            for i in range(first, pages_of(len(keep), self.page)):
                self.table[r][i] = got.pop(0)
                self.counts[self.table[r][i]] = 1
            for pool in (self.k, self.v):
                if pool is not None:
                    for t in range(first * self.page, len(keep)):
                        src = old[keep[t] // self.page]
                        pool[:, self.table[r][t // self.page], t % self.page] = pool[:, src, keep[t] % self.page]
            self.ctx[r] = len(keep)
        for p in dropped:
            self._drop(p)
        return 0

    def release(self, rows):
        for r in rows:
            if not 0 <= r < len(self.ctx):
                continue
            for i in range(pages_of(self.ctx[r], self.page)):
                self._drop(self.table[r][i])
                self.table[r][i] = -1
            self.ctx[r] = 0
