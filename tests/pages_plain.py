"""The pages of the cache by lists and loops, from the definitions of quarot.h."""
import numpy as np


def up(x, page):
    return -(-x // page)


class Pages:
    def __init__(self, batch, most, n, page):
        self.page, self.n, self.most = page, n, most
        self.table = [[-1] * most for _ in range(batch)]
        self.lens, self.refs = [0] * batch, [0] * n

    def _is(self, e):
        return 0 <= e < self.n

    def fork(self, parent):
        old, lens = [list(r) for r in self.table], list(self.lens)
        for b, p in enumerate(parent):
            there = 0 <= p < len(old)
            for e in old[b]:
                if self._is(e):
                    self.refs[e] -= 1
            self.table[b] = list(old[p]) if there else [-1] * self.most
            self.lens[b] = lens[p] if there else 0
            for e in self.table[b]:
                if self._is(e):
                    self.refs[e] += 1

    def reserve(self, new):
        """(cu, src, dst, missing)"""
        B, page = len(new), self.page
        none = [0] * (B + 1), [-1] * B, [-1] * B
        after = [max(0, x + n) for x, n in zip(self.lens, new)]
        if max(after) > self.most * page or sum(max(0, n) for n in new) > 1 << 30:
            return *none, -1
        writers = {}
        for b, n in enumerate(new):
            j = self.lens[b] // page
            if n > 0 and self.lens[b] % page and j < self.most and self._is(self.table[b][j]):
                writers.setdefault(self.table[b][j], []).append(b)
        want = []  # (sequence, entry, page that it leaves or -1, copied)
        for b, n in enumerate(new):
            if n <= 0:
                continue
            for j in range(self.lens[b] // page, up(after[b], page)):
                e, older = self.table[b][j], j * page < self.lens[b]
                if older:
                    if self._is(e) and self.refs[e] > 1 and not (
                            len(writers[e]) == self.refs[e] and writers[e][0] == b):
                        want.append((b, j, e, True))
                elif not self._is(e):
                    want.append((b, j, -1, False))
                elif self.refs[e] > 1:
                    want.append((b, j, e, False))
        free = [i for i, r in enumerate(self.refs) if r == 0]
        if len(free) < len(want):
            return *none, len(want) - len(free)
        cu, src, dst = [0], [-1] * B, [-1] * B
        for n in new:
            cu.append(cu[-1] + max(0, n))
        for (b, j, e, copied), y in zip(want, free):
            self.table[b][j] = y
            self.refs[y] = 1
            if e >= 0:
                self.refs[e] -= 1
            if copied:
                src[b], dst[b] = e, y
        for b, n in enumerate(new):
            if n < 0:
                for j in range(up(after[b], page), min(self.most, up(self.lens[b], page))):
                    if self._is(self.table[b][j]):
                        self.refs[self.table[b][j]] -= 1
                    self.table[b][j] = -1
        self.lens = after
        return cu, src, dst, 0

    def compact(self):
        live = sum(r > 0 for r in self.refs)
        src = [i for i in range(live, self.n) if self.refs[i] > 0]
        dst = [i for i in range(live) if self.refs[i] <= 0]
        to = dict(zip(src, dst))
        self.table = [[to.get(e, e) for e in r] for r in self.table]
        for s, d in to.items():
            self.refs[d], self.refs[s] = self.refs[s], 0
        pad = [-1] * (self.n // 2 - len(src))
        return src + pad, dst + pad, live

    def consistent(self):
        count = np.zeros(self.n, np.int64)
        for r in self.table:
            for e in r:
                if self._is(e):
                    count[e] += 1
        return count.tolist() == self.refs
