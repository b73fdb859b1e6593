"""CPU oracle for page bookkeeping: one row and one page after the other.

TEST INFRASTRUCTURE ONLY.  The product path never calls it and shares no code
with it.  A `Pages` holds what the device holds: ref_counts, tables, lengths.
Every call returns (status, pairs, pages, bad) with status 0 or 4, the result
words of the library's call of that name.
"""
from __future__ import annotations

import numpy as np

OK, BOUNDS = 0, 4


class Pages:
    def __init__(self, refs, tables, lens, page_size):
        self.refs = [int(x) for x in refs]
        self.tables = np.array(tables, dtype=np.int64).copy()
        self.lens = [int(x) for x in lens]
        self.P = int(page_size)

    def _ok(self, row):
        return 0 <= row < len(self.lens)

    def _good_len(self, n):
        return 0 <= n <= self.tables.shape[1] * self.P

    def _page(self, e):
        return 0 <= e < len(self.refs)

    def _held(self, n):
        return -(-n // self.P)

    def _take(self):
        p = self.refs.index(0)
        self.refs[p] = 1
        return p

    def count(self):
        self.refs = [0] * len(self.refs)
        bad = 0
        for row, n in enumerate(self.lens):
            if not self._good_len(n):
                bad += 1
                continue
            for e in self.tables[row, :self._held(n)]:
                if self._page(e):
                    self.refs[e] += 1
                else:
                    bad += 1
        return BOUNDS if bad else OK, [], sum(1 for c in self.refs if c), bad

    def free(self, rows, keep=None):
        bad = gone = 0
        for i, row in enumerate(rows):
            k = 0 if keep is None else int(keep[i])
            if not self._ok(row) or k < 0 or not self._good_len(self.lens[row]):
                bad += 1
                continue
            n = self.lens[row]
            for j in range(self._held(min(k, n)), self._held(n)):
                e = int(self.tables[row, j])
                self.tables[row, j] = -1
                if e == -1:
                    continue
                if not self._page(e) or self.refs[e] <= 0:
                    bad += 1
                else:
                    self.refs[e] -= 1
                    gone += 1
            self.lens[row] = min(n, k)
        return BOUNDS if bad else OK, [], gone, bad

    def fork(self, parents, children):
        bad = 0
        for i, c in enumerate(children):
            p = parents[i]
            last = max(k for k, x in enumerate(children) if x == c)
            bad += not (self._ok(c) and last == i and self._ok(p) and self.lens[c] == 0 and self._good_len(self.lens[p]))
        ok = [i for i, c in enumerate(children) if self._ok(parents[i]) and self._good_len(self.lens[parents[i]])]
        want = sum(1 for i in ok if self.lens[parents[i]] % self.P)
        if bad:
            return BOUNDS, [], None, bad
        if want > self.refs.count(0):
            return BOUNDS, [], want, 0
        pairs, lens = [], [self.lens[p] for p in parents]
        taken = []
        for n in lens:
            taken.append(self._take() if n % self.P else None)
        for i, c in enumerate(children):
            n, p = lens[i], parents[i]
            for j in range(n // self.P):
                e = int(self.tables[p, j])
                self.tables[c, j] = e
                if self._page(e):
                    self.refs[e] += 1
                else:
                    bad += 1
            if n % self.P:
                e = int(self.tables[p, n // self.P])
                bad += not self._page(e)
                self.tables[c, n // self.P] = taken[i]
                pairs.append((e, taken[i]))
            self.lens[c] = n
        return BOUNDS if bad else OK, pairs, want, bad

    def grow(self, rows, new_lens):
        bad, plan, want = 0, [], 0
        for i, row in enumerate(rows):
            last = max(k for k, x in enumerate(rows) if x == row)
            if not self._ok(row) or last != i:
                bad += 1
                continue
            old, new = self.lens[row], int(new_lens[i])
            if not (self._good_len(old) and old <= new and self._good_len(new)):
                bad += 1
                continue
            e = int(self.tables[row, old // self.P]) if old % self.P else -1
            own = new > old and old % self.P != 0 and self._page(e) and self.refs[e] > 1
            plan.append((row, old, new, e if own else None))
            want += self._held(new) - self._held(old) + own
        if bad:
            return BOUNDS, [], None, bad
        if want > self.refs.count(0):
            return BOUNDS, [], want, 0
        pairs, shared = [], []
        for row, old, new, e in plan:
            if e is not None:
                p = self._take()
                self.tables[row, old // self.P] = p
                pairs.append((e, p))
                shared.append(e)
            for j in range(self._held(old), self._held(new)):
                self.tables[row, j] = self._take()
            self.lens[row] = new
        for e in shared:                       # given back after every page of the call is taken
            self.refs[e] -= 1
        return OK, pairs, want, 0

    def compact(self):
        live = sum(1 for c in self.refs if c > 0)
        holes = [p for p in range(live) if self.refs[p] <= 0]
        movers = [p for p in range(len(self.refs) - 1, live - 1, -1) if self.refs[p] > 0]
        to = dict(zip(movers, holes))
        bad = 0
        for row, n in enumerate(self.lens):
            if not self._good_len(n):
                bad += 1
                continue
            for j in range(self._held(n)):
                e = int(self.tables[row, j])
                if not self._page(e):
                    bad += 1
                elif e in to:
                    self.tables[row, j] = to[e]
        for s, d in to.items():
            self.refs[d], self.refs[s] = self.refs[s], 0
        return BOUNDS if bad else OK, list(to.items()), live, bad
