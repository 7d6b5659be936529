"""Pages of a pool that sequences share, one page after the other (numpy).

State: table [rows, pages per row], lens [rows], refs [pages] (rows that hold a page; 0: free), arrays with one entry per page.
A row holds the first ceil(len / page_size) pages of its table row.  Every function changes the state in place and returns the
set of things that went wrong ("arg", "capacity")."""
from __future__ import annotations

import numpy as np


class Pool:
    def __init__(self, table, lens, refs, arrays, page_size):
        self.table, self.lens, self.refs, self.page_size = table.copy(), lens.copy(), refs.copy(), page_size
        self.arrays = [a.copy() for a in arrays]

    def held(self, n):
        if n <= 0 or n > self.table.shape[1] * self.page_size:
            return 0
        return -(-int(n) // self.page_size)

    def fits(self, n):
        return n <= self.table.shape[1] * self.page_size

    def lowest_free(self):
        free = np.flatnonzero(self.refs <= 0)
        return int(free[0]) if free.size else None

    def free(self, rows):
        bad = set()
        for r in rows:
            if not 0 <= r < len(self.lens):
                bad.add("arg")
                continue
            n, self.lens[r] = self.lens[r], 0
            if not self.fits(n):
                bad.add("capacity")
            for p in self.table[r, :self.held(n)]:
                if 0 <= p < len(self.refs):
                    self.refs[p] -= 1
                else:
                    bad.add("capacity")
        return bad

    def fork(self, parents, children):
        bad, begin, seen = set(), self.lens.copy(), set()
        plan = []
        for a, c in zip(parents, children):
            rows = len(self.lens)
            if not (0 <= a < rows and 0 <= c < rows) or begin[c] > 0 or c in seen:
                bad.add("arg")
                continue
            if not self.fits(begin[a]):
                bad.add("capacity")
                continue
            seen.add(c)
            plan.append((a, c))
        # pages are taken in the order of the list; what a fork shares stays used in any case
        for a, c in plan:
            n = max(int(begin[a]), 0)
            self.lens[c] = 0
            last = n // self.page_size
            page = None
            if n % self.page_size:
                page = self.lowest_free()
                if page is None:
                    bad.add("capacity")
                    continue
                self.refs[page] = 1
                for x in self.arrays:
                    x[page] = x[self.table[a, last]]
            self.table[c, :last] = self.table[a, :last]
            np.add.at(self.refs, self.table[a, :last], 1)
            if page is not None:
                self.table[c, last] = page
            self.lens[c] = n
        return bad

    def grow(self, room):
        bad = set()
        free = list(np.flatnonzero(self.refs <= 0))
        at = 0
        for r, more in enumerate(room):
            if more <= 0:
                continue
            n = max(int(self.lens[r]), 0)
            if not self.fits(n + int(more)):
                bad.add("capacity")
                continue
            old, now = self.held(n), self.held(n + int(more))
            mine = free[at:at + now - old]
            at += now - old
            if len(mine) < now - old:
                bad.add("capacity")
                continue
            self.table[r, old:now] = mine
            self.refs[mine] = 1
            self.lens[r] = n + more
        return bad

    def compact(self):
        used = self.refs > 0
        n = int(used.sum())
        src = [p for p in range(n, len(self.refs)) if used[p]]
        dst = [p for p in range(n) if not used[p]]
        for s, d in zip(src, dst):
            for x in self.arrays:
                x[d] = x[s]
            for r in range(len(self.lens)):
                row = self.table[r, :self.held(self.lens[r])]
                row[row == s] = d
        self.refs[dst] = self.refs[src]
        self.refs[n:] = 0
        return n
