"""Oracle: the pages of a pool -- reserved, shared, given back, compacted -- one
list entry after the other, on plain Python lists.

TEST INFRASTRUCTURE ONLY (see ``oracle/__init__.py``).

A pool is (tables [n_seqs][width], kv_len [n_seqs], refs [n_pages], caches: arrays
[n_pages, ...]); refs counts the entries that name a page, 0 is free, and the lowest
free page is given first.  (Sec. 7.1: cache blocks are shared by prefix; Sec. 8:
blocks are reserved and released.  Reference counts and their order are readings:
the paper names neither.)
"""

from __future__ import annotations

B = 16


class Pool:
    def __init__(self, tables, kv_len, refs, caches=()):
        self.tables = [list(map(int, row)) for row in tables]
        self.kv_len, self.refs = list(map(int, kv_len)), list(map(int, refs))
        self.caches = [c.copy() for c in caches]
        self.width = len(self.tables[0]) if self.tables else 0

    def _take(self, n):
        """The lowest n free pages, or None."""
        free = [p for p, r in enumerate(self.refs) if r == 0]
        return free[:n] if n <= len(free) else None

    def _partial_page_gone(self, table, length):
        """The last page is filled in part and the table does not name it."""
        return length % B > 0 and not 0 <= table[length // B] < len(self.refs)

    def reserve(self, seqs, add):
        missing, seen, out = 0, set(), False
        for s, a in zip(seqs, add):
            if not 0 <= s < len(self.tables) or s in seen:
                continue
            seen.add(s)
            to = self.kv_len[s] + a
            first, last = -(-self.kv_len[s] // B), -(-to // B)
            if a < 0 or last > self.width or (a > 0 and self._partial_page_gone(self.tables[s], self.kv_len[s])):
                missing += 1
                continue
            n = last - first
            pages = None if out and n else self._take(n)
            if pages is None:
                out, missing = True, missing + 1
                continue
            for j, p in enumerate(pages):
                self.tables[s][first + j], self.refs[p] = p, 1
            self.kv_len[s] = to
        return missing

    def fork(self, parents, children):
        missing, seen, out = 0, set(), False
        before = [list(t) for t in self.tables], list(self.kv_len)
        n_seqs = len(self.tables)
        shared = []
        for a, c in zip(parents, children):
            named, _ = c in seen, seen.add(c)
            if not (0 <= a < n_seqs and 0 <= c < n_seqs) or named:
                continue
            if c in parents:
                missing += 1
                continue
            length = before[1][a]
            whole, part = divmod(length, B)
            pages = None if out and part else self._take(1 if part else 0)
            bad = -(-length // B) > self.width or self._partial_page_gone(before[0][a], length)
            if bad:
                pages = None
            self.tables[c] = [-1] * self.width
            if pages is None:
                out |= not bad
                missing += 1
                self.kv_len[c] = 0
                continue
            self.kv_len[c] = length
            self.tables[c][:whole] = before[0][a][:whole]
            shared += [p for p in before[0][a][:whole] if 0 <= p < len(self.refs)]
            if part:
                self.tables[c][whole], self.refs[pages[0]] = pages[0], 1
                for x in self.caches:
                    x[pages[0]] = x[before[0][a][whole]]
        for p in shared:
            self.refs[p] += 1
        return missing

    def free(self, seqs, begin, end):
        seen = set()
        for s, lo, hi in zip(seqs, begin, end):
            if not 0 <= s < len(self.tables) or s in seen:
                continue
            seen.add(s)
            n = self.kv_len[s]
            for j in range(min(self.width, -(-n // B))):
                if j * B >= lo and min(n, j * B + B) <= hi and self.tables[s][j] != -1:
                    p, self.tables[s][j] = self.tables[s][j], -1
                    if 0 <= p < len(self.refs):
                        self.refs[p] -= 1
            if lo <= 0 and hi >= n:
                self.kv_len[s] = 0

    def compact(self):
        n = sum(r > 0 for r in self.refs)
        behind = [p for p, r in enumerate(self.refs) if r > 0 and p >= n]
        holes = [p for p in range(n) if self.refs[p] <= 0]
        to = dict(zip(behind, holes))
        self.tables = [[to.get(p, p) for p in row] for row in self.tables]
        for a, b in to.items():
            self.refs[b], self.refs[a] = self.refs[a], 0
            for x in self.caches:
                x[b] = x[a]

    def consistent(self):
        """refs is what the tables say."""
        count = [0] * len(self.refs)
        for row in self.tables:
            for p in row:
                if 0 <= p < len(count):
                    count[p] += 1
        return count == self.refs
