"""A pool of pages and the sequences that hold them, as Python lists: the
definitions in include/dart_cache.h, one sequence and one page at a time."""
from __future__ import annotations


class Pool:
    def __init__(self, num_pages, page, nseq, max_pages):
        self.page, self.max_pages = page, max_pages
        self.refs, self.rows = [0] * num_pages, [[] for _ in range(nseq)]

    def _pages(self, tokens):
        return -(-tokens // self.page)

    def select(self, parents, lens):
        """The lengths afterwards."""
        old, now = [list(r) for r in self.rows], list(lens)
        for s, p in enumerate(parents):
            if p == s or not -1 <= p < len(old):
                continue
            for x in old[s]:
                self.refs[x] -= 1
            self.rows[s] = old[p][:self._pages(lens[p])] if p >= 0 else []
            for x in self.rows[s]:
                self.refs[x] += 1
            now[s] = lens[p] if p >= 0 else 0
        return now

    def reserve(self, lens, n_rows):
        """The copies (from, to), and the sequences that got no room."""
        users, free = list(self.refs), [p for p, n in enumerate(self.refs) if n == 0]
        pairs, refused, out = [], [], False
        for s, row in enumerate(self.rows):
            if n_rows[s] <= 0:
                continue
            need = self._pages(lens[s] + n_rows[s])
            if need > self.max_pages:
                refused.append(s)
                continue
            places = [i for i in range(min(lens[s] // self.page, len(row)), need) if i >= len(row) or users[row[i]] > 1]
            out = out or len(places) > len(free)
            if out and places:
                refused.append(s)
                continue
            for i in places:
                new = free.pop(0)
                self.refs[new] = 1
                if i >= len(row):
                    row.append(new)
                    continue
                self.refs[row[i]] -= 1
                if i == lens[s] // self.page and lens[s] % self.page:
                    pairs.append((row[i], new))
                row[i] = new
        return pairs, refused

    def trim(self, lens):
        for row, n in zip(self.rows, lens):
            for x in row[self._pages(n):]:
                self.refs[x] -= 1
            del row[self._pages(n):]

    def compact(self):
        """The moves (from, to)."""
        n = sum(r > 0 for r in self.refs)
        moves = dict(zip([p for p in range(n, len(self.refs)) if self.refs[p]], [p for p in range(n) if not self.refs[p]]))
        for a, b in moves.items():
            self.refs[b], self.refs[a] = self.refs[a], 0
        self.rows = [[moves.get(x, x) for x in row] for row in self.rows]
        return list(moves.items())
