"""Pages of the cache in Python's numbers: which row of the block table holds which page, how often a page is held, and whose first
content each page has.  (The paper has no counterpart.)"""
from __future__ import annotations


class Book:
    def __init__(self, page, max_pages, n_pages, rows):
        self.page, self.max_pages, self.n_pages = page, max_pages, n_pages
        self.refs, self.lengths = [0] * n_pages, [0] * rows
        self.table = [[-1] * max_pages for _ in range(rows)]
        self.content = list(range(n_pages))               # page p has what page content[p] had at first

    def places(self, length):
        return -(-length // self.page)

    def held(self, row):
        return [p for p in self.table[row][:self.places(self.lengths[row])] if 0 <= p < self.n_pages]

    def consistent(self):
        """refs counts the places, and a partly filled page is held by several rows only where none has grown in it."""
        count = [0] * self.n_pages
        for b in range(len(self.lengths)):
            for p in self.held(b):
                count[p] += 1
        return count == self.refs

    def copy(self, src, dst):
        was = list(self.content)
        for a, b in zip(src, dst):
            if 0 <= a < self.n_pages and 0 <= b < self.n_pages:
                self.content[b] = was[a]

    def fork(self, parent):
        table, lengths = [list(t) for t in self.table], list(self.lengths)
        for b, p in enumerate(parent):
            if p == b or not -1 <= p < len(parent):
                continue
            for q in self.held(b):
                self.refs[q] -= 1
            n = lengths[p] if p >= 0 else 0
            had, have = self.places(lengths[b]), self.places(n)
            for i in range(max(had, have)):
                self.table[b][i] = table[p][i] if i < have else -1
            self.lengths[b] = n
            for q in self.held(b):
                self.refs[q] += 1

    def resize(self, to):
        """Returns what is lacking."""
        if any(not 0 <= n <= self.max_pages * self.page for n in to):
            return -1
        free = [p for p in range(self.n_pages) if self.refs[p] == 0]
        grows_in, gaps = [], []                           # the page that a row grows in; whether there is none in that place
        for b, n in enumerate(self.lengths):
            inside = n % self.page and to[b] > n
            p = self.table[b][self.places(n) - 1] if inside else -1
            grows_in.append(p if 0 <= p < self.n_pages else -1)
            gaps.append(bool(inside) and grows_in[b] < 0)
        takes = []
        for b, p in enumerate(grows_in):
            growing = [c for c, q in enumerate(grows_in) if q == p]
            keeps = len(growing) == self.refs[p] and growing[0] == b
            takes.append(p >= 0 and self.refs[p] > 1 and not keeps)
        need = sum(takes) + sum(gaps) + sum(max(0, self.places(m) - self.places(n)) for n, m in zip(self.lengths, to))
        if need > len(free):
            return need - len(free)
        was = list(self.content)
        for b, (n, m) in enumerate(zip(list(self.lengths), to)):
            had, have = self.places(n), self.places(m)
            if takes[b]:
                p = free.pop(0)
                self.content[p], self.refs[p] = was[grows_in[b]], 1
                self.refs[grows_in[b]] -= 1
                self.table[b][had - 1] = p
            for i in range(had - gaps[b], have):
                p = free.pop(0)
                self.refs[p], self.table[b][i] = 1, p
            for i in range(have, had):
                p = self.table[b][i]
                if 0 <= p < self.n_pages:
                    self.refs[p] -= 1
                self.table[b][i] = -1
            self.lengths[b] = m
        return 0

    def trim(self, window, sinks):
        for b, n in enumerate(self.lengths):
            for i in range(self.places(n)):
                tokens = range(i * self.page, (i + 1) * self.page)
                p = self.table[b][i]
                # (a token at n or behind sees j > n - window at the most)
                if 0 <= p < self.n_pages and not any(j > n - window or j < sinks for j in (tokens[0], tokens[-1])):
                    self.refs[p] -= 1
                    self.table[b][i] = -1

    def compact(self):
        """Returns the number of used pages."""
        used = sum(r > 0 for r in self.refs)
        holes = [p for p in range(used) if self.refs[p] == 0]
        moved = dict(zip([p for p in range(used, self.n_pages) if self.refs[p]], holes))
        for p, h in moved.items():
            self.content[h], self.refs[h], self.refs[p] = self.content[p], self.refs[p], 0
        for b in range(len(self.lengths)):
            for i in range(self.places(self.lengths[b])):
                self.table[b][i] = moved.get(self.table[b][i], self.table[b][i])
        return used
