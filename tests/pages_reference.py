"""The calls on pages in plain Python, one row at a time: what they do to the books, and which pages they copy."""
from __future__ import annotations

import random


class Books:
    def __init__(self, n_seqs, columns, n_pages, page_len):
        self.pages = [[-1] * columns for _ in range(n_seqs)]
        self.len = [0] * n_seqs
        self.refs = [0] * n_pages
        self.page_len, self.columns = page_len, columns
        self.short = False

    def copy(self):
        b = Books(len(self.len), self.columns, len(self.refs), self.page_len)
        b.pages, b.len, b.refs = [list(r) for r in self.pages], list(self.len), list(self.refs)
        return b

    def used_columns(self, length):
        return -(-length // self.page_len)

    def _free(self):
        return [p for p, r in enumerate(self.refs) if r == 0]

    def fork(self, src, dst):
        """Copies (from, to).  Forks that the call has to refuse are left out by the caller."""
        free, need, copies = self._free(), 0, []
        before = [(self.len[s], list(self.pages[s])) for s in src]
        for (length, row), d in zip(before, dst):
            part = length % self.page_len != 0
            need += part
            if part and need > len(free):
                self.short = True
                continue
            whole = length // self.page_len
            for e in range(whole):
                self.refs[row[e]] += 1
                self.pages[d][e] = row[e]
            if part:
                p = free[need - 1]
                copies.append((row[whole], p))
                self.refs[p] = 1
                self.pages[d][whole] = p
            self.len[d] = length
        return copies

    def resize(self, target):
        for s, n in enumerate(target):
            for e in range(self.used_columns(n), self.used_columns(self.len[s])):
                self.refs[self.pages[s][e]] -= 1
                self.pages[s][e] = -1
        free, need, copies, plans = self._free(), 0, [], []
        for s, n in enumerate(target):
            kept = min(n, self.len[s])
            copy = kept % self.page_len != 0 and self.refs[self.pages[s][kept // self.page_len]] > 1
            more = max(0, self.used_columns(n) - self.used_columns(self.len[s]))
            plans.append((need, copy, more, kept // self.page_len))
            need += copy + more
        for s, ((at, copy, more, column), n) in enumerate(zip(plans, target)):
            if copy + more and at + copy + more > len(free):
                self.short = True
                if n < self.len[s]:
                    self.len[s] = n
                continue
            if copy:
                old = self.pages[s][column]
                copies.append((old, free[at]))
                self.refs[old] -= 1
                self.refs[free[at]] = 1
                self.pages[s][column] = free[at]
            have = self.used_columns(self.len[s])
            for e in range(more):
                self.pages[s][have + e] = free[at + copy + e]
                self.refs[free[at + copy + e]] = 1
            self.len[s] = n
        return copies

    def compact(self):
        held = [p for p, r in enumerate(self.refs) if r]
        used = len(held)
        copies = list(zip([p for p in held if p >= used], [p for p, r in enumerate(self.refs[:used]) if r == 0]))
        to = dict(copies)
        for s, row in enumerate(self.pages):
            for e in range(self.used_columns(self.len[s])):
                row[e] = to.get(row[e], row[e])
        for f, t in copies:
            self.refs[t], self.refs[f] = self.refs[f], 0
        return copies, used

    def check(self):
        """Every page is held as often as refs says, and a page that is kept in part by one row only, unless a call was short."""
        count = [0] * len(self.refs)
        for s, row in enumerate(self.pages):
            for e in range(self.used_columns(self.len[s])):
                count[row[e]] += 1
            if self.len[s] % self.page_len and not self.short:
                assert self.refs[row[self.len[s] // self.page_len]] == 1
        assert count == self.refs


def random_targets(books, r: random.Random, most):
    out = []
    for length in books.len:
        what = r.random()
        out.append(length if what < 0.3 else 0 if what < 0.4 else r.randint(0, length) if what < 0.6 else r.randint(length, most))
    return out
