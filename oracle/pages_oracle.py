"""CPU oracle of the page operations: plain Python on lists, one page and one sequence at a time."""
from __future__ import annotations

import numpy as np

PAGE = 64


class Pool:
    """Block table, lengths, reference counts, and one integer per page that stands for its contents."""

    def __init__(self, num_pages: int, batch: int, max_pages: int):
        self.table = -np.ones((batch, max_pages), np.int64)
        self.lens = np.zeros(batch, np.int64)
        self.refs = np.zeros(num_pages, np.int64)
        self.contents = np.arange(num_pages)
        self.invalid = self.capacity = False

    def used(self, n_tokens: int) -> int:
        return -(-n_tokens // PAGE)

    def fork(self, src, dst):
        dst0 = list(dst)
        lens0 = self.lens.copy()
        empty0 = [self.lens[d] == 0 and (self.table[d] < 0).all() if 0 <= d < len(self.lens) else False for d in dst0]
        for i, (a, b) in enumerate(zip(src, dst0)):
            ok = 0 <= a < len(self.lens) and 0 <= b < len(self.lens) and b not in dst0[:i] and a not in dst0 and empty0[i]
            if ok:
                pages = self.table[a, :self.used(lens0[a])]
                ok = bool((pages >= 0).all())
            if not ok:
                self.invalid = True
                continue
            self.table[b, :len(pages)] = pages
            self.refs[pages] += 1
            self.lens[b] = lens0[a]

    def reserve(self, seqs, n_tokens):
        todo, free = [], [p for p in range(len(self.refs)) if self.refs[p] == 0]
        refs = self.refs.copy()
        done = set()
        for s, n in zip(seqs, n_tokens):
            if not 0 <= s < len(self.lens) or n < 0 or s in done:
                self.invalid = True
                continue
            done.add(s)
            ln = int(self.lens[s])
            if self.used(ln + n) > self.table.shape[1]:
                self.capacity = True
                return
            behind = self.table[s, self.used(ln):self.used(ln + n)]
            if (self.refs[behind[behind >= 0]] != 1).any():    # pages that somebody else holds, or nobody, behind the last token
                self.invalid = True
                continue
            if n and ln % PAGE:
                p = self.table[s, ln // PAGE]
                if self.refs[p] <= 0:
                    self.invalid = True
                    continue
                if refs[p] > 1:
                    refs[p] -= 1
                    todo.append((s, ln // PAGE, p))
            for e in range(self.used(ln), self.used(ln + n)):
                if self.table[s, e] < 0:
                    todo.append((s, e, -1))
        if len(todo) > len(free):
            self.capacity = True
            return
        for (s, e, copied), page in zip(todo, free):
            if copied >= 0:
                self.refs[copied] -= 1
                self.contents[page] = self.contents[copied]
            self.table[s, e] = page
            self.refs[page] = 1

    def free(self, seqs):
        for s in seqs:
            if not 0 <= s < len(self.lens):
                self.invalid = True
                continue
            for p in self.table[s][self.table[s] >= 0]:
                self.refs[p] -= 1
            self.table[s] = -1
            self.lens[s] = 0

    def compact(self) -> int:
        named = self.table[self.table >= 0]
        if (named >= len(self.refs)).any() or (self.refs[named] <= 0).any():   # the table is wrong: nothing moves
            self.invalid = True
            return len(self.refs)
        n = int((self.refs > 0).sum())
        gaps = [p for p in range(n) if self.refs[p] == 0]
        for p in range(n, len(self.refs)):
            if self.refs[p] == 0:
                continue
            q = gaps.pop(0)
            self.contents[q] = self.contents[p]
            self.refs[q], self.refs[p] = self.refs[p], 0
            self.table[self.table == p] = q
        return n

    def check(self):
        """Counts are what the table says; nothing is mapped behind the first unmapped entry."""
        want = np.bincount(self.table[self.table >= 0], minlength=len(self.refs))
        assert np.array_equal(want, self.refs)
        for row, ln in zip(self.table, self.lens):
            n = int((row >= 0).sum())
            assert (row[:n] >= 0).all() and n >= self.used(ln)
