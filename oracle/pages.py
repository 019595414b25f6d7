"""The book of a cache's pages from its definition, entry by entry on the CPU: test infrastructure that shares no code with
the kernels."""
from __future__ import annotations

import numpy as np


class Book:
    def __init__(self, refs, table, kv_len, page_size):
        self.refs, self.table, self.kv_len = (np.array(x, dtype=np.int64) for x in (refs, table, kv_len))
        self.page = page_size

    def pages(self, tokens):
        return -(-tokens // self.page)

    @property
    def most(self):
        return self.table.shape[1] * self.page

    def _fine(self, row):
        return 0 <= row < len(self.kv_len) and 0 <= self.kv_len[row] <= self.most

    def _take(self, wants):
        """wants: (row, first entry, pages) or None for each of the list; who gets its pages."""
        free = [p for p in range(len(self.refs)) if self.refs[p] == 0]
        out, at, short = [], 0, False
        for w in wants:
            if w is None:
                out.append(False)
                continue
            row, first, n = w
            if n and (short or at + n > len(free)):
                short = True
                out.append(False)
                continue
            for e in range(n):
                self.table[row, first + e] = free[at + e]
                self.refs[free[at + e]] = 1
            at += n
            out.append(True)
        return out

    def grow(self, counts, which=None, T=0):
        """done, slots, pos."""
        which = list(range(len(counts))) if which is None else list(which)
        wants = []
        for i, (row, c) in enumerate(zip(which, counts)):
            fine = self._fine(row) and c >= 0 and row not in which[:i] and self.kv_len[row] + c <= self.most
            wants.append((row, self.pages(self.kv_len[row]), self.pages(self.kv_len[row] + c) - self.pages(self.kv_len[row]))
                         if fine else None)
        got = self._take(wants)
        done, slots, pos = [], [], []
        for row, c, ok in zip(which, counts, got):
            for x in range(max(c, 0)):
                if len(slots) == T:
                    break
                p = self.kv_len[row] + x if ok else 0
                slots.append(self.table[row, p // self.page] * self.page + p % self.page if ok else -1)
                pos.append(p)
            if ok:
                self.kv_len[row] += c
            done.append(self.kv_len[row] if ok else -1)
        return done, slots + [-1] * (T - len(slots)), pos + [0] * (T - len(pos))

    def fork(self, parents, to):
        """done, src, dst."""
        before, wants = self.kv_len.copy(), []
        for i, (a, b) in enumerate(zip(parents, to)):
            fine = self._fine(a) and 0 <= b < len(before) and before[b] == 0 and b not in list(to)[:i]
            wants.append((b, before[a] // self.page, int(before[a] % self.page != 0)) if fine else None)
        got = self._take(wants)
        done, src, dst = [], [], []
        for a, b, w, ok in zip(parents, to, wants, got):
            copied = ok and w[2]
            src.append(self.table[a, w[1]] if copied else -1)
            dst.append(self.table[b, w[1]] if copied else -1)
            done.append(before[a] if ok else -1)
            if ok:
                for e in range(w[1]):
                    self.table[b, e] = self.table[a, e]
                    self.refs[self.table[a, e]] += 1
                self.kv_len[b] = before[a]
        return done, src, dst

    def free(self, which):
        for row in which:
            if 0 <= row < len(self.kv_len):
                for e in range(self.pages(min(max(self.kv_len[row], 0), self.most))):
                    if 0 <= self.table[row, e] < len(self.refs):
                        self.refs[self.table[row, e]] -= 1
                self.kv_len[row] = 0

    def compact(self, n):
        """src, dst."""
        src, dst = [], []
        for _ in range(n):
            used, free = np.flatnonzero(self.refs), np.flatnonzero(self.refs == 0)
            if not len(used) or not len(free) or used[-1] < free[0]:
                break
            a, b = used[-1], free[0]
            src.append(a)
            dst.append(b)
            self.refs[b], self.refs[a] = self.refs[a], 0
            for row in range(len(self.kv_len)):
                held = self.table[row, :self.pages(self.kv_len[row])]
                held[held == a] = b
        return src + [-1] * (n - len(src)), dst + [-1] * (n - len(dst))

    def held(self):
        """The pages of every row."""
        return [self.table[r, :self.pages(min(max(m, 0), self.most))].tolist() for r, m in enumerate(self.kv_len)]

    def check(self):
        """What has to hold of a book, whatever was done to it."""
        count, last = np.zeros(len(self.refs), dtype=np.int64), set()
        for row, pages in enumerate(self.held()):
            for p in pages:
                count[p] += 1
            if self.kv_len[row] % self.page:
                last.add(pages[-1])
        assert np.array_equal(count, self.refs)
        assert all(count[p] == 1 for p in last)  # a partly full page is one row's alone
