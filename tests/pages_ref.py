"""The books of a cache's pages, place by place on the host (test infrastructure only)."""
import numpy as np

BLOCK = 16


class Books:
    """uses, a page table (lists of lists) and lengths."""

    def __init__(self, uses, table, page, length=None):
        self.uses, self.table, self.page = [int(u) for u in uses], [[int(e) for e in row] for row in table], page
        self.length = None if length is None else [int(n) for n in length]

    def names(self, e):
        return 0 <= e < len(self.uses)

    def take(self, wants):
        """Pages for places [(sequence, place)], in order; how many got none."""
        short, at = 0, 0
        for b, i in wants:
            while at < len(self.uses) and self.uses[at] > 0:
                at += 1
            if at < len(self.uses):
                self.table[b][i], self.uses[at] = at, 1
            else:
                self.table[b][i] = -1
                short += 1
        return short

    def update(self, drop=None, take=None):
        for b, row in enumerate(self.table):
            if drop is not None:
                for i, e in enumerate(row):
                    if self.names(e) and max(drop[0][b], 0) <= i * self.page and (i + 1) * self.page <= drop[1][b] and drop[0][b] < drop[1][b]:
                        self.uses[e] -= 1
                        row[i] = -1
        if take is None:
            return 0
        wants = []
        for b, row in enumerate(self.table):
            lo, hi = max(take[0][b], 0), take[1][b]
            wants += [(b, i) for i, e in enumerate(row) if lo < hi and i * self.page < hi and (i + 1) * self.page > lo and not self.names(e)]
        return self.take(wants)

    def fork(self, parent):
        """(places without a page, copies [(from, to, tokens)])"""
        old, n, met, wants, length = self.table, len(self.table), set(), [], []
        new = []
        for j, p in enumerate(parent):
            row, tokens = [-1] * len(old[j]), 0
            if 0 <= p < n:
                tokens = max(self.length[p], 0)
                whole, rest = divmod(tokens, self.page)
                for i, e in enumerate(old[p]):
                    if i < whole or p not in met:
                        row[i] = e
                if p in met and rest and whole < len(row) and self.names(old[p][whole]):
                    wants.append((j, whole, old[p][whole], rest))
                met.add(p)
            new.append(row)
            length.append(tokens)
        for rows, sign in ((old, -1), (new, 1)):
            for e in (e for row in rows for e in row):
                if self.names(e):
                    self.uses[e] += sign
        self.table, self.length = new, length
        short = self.take([w[:2] for w in wants])
        return short, [(src, self.table[j][i], rest) for j, i, src, rest in wants if self.table[j][i] >= 0]

    def compact(self):
        """(pages in use, moves [(from, to, tokens)])"""
        n, moves = sum(u > 0 for u in self.uses), []
        free = [p for p in range(n) if self.uses[p] <= 0]
        late = [p for p in range(len(self.uses) - 1, n - 1, -1) if self.uses[p] > 0]
        for a, b in zip(late, free):
            moves.append((a, b, self.page))
            self.uses[b], self.uses[a] = self.uses[a], 0
        now = {a: b for a, b, _ in moves}
        self.table = [[now.get(e, e) for e in row] for row in self.table]
        return n, moves


def copied(arrays, moves):
    """k [pages, heads, page, d], v [pages, heads, page / 16, d, 16] and their scales [pages, heads, page / 16] after copies [(from, to, tokens)]."""
    k, v, ks, vs = (a.copy() for a in arrays)
    for a, b, tokens in moves:
        n = -(-min(max(tokens, 0), k.shape[2]) // BLOCK)
        k[b, :, :n * BLOCK] = arrays[0][a, :, :n * BLOCK]
        for x, y in ((v, arrays[1]), (ks, arrays[2]), (vs, arrays[3])):
            x[b, :, :n] = y[a, :, :n]
    return k, v, ks, vs


def random_books(rng, pages, batch, places, page, fill=0.5, shared=0.2, strange=0.02, pinned=0.02):
    """Books in use: part of the places have pages, of which some are named several times, some places name none by odd numbers, and some pages are kept by a caller."""
    order = rng.permutation(pages)
    table = np.full((batch, places), -1, np.int64)
    at = 0
    for b in range(batch):
        for i in range(places):
            if rng.random() < fill and at < pages:
                if at and rng.random() < shared:
                    table[b, i] = order[rng.integers(0, at)]
                else:
                    table[b, i] = order[at]
                    at += 1
            elif rng.random() < strange:
                table[b, i] = rng.choice([-7, pages, pages + 5, -(1 << 31), (1 << 31) - 1])
    uses = np.zeros(pages, np.int64)
    named = table[(table >= 0) & (table < pages)]
    np.add.at(uses, named, 1)
    uses += rng.random(pages) < pinned
    length = rng.integers(0, places * page + 1, batch) if places else np.zeros(batch, np.int64)
    return Books(uses, table, page, length)
