"""A pool of pages by its definition (numpy, CPU): what the GPU tests of the page calls compare with."""
import numpy as np


class Pool:
    def __init__(self, pages, rows, width, page):
        self.refs, self.table, self.page = np.zeros(pages, dtype=np.int64), np.full((rows, width), -1, dtype=np.int64), page

    def pages(self, n):
        return min(self.table.shape[1], -(-max(int(n), 0) // self.page))

    def is_page(self, p):
        return 0 <= p < len(self.refs)

    def is_row(self, r):
        return 0 <= r < len(self.table)

    def grow(self, rows, lens):
        free, missing = list(np.nonzero(self.refs == 0)[0]), 0
        for r, n in zip(rows, lens):
            if not self.is_row(r):
                continue
            for j in range(self.pages(n)):
                if self.table[r, j] < 0:
                    if free:
                        self.table[r, j] = free.pop(0)
                        self.refs[self.table[r, j]] = 1
                    else:
                        missing += 1
        return missing

    def free(self, rows, lens=None):
        for i, r in enumerate(rows):
            if self.is_row(r):
                self.let_go(r, 0 if lens is None else self.pages(lens[i]))

    def let_go(self, r, first):
        for p in self.table[r, first:]:
            if self.is_page(p):
                self.refs[p] -= 1
        self.table[r, first:] = -1

    def fork(self, parents, children, lens):
        n, missing = len(children), 0
        free, pairs = list(np.nonzero(self.refs == 0)[0]), []
        for a, c, x in zip(parents, children, lens):
            if not self.is_row(c):
                continue
            row = np.full(self.table.shape[1], -1)
            if self.is_row(a):
                x = min(max(int(x), 0), self.table.shape[1] * self.page)
                full = x // self.page
                row[:full] = [p if self.is_page(p) else -1 for p in self.table[a, :full]]
                for p in row[:full]:
                    if p >= 0:
                        self.refs[p] += 1
                if x % self.page and self.is_page(self.table[a, full]):
                    if free:
                        row[full] = free.pop(0)
                        self.refs[row[full]] += 1
                        pairs.append((self.table[a, full], row[full], x % self.page))
                    else:
                        missing += 1
            self.let_go(c, 0)
            self.table[c] = row
        lists = np.full((3, n), -1)
        for i, p in enumerate(pairs):
            lists[:, i] = p
        return lists[0], lists[1], lists[2], np.array([len(pairs), missing])

    def compact(self, most):
        used, free = np.nonzero(self.refs != 0)[0], np.nonzero(self.refs == 0)[0]
        lists, name, n = np.full((2, most), -1), np.arange(len(self.refs)), 0
        for a, b in zip(used[::-1], free):
            if b >= a or n == most:
                break
            lists[:, n] = a, b
            name[a] = b
            n += 1
        for a, b in lists[:, :n].T:
            self.refs[b], self.refs[a] = self.refs[a], 0
        inside = (self.table >= 0) & (self.table < len(self.refs))
        self.table[inside] = name[self.table[inside]]
        return lists[0], lists[1], np.array([n, len(used)])

    def counts_hold(self):
        inside = self.table[(self.table >= 0) & (self.table < len(self.refs))]
        return (np.bincount(inside, minlength=len(self.refs)) == self.refs).all()


def filled(rng, pages, rows, width, page, load):
    """A pool of which about 'load' of the pages are in use, in random places, rows of different lengths; some are shared."""
    pool = Pool(pages, rows, width, page)
    order, at = rng.permutation(pages)[:int(load * pages)], 0
    lens = np.zeros(rows, dtype=np.int64)
    for r in range(rows):
        c = min(int(rng.integers(0, width + 1)), len(order) - at)
        pool.table[r, :c] = order[at:at + c]
        at += c
        lens[r] = max(0, c * page - int(rng.integers(0, page)))
        if r and c and rng.random() < 0.3:                 # shares its first page with the row before
            first = pool.table[r - 1, 0]
            if first >= 0:
                pool.table[r, 0] = first
    inside = pool.table[pool.table >= 0]
    pool.refs = np.bincount(inside, minlength=pages).astype(np.int64)
    return pool, lens
