"""Rows of a pool that share pages and are written again: a row that is its own parent in tl_kv_fork gets the last page that it
fills in part for itself, and loses nothing where none is free; and forks that find too few pages, which are repeated."""
import numpy as np
import pytest

import paper_2607_04031_amd as tl
from tests import _pool
from tests._gpu import banner
from tests.test_gpu_kv import _int, _lib  # noqa: F401
from tests.test_gpu_pages import _get, _same, _up

pytestmark = pytest.mark.gpu


class Pool(_pool.Pool):
    """A pool whose rows may be their own parents: the last page of such a row stays if no other entry names it, and where no
    page is free."""

    def fork(self, parents, children, lens):
        free, pairs, missing, before = list(np.nonzero(self.refs == 0)[0]), [], 0, self.refs.copy()
        for a, c, x in zip(parents, children, lens):
            full, rest = divmod(min(max(int(x), 0), self.table.shape[1] * self.page), self.page)
            row = np.full(self.table.shape[1], -1)
            row[:full] = self.table[a, :full]
            last = self.table[a, full] if rest else -1
            if last >= 0 and not (a == c and before[last] == 1):
                if free:
                    pairs.append((last, free[0], rest))
                    last = free.pop(0)
                else:
                    missing, last = missing + 1, last if a == c else -1
            if rest:
                row[full] = last
            for p in row[row >= 0]:
                self.refs[p] += 1
            self.let_go(c, 0)
            self.table[c] = row
        lists = np.full((3, len(children)), -1)
        for i, p in enumerate(pairs):
            lists[:, i] = p
        return lists[0], lists[1], lists[2], np.array([len(pairs), missing])


def _shared(rng, pages, rows, width, spare):
    """Rows of random lengths, about half of whose entries are an earlier row's first page; of the other pages all but 'spare' are
    held by somebody else."""
    pool = Pool(pages, rows, width, 64)
    order, at = rng.permutation(pages), 0
    for r in range(rows):
        for j in range(int(rng.integers(1, width + 1))):
            if r and rng.random() < 0.5:
                pool.table[r, j] = pool.table[rng.integers(0, r), 0]
            else:
                pool.table[r, j] = order[at]
                at += 1
    pool.refs = np.bincount(pool.table[pool.table >= 0], minlength=pages).astype(np.int64)
    pool.refs[order[at:pages - spare]] = 1
    return pool


@pytest.mark.parametrize("pages,rows,width,spare", [(40, 9, 6, 9), (40, 9, 6, 0), (40, 9, 6, 2), (600, 120, 7, 200), (600, 120, 7, 20),
                                                    (20000, 60, 40, 10000)])
def test_rows_that_are_their_own_parents(pages, rows, width, spare):
    """Among ordinary pairs: lists, table and references as defined, with enough free pages, few and none."""
    banner(f"pages: rows forked onto themselves, {pages} pages, {rows} x {width}, {spare} spare")
    for seed in range(3):
        rng = np.random.default_rng(100 * pages + spare + seed)
        pool = _shared(rng, pages, rows, width, spare)
        order = rng.permutation(rows)
        alone, up, down = np.array_split(order, 3)
        parents, children = np.concatenate([alone, rng.choice(up, len(down))]), np.concatenate([alone, down])
        mix = rng.permutation(len(parents))
        parents, children = parents[mix], children[mix]
        lens = rng.integers(0, 64 * (pool.table[parents] >= 0).sum(axis=1) + 30)
        lens[::5] = lens[::5] // 64 * 64                   # cuts at a page's end
        held = pool.refs - np.bincount(pool.table[pool.table >= 0], minlength=pages)
        dev = _up(pool)
        lists = pool.fork(parents, children, lens)
        got = tl.kv_fork(dev, _int(parents), _int(children), _int(lens))
        for x, y in zip(got, lists):
            np.testing.assert_array_equal(_get(x), y)
        _same(dev, pool)
        assert (np.bincount(pool.table[pool.table >= 0], minlength=pages) + held == pool.refs).all()


class Run:
    """Rows of a pool with caches of two layers, and what each row's tokens are."""

    def __init__(self, elem, pages, rows, width=6, H=2, Hq=8, D=128, page=64):
        self.elem, self.H, self.Hq, self.D, self.page = elem, H, Hq, D, page
        self.pool = tl.kv_pages(pages, rows, width, page)
        self.caches = [tl.kv_cache(pages, H, D, page, elem) for _ in range(2)]
        self.text = {}

    def len(self, r):
        return len(self.text[r][0][0])

    def write(self, r, number):
        """Pages for so many more tokens of row r, and the tokens."""
        import torch
        layers = self.text.setdefault(r, [([], []) for _ in self.caches])
        n = self.len(r)
        assert _get(tl.kv_grow(self.pool, _int([r]), _int([n + number]))).tolist() == [0]
        table = _get(self.pool.table)
        slots = _int([table[r, t // self.page] * self.page + t % self.page for t in range(n, n + number)])
        for cache, layer in zip(self.caches, layers):
            k, v = (torch.randn((number, self.H, self.D), device="cuda") for _ in range(2))
            tl.kv_append(None, k, v, cache, slots)
            for x, y in zip(layer, (k, v)):
                x.extend(y.unbind())

    def cut(self, r, n):
        self.text[r] = [tuple(x[:n] for x in layer) for layer in self.text[r]]

    def fork(self, parents, children, lens):
        """[pairs, children without a page], the copies made."""
        src, dst, tokens, count = tl.kv_fork(self.pool, _int(parents), _int(children), _int(lens))
        for c in self.caches:
            tl.kv_copy(c, src, dst, tokens, count)
        for p, c, n in zip(parents, children, lens):
            self.text[c] = [tuple(x[:n] for x in layer) for layer in self.text[p]]
        return _get(count).tolist()

    def check(self):
        """Attention over every row is that over a cache of the row alone, bit for bit."""
        import torch
        for r in sorted(self.text):
            n = self.len(r)
            need = -(-n // self.page)
            q = torch.randn((1, self.Hq, self.D), device="cuda").to(torch.bfloat16)
            args = (_int([n]), _int([0, 1]), 1, n, self.D ** -0.5)
            for cache, layer in zip(self.caches, self.text[r]):
                own = tl.kv_cache(need, self.H, self.D, self.page, self.elem)
                k, v = (torch.stack(list(x)) for x in layer)
                tl.kv_append(None, k, v, own, _int(np.arange(n)))
                want = tl.attention(q, own, _int([np.arange(need)]), *args)
                got = tl.attention(q, cache, self.pool.table[r:r + 1].contiguous(), *args)
                torch.cuda.synchronize()
                assert torch.isfinite(got).all() and torch.equal(got, want), f"row {r} of {n} tokens"


@pytest.mark.parametrize("elem", [1, 2, tl.TL_KV_E2M1])
@pytest.mark.parametrize("shorten_first", [False, True])
def test_a_row_cut_inside_a_shared_page_is_written_on(elem, shorten_first):
    """The child, and then the parent, loses tokens back into a page that both share, gets it for itself and goes on: neither
    sees what the other writes."""
    banner(f"pages: rows cut inside shared pages, elem={elem}, shorten_first={shorten_first}")
    run = Run(elem, 20, 3)
    run.write(0, 200)
    assert run.fork([0], [1], [190]) == [1, 0]
    run.check()
    for r, n in ((1, 100), (0, 30)):                       # pages 1 and 0 are shared
        if shorten_first:
            tl.kv_free(run.pool, _int([r]), _int([n]))
        run.cut(r, n)
        assert run.fork([r], [r], [n]) == [1, 0]
        run.check()
        run.write(r, 75)
        run.check()
    # page 0 of row 1 is its own by now: nothing to copy, and no page is taken
    free = int((run.pool.refs == 0).sum())
    run.cut(1, 40)
    assert run.fork([1], [1], [40]) == [0, 0]
    assert int((run.pool.refs == 0).sum()) == free + 2     # its pages 1 and 2
    run.write(1, 50)
    run.check()


def test_nothing_is_lost_where_no_page_is_free():
    banner("pages: rows forked onto themselves without a free page")
    run = Run(1, 5, 3)
    run.write(0, 150)                                      # pages 0 .. 2
    assert run.fork([0], [1], [140]) == [1, 0]             # page 3
    run.write(2, 9)                                        # page 4: none is free
    table = _get(run.pool.table)
    run.cut(1, 100)                                        # shared page 1 stays shared, and page 3 is free then
    assert run.fork([1], [1], [100]) == [0, 1]
    np.testing.assert_array_equal(_get(run.pool.table)[1], [table[1, 0], table[1, 1], -1, -1, -1, -1])
    assert _get(run.pool.refs).tolist() == [2, 2, 1, 0, 1]
    run.check()
    assert run.fork([1], [1], [100]) == [1, 0]             # again, with page 3
    assert _get(run.pool.refs).tolist() == [2, 1, 1, 1, 1]
    run.write(1, 28)
    run.check()
    run.cut(0, 70)                                         # page 1 is row 0's alone now, page 2 is given back
    assert run.fork([0], [0], [70]) == [0, 0]
    run.write(0, 60)
    run.check()


@pytest.mark.parametrize("elem", [2, tl.TL_KV_E2M1])
def test_forks_that_find_too_few_pages_are_repeated(elem):
    """The last of the children that need a page are those without one; forked again once pages are free, and only then given
    pages for more tokens, they are what they would have been."""
    banner(f"pages: forks without free pages, elem={elem}")
    run = Run(elem, 6, 6)
    run.write(0, 100)                                      # pages 0, 1
    run.write(5, 130)                                      # pages 2, 3, 4
    children, lens = [1, 2, 3, 4], [100, 64, 90, 100]      # the second needs no page of its own
    assert run.fork([0] * 4, children, lens) == [1, 2]
    needs = [c for c, n in zip(children, lens) if n % 64]
    short = needs[len(needs) - 2:]
    assert short == [3, 4] and (_get(run.pool.table)[short, 1] == -1).all() and (_get(run.pool.table)[short, 0] >= 0).all()
    for r in short:
        del run.text[r]
    run.check()
    tl.kv_free(run.pool, _int([5]))
    del run.text[5]
    assert run.fork([0, 0], short, [90, 100]) == [2, 0]
    run.check()
    for r in (0, 3, 4):
        run.write(r, 20)
    run.check()
    assert int((run.pool.refs == 0).sum()) == 1            # of six pages one: rows 0, 1, 3 and 4 have a second page each
