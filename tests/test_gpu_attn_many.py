"""tl_attn over many rows or many sequences: 128-row tiles whose waves share their chunks (whole, split and joined), what the
rows do not see in them, more sequences than one scan holds, and more tiles than are split.

The tolerance of every element is that of tests/test_gpu_attn.py: 2^-8 |o| + 1.25 * 2^-8 A."""
import numpy as np
import pytest

import paper_2607_04031_amd as tl
from tests import _serve
from tests._gpu import banner
from tests.test_gpu_attn import Case, _tree

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    import torch
    assert torch.cuda.is_available()
    tl.load_library()
    yield
    torch.cuda.synchronize()


@pytest.mark.parametrize("D,elem,page", [(128, 1, 64), (128, 2, 128), (64, 1, 256), (64, 2, 64)])
@pytest.mark.parametrize("tree", [False, True])
def test_many_rows_over_long_sequences(D, elem, page, tree):
    """128-row tiles whose chunks several workgroups share; pieces that begin and end inside a tile."""
    import torch
    banner(f"attn many rows, split: D={D} elem={elem} page={page} tree={tree}")
    new, lens = [100, 1, 70, 33], [1700, 1100, 130, 33]
    rng = np.random.default_rng(41)
    c = Case(42, lens, new, 6, 2, D, elem, page, mask=np.concatenate([_tree(rng, n, 4) for n in new]) if tree else None)
    out = c.run()
    c.check(out)
    again = c.run()
    torch.cuda.synchronize()
    assert torch.equal(again.view(torch.int16), out.view(torch.int16))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("elem", [1, 2])
@pytest.mark.parametrize("long", [False, True])
def test_many_rows_and_pages_that_are_none(D, elem, long):
    """Pages outside the cache among those that all rows see and among those at the causal edge; what a load of them
    takes instead (the first page) holds NaNs."""
    banner(f"attn many rows, page ids outside the cache: D={D} elem={elem} long={long}")
    lens, new = [400, 260, 1200 if long else 200], [70, 130, 80]
    for seed in range(50, 80):
        c = Case(seed, lens, new, 4, 2, D, elem, 64, spare=6)
        if 0 not in c.table:
            break
    assert 0 not in c.table
    c.table[0, 1], c.table[0, 4], c.table[0, 6] = -5, 10 ** 6, -1         # seen by all; the last two at the edge
    c.table[1, 0], c.table[1, 3] = c.cache.pages, -1
    c.table[2, 1], c.table[2, 2] = -1, 10 ** 9
    c.check(c.run())


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("elem", [1, 2])
@pytest.mark.parametrize("tree", [False, True])
def test_many_rows_and_entries_that_some_do_not_see(D, elem, tree):
    banner(f"attn many rows, NaN and infinities in unseen entries: D={D} elem={elem} tree={tree}")
    rng = np.random.default_rng(60)
    n, L, at = 50, 150, 21
    mask = _tree(rng, n, 2) if tree else None
    c = Case(61, [L], [n], 4, 2, D, elem, 64, mask=mask)
    slot = c.table[0, (L - n + at) // 64] * 64 + (L - n + at) % 64
    k, v = rng.standard_normal((2, D)), rng.standard_normal((2, D))
    k[0, 3] = np.nan
    v[0, 5], v[1, 2] = np.nan, np.nan
    if elem == 2:
        v[1, 9], v[1, D - 1] = np.inf, -np.inf
    c.cache.put(slot, k, v)
    with np.errstate(invalid="ignore"):
        want, size = _serve.attention(c.q, c.cache, c.table, c.lens, c.offsets, c.scale, c.mask)
    got = c.run().cpu().double().numpy()
    for i in range(n):
        sees = i >= at if mask is None else bool(int(mask[i, at // 32]) >> (at % 32) & 1)
        ok = np.ones(D, dtype=bool)
        if sees:
            assert np.isnan(got[i, :2]).all()              # a NaN score
            assert np.isnan(got[i, 2:, 2]).all()
            ok[2] = False
            if elem == 2:
                assert (got[i, 2:, 9] == np.inf).all() and (got[i, 2:, D - 1] == -np.inf).all()
                ok[[9, D - 1]] = False
        for h in range(2 if sees else 0, 4):
            assert np.isfinite(got[i, h, ok]).all()
            assert (np.abs(got[i, h, ok] - want[i, h, ok]) <= 2.0 ** -8 * np.abs(want[i, h, ok]) + 1.25 * 2.0 ** -8 * size[i, h, ok]).all()


@pytest.mark.parametrize("elem", [1, 2])
@pytest.mark.parametrize("most", [4, 20, 60])
def test_more_sequences_than_one_scan_holds(elem, most):
    """70 to 150 sequences, some without a query, some without a key, one long: rows of every tile size."""
    banner(f"attn many sequences: elem={elem} most new tokens={most}")
    rng = np.random.default_rng(70 + most)
    count = 150 if most == 4 else 70
    new = rng.integers(0, most + 1, count)
    lens = new + rng.integers(0, 90, count)
    new[3], lens[3] = most, 1500
    new[64], lens[64] = 0, 5
    new[65], lens[65] = 2, 0
    c = Case(71, lens, new, 4, 2, 64, elem, 64)
    c.check(c.run())


def test_more_tiles_than_are_split():
    banner("attn: as many tiles as fill the chip, one of them long")
    rng = np.random.default_rng(80)
    lens = rng.integers(1, 20, 260)
    lens[100] = 1100
    c = Case(81, lens, [1] * 260, 8, 8, 64, 2, 64)
    c.check(c.run())
