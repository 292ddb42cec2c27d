"""The page calls at their largest number of rows, and a compaction that may move nothing."""
import numpy as np
import pytest

import paper_2607_04031_amd as tl
from tests import _pool
from tests._gpu import banner
from tests.test_gpu_kv import _int, _lib  # noqa: F401
from tests.test_gpu_pages import _get, _same, _up

pytestmark = pytest.mark.gpu


def test_65536_rows():
    banner("pages: 65536 rows grown, forked and cut at once")
    n, width = 65536, 2
    rng = np.random.default_rng(41)
    pool = _pool.Pool(2 * n, 2 * n, width, 64)
    dev = _up(pool)
    rows = rng.permutation(2 * n)
    up, down = rows[:n], rows[n:]
    lens = rng.integers(0, 129, n)
    assert pool.grow(up, lens) == _get(tl.kv_grow(dev, _int(up), _int(lens)))[0] == 0
    _same(dev, pool)
    parents = rng.integers(0, n, n)
    cut = np.maximum(lens[parents] - rng.integers(0, 30, n), 0)
    lists = pool.fork(up[parents], down, cut)
    assert lists[3][1] > 0                                 # there are pages for some of them only
    for x, y in zip(tl.kv_fork(dev, _int(up[parents]), _int(down), _int(cut)), lists):
        np.testing.assert_array_equal(_get(x), y)
    _same(dev, pool)
    pool.free(up, lens // 2)
    tl.kv_free(dev, _int(up), _int(lens // 2))
    _same(dev, pool)
    want = np.full(n, 128)
    missing = pool.grow(up, want)
    assert missing > 0 and _get(tl.kv_grow(dev, _int(up), _int(want)))[0] == missing
    _same(dev, pool)
    assert pool.counts_hold()


@pytest.mark.parametrize("pages,rows,width", [(30, 4, 6), (20000, 40, 200)])
def test_compact_counts_the_pages_in_use_where_it_moves_none(pages, rows, width):
    banner(f"pages compact: no moves, {pages} pages")
    pool, _ = _pool.filled(np.random.default_rng(1), pages, rows, width, 64, 0.5)
    dev = _up(pool)
    src, dst, count = tl.kv_compact(dev, 0)
    assert _get(count).tolist() == [0, int((pool.refs > 0).sum())] and src.numel() == dst.numel() == 0
    _same(dev, pool)
