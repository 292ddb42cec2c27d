"""The pages of a pool: tl_kv_grow, tl_kv_free, tl_kv_fork and tl_kv_compact against the definition, whole numbers and so
equal, and tl_kv_copy byte for byte in caches of every element type."""
import copy

import numpy as np
import pytest

import paper_2607_04031_amd as tl
from tests import _pool, _serve
from tests._gpu import banner
from tests.test_gpu_kv import _int, _lib  # noqa: F401

pytestmark = pytest.mark.gpu
# (pages, rows, width): one workgroup, several, a last block of pages that is full, one page, more rows than waves
SIZES = [(25, 4, 9), (200, 40, 20), (4096, 16, 300), (15485, 64, 210), (9000, 500, 33), (1, 1, 1), (4097, 2, 2500), (300000, 70, 600)]


def _up(pool):
    import torch
    return tl.KVPages(_int(pool.refs), _int(pool.table), pool.page) if torch.cuda.is_available() else None


def _same(pages, pool):
    np.testing.assert_array_equal(pages.table.cpu().numpy(), pool.table)
    np.testing.assert_array_equal(pages.refs.cpu().numpy(), pool.refs)


def _get(x):
    return x.cpu().numpy()


@pytest.mark.parametrize("pages,rows,width", SIZES)
@pytest.mark.parametrize("load", [0.0, 0.5, 0.97])
def test_grow(pages, rows, width, load):
    banner(f"pages grow: {pages} pages, {rows} x {width}, load {load}")
    rng = np.random.default_rng(pages + rows)
    pool, lens = _pool.filled(rng, pages, rows, width, 64, load)
    some = rng.permutation(rows)[:max(1, rows - 1)]
    for r in some[:3]:                                     # holes, and entries past the sequence
        pool.let_go(r, width // 2)
        if pool.table[r, 0] >= 0:
            pool.refs[pool.table[r, 0]] -= 1
            pool.table[r, 0] = -7
    want = np.minimum(lens[some] + rng.integers(0, 200, len(some)), 2 ** 31 - 1)
    want[0] = width * 64 + 1000                            # more than the table holds
    dev = _up(pool)
    missing = pool.grow(some, want)
    assert _get(tl.kv_grow(dev, _int(some), _int(want)))[0] == missing
    _same(dev, pool)
    assert pool.counts_hold()


def test_grow_missing_past_31_bits():
    import torch
    banner("pages grow: a row of 2^25 entries, named 66 times, one page")
    width = 2 ** 25                                        # 66 * 2^25 - 1 entries go without: more than int32 holds
    dev = tl.kv_pages(1, 1, width)
    missing = tl.kv_grow(dev, torch.zeros(66, dtype=torch.int32, device="cuda"), torch.full((66,), 2 ** 31 - 1, dtype=torch.int32, device="cuda"))
    assert missing.tolist() == [2 ** 31 - 1] and dev.refs.tolist() == [1]
    assert int(dev.table[0, 0]) == 0 and int((dev.table == -1).sum()) == width - 1


@pytest.mark.parametrize("pages,rows,width", SIZES)
def test_free(pages, rows, width):
    banner(f"pages free: {pages} pages, {rows} x {width}")
    rng = np.random.default_rng(pages + 1)
    pool, lens = _pool.filled(rng, pages, rows, width, 128, 0.9)
    dev = _up(pool)
    some = rng.permutation(rows)[:max(1, rows // 2)]
    keep = lens[some] // 2
    pool.free(some, keep)
    tl.kv_free(dev, _int(some), _int(keep))
    _same(dev, pool)
    some = np.concatenate([some, some[:2], [-1, rows, 2 ** 31 - 1, -2 ** 31]])       # rows twice, rows that are none
    pool.free(some)
    tl.kv_free(dev, _int(some))
    _same(dev, pool)
    assert pool.counts_hold()


@pytest.mark.parametrize("pages,rows,width", SIZES)
@pytest.mark.parametrize("load", [0.5, 0.97])
def test_fork(pages, rows, width, load):
    banner(f"pages fork: {pages} pages, {rows} x {width}, load {load}")
    rng = np.random.default_rng(pages + 2)
    pool, lens = _pool.filled(rng, pages, rows, width, 64, load)
    order = rng.permutation(rows)
    up, children = order[:max(1, rows // 3)], order[max(1, rows // 3):]
    if rows == 1:
        up, children = np.array([0]), np.array([], dtype=np.int64)
    parents = rng.choice(up, len(children))
    want = np.maximum(lens[parents] - rng.integers(0, 130, len(children)), 0)
    if len(children) > 3:
        parents[0], children[1], want[2] = -1, rows + 5, 2 ** 31 - 1
    dev = _up(pool)
    lists = pool.fork(parents, children, want)
    got = tl.kv_fork(dev, _int(parents), _int(children), _int(want))
    for x, y in zip(got, lists):
        np.testing.assert_array_equal(_get(x), y)
    _same(dev, pool)
    assert pool.counts_hold()


@pytest.mark.parametrize("pages,rows,width", SIZES)
@pytest.mark.parametrize("load,part", [(0.0, False), (0.5, False), (0.5, True), (0.97, False), (1.0, False)])
def test_compact(pages, rows, width, load, part):
    banner(f"pages compact: {pages} pages, {rows} x {width}, load {load} part={part}")
    rng = np.random.default_rng(pages + 3)
    pool, _ = _pool.filled(rng, pages, rows, width, 64, load)
    pool.let_go(0, width - 1)
    pool.table[0, -1] = pages + 3                          # an entry that is no page stays
    most = 7 if part else pages // 2 + 1
    dev = _up(pool)
    lists = pool.compact(most)
    got = tl.kv_compact(dev, most)
    for x, y in zip(got, lists):
        np.testing.assert_array_equal(_get(x), y)
    _same(dev, pool)
    assert pool.counts_hold()
    if not part:                                           # nothing is left to do
        used = int((pool.refs > 0).sum())
        assert not pool.refs[used:].any()
        src, dst, count = tl.kv_compact(dev, 3)
        assert _get(count).tolist() == [0, used] and (_get(src) == -1).all() and (_get(dst) == -1).all()
        _same(dev, pool)


def test_empty_lists():
    import torch
    banner("pages: nothing to do")
    pool, _ = _pool.filled(np.random.default_rng(1), 30, 4, 6, 64, 0.5)
    dev, none = _up(pool), _int([]).reshape(0)
    assert _get(tl.kv_grow(dev, none, none))[0] == 0
    tl.kv_free(dev, none)
    count = torch.full((2,), 9, dtype=torch.int32, device="cuda")
    tl.kv_fork(dev, none, none, none, out=(none, none, none, count))
    assert _get(count).tolist() == [0, 0]
    src, dst, count = tl.kv_compact(dev, 0)
    assert _get(count).tolist() == [0, 15] or _get(count)[0] == 0
    _same(dev, pool)


@pytest.mark.parametrize("rows", [6, 300])
def test_rows_named_twice_keep_the_counts(rows):
    """Which pages or tokens such rows get is not specified; that every entry holds one reference is."""
    banner(f"pages: rows named twice, {rows} rows")
    for seed in range(3):
        rng = np.random.default_rng(seed)
        pool, lens = _pool.filled(rng, 3000, rows, 20, 64, 0.6)
        dev = _up(pool)
        twice = np.concatenate([np.arange(rows)] * 2)
        tl.kv_grow(dev, _int(twice), _int(np.concatenate([lens + 200] * 2)))
        after = copy.deepcopy(pool)
        after.table, after.refs = _get(dev.table).astype(np.int64), _get(dev.refs).astype(np.int64)
        assert after.counts_hold()
        for r in range(rows):
            assert (after.table[r, :after.pages(lens[r] + 200)] >= 0).all()
        again = rng.integers(0, rows, 3 * rows)            # children twice, children that are parents, their own parents
        tl.kv_fork(dev, _int(rng.integers(0, rows, 3 * rows)), _int(again), _int(rng.integers(0, 20 * 64, 3 * rows)))
        after.table, after.refs = _get(dev.table).astype(np.int64), _get(dev.refs).astype(np.int64)
        assert after.counts_hold()


@pytest.mark.parametrize("D,elem,H,page", [(128, 1, 2, 64), (64, 1, 3, 128), (128, 2, 1, 256), (64, 2, 2, 64), (128, tl.TL_KV_E2M1, 2, 128),
                                           (64, tl.TL_KV_E2M1, 3, 64)])
@pytest.mark.parametrize("pairs", [5, 700])
def test_copy(D, elem, H, page, pairs):
    import torch
    banner(f"pages copy: D={D} elem={elem} H={H} page={page} pairs={pairs}")
    rng = np.random.default_rng(D + pairs)
    pages = 2 * pairs + 3
    cache = tl.kv_cache(pages, H, D, page, elem)
    arrays = [x for x in (cache.k, cache.v, cache.k_exp, cache.v_exp) if x is not None]
    for x in arrays:
        x.view(torch.uint8).copy_(torch.randint(0, 256, x.view(torch.uint8).shape, dtype=torch.uint8, device="cuda"))
    order = rng.permutation(pages)
    src, dst = order[:pairs].copy(), order[pairs:2 * pairs].copy()
    tokens = rng.integers(-3, page + 5, pairs)
    if pairs > 10:
        src[3], dst[4], src[5], dst[6], dst[7] = -1, -2, pages, 2 ** 31 - 1, src[7]
    before = [x.view(torch.uint8).cpu().numpy().copy() for x in arrays]

    def want(number, tokens):
        out = [x.copy() for x in before]
        for i in range(number):
            a, b = src[i], dst[i]
            if 0 <= a < pages and 0 <= b < pages:
                groups = min(page // 64, max(0, -(-(page if tokens is None else int(tokens[i])) // 64)))
                for x, y in zip(out, before):
                    x[b].reshape(H, page // 64, -1)[:, :groups] = y[a].reshape(H, page // 64, -1)[:, :groups]
        return out

    def check(number, tokens):
        torch.cuda.synchronize()
        for x, y in zip(arrays, want(number, tokens)):
            np.testing.assert_array_equal(x.view(torch.uint8).cpu().numpy(), y)
        for x, y in zip(arrays, before):
            x.view(torch.uint8).copy_(torch.from_numpy(y))

    tl.kv_copy(cache, _int(src), _int(dst), _int(tokens))
    check(pairs, tokens)
    tl.kv_copy(cache, _int(src), _int(dst), count=_int([pairs - 2, 99]))
    check(pairs - 2, None)
    tl.kv_copy(cache, _int(src), _int(dst), count=_int([pairs + 100]))
    check(pairs, None)
    for none in (0, -5):
        tl.kv_copy(cache, _int(src), _int(dst), count=_int([none]))
        check(0, None)


def test_copy_past_four_gigabytes():
    import torch
    banner("pages copy past 2^32 bytes")
    pages, H, D, page = 36000, 8, 128, 128
    cache = tl.kv_cache(pages, H, D, page, 1)
    cache.k[17].fill_(3), cache.v[35999].fill_(5), cache.k_exp[17].fill_(7), cache.v_exp[35999].fill_(11)
    tl.kv_copy(cache, _int([17, 35999]), _int([35998, 0]))
    torch.cuda.synchronize()
    assert (cache.k[35998] == 3).all() and (cache.v[0] == 5).all() and (cache.k_exp[35998] == 7).all() and (cache.v_exp[0] == 11).all()


@pytest.mark.parametrize("pages,rows,width", [(60, 6, 9), (12000, 200, 50)])
def test_streams_and_graph_replay(pages, rows, width):
    """Every call on a stream of its own and in a graph, replayed between eager work on other pools."""
    import torch
    banner(f"pages in a graph: {pages} pages")
    rng = np.random.default_rng(5)
    work, lens = _pool.filled(rng, pages, rows, width, 64, 0.5)
    dev, side = _up(work), torch.cuda.Stream()
    half = rows // 2
    a, b, c = np.arange(half), np.arange(half, rows), np.arange(0, rows, 2)
    at, bt, ct, lt = _int(a), _int(b), _int(c), _int(lens[:half])
    gt = _int(lens[c] + 70)
    out = tuple(torch.empty(half, dtype=torch.int32, device="cuda") for _ in range(3)) + (torch.empty(2, dtype=torch.int32, device="cuda"),)
    most = pages // 2 + 1
    moves = (torch.empty(most, dtype=torch.int32, device="cuda"), torch.empty(most, dtype=torch.int32, device="cuda"),
             torch.empty(2, dtype=torch.int32, device="cuda"))
    missing = torch.empty(1, dtype=torch.int32, device="cuda")
    parents, children = at[:half], bt[:half]

    def calls():
        tl.kv_fork(dev, parents, children, lt, out=out)
        tl.kv_free(dev, ct)
        tl.kv_grow(dev, ct, gt, missing=missing)
        tl.kv_compact(dev, most, out=moves)

    def by_definition(pool):
        lists = pool.fork(a[:half], b[:half], lens[:half])
        pool.free(c)
        short = pool.grow(c, lens[c] + 70)
        return list(lists) + list(pool.compact(most)) + [np.array([short])]

    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        calls()
    side.synchronize()
    lists = by_definition(work)
    for x, y in zip(list(out) + list(moves) + [missing], lists):
        np.testing.assert_array_equal(_get(x), y)
    _same(dev, work)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        calls()
    for step in range(3):
        work, now = _pool.filled(np.random.default_rng(6 + step), pages, rows, width, 64, 0.5)
        lens[:] = now
        dev.refs.copy_(_int(work.refs)), dev.table.copy_(_int(work.table)), lt.copy_(_int(lens[:half])), gt.copy_(_int(lens[c] + 70))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        lists = by_definition(work)
        for x, y in zip(list(out) + list(moves) + [missing], lists):
            np.testing.assert_array_equal(_get(x), y)
        _same(dev, work)
        other, _ = _pool.filled(np.random.default_rng(60 + step), 500, 20, 30, 64, 0.5)
        tl.kv_compact(_up(other), 300)
        assert torch.isfinite(torch.randn(1000, device="cuda").sum())


@pytest.mark.parametrize("elem", [1, 2, tl.TL_KV_E2M1])
def test_a_serving_run_over_one_pool(elem):
    """Prompts, forks, samples of their own, an end, a compaction: attention over the pool gives at every step what it gives
    over caches of each sequence alone, bit for bit."""
    import torch
    banner(f"pages: a run with forks and compactions, elem={elem}")
    H, Hq, D, page, layers = 2, 8, 128, 64, 2
    rows, width, pages = 12, 8, 70
    rng = np.random.default_rng(17)
    pool = tl.kv_pages(pages, rows, width, page)
    caches = [tl.kv_cache(pages, H, D, page, elem) for _ in range(layers)]
    text = {}                                              # row -> [layers][keys and values] of its tokens

    def check():
        live = sorted(text)
        lens = [len(text[r][0][0]) for r in live]
        q = torch.randn((len(live), Hq, D), device="cuda").to(torch.bfloat16)
        for layer in range(layers):
            own = tl.kv_cache(sum(-(-n // page) for n in lens), H, D, page, elem)
            table, at = torch.full((len(live), width), -1, dtype=torch.int32), 0
            for i, r in enumerate(live):
                need = -(-lens[i] // page)
                table[i, :need] = torch.arange(at, at + need)
                k, v = (torch.stack(x) for x in text[r][layer])
                tl.kv_append(None, k, v, own, at * page + torch.arange(lens[i], dtype=torch.int32, device="cuda"))
                at += need
            args = (_int(lens), _int(range(len(live) + 1)), 1, max(lens), D ** -0.5)
            want = tl.attention(q, own, table.cuda(), *args)
            got = tl.attention(q, caches[layer], pool.table[torch.tensor(live, device="cuda")].contiguous(), *args)
            torch.cuda.synchronize()
            assert torch.isfinite(got).all() and torch.equal(got, want)

    def write(news):
        """{row: number of new tokens}"""
        live = sorted(news)
        lens = [len(text[r][0][0]) if r in text else 0 for r in live]
        assert _get(tl.kv_grow(pool, _int(live), _int([n + news[r] for r, n in zip(live, lens)])))[0] == 0
        table = _get(pool.table)
        for r, n in zip(live, lens):
            slots = _int([table[r, t // page] * page + t % page for t in range(n, n + news[r])])
            for layer in range(layers):
                k, v = (torch.randn((news[r], H, D), device="cuda") for _ in range(2))
                tl.kv_append(None, k, v, caches[layer], slots)
                for x, y in zip(text.setdefault(r, [([], []) for _ in range(layers)])[layer], (k, v)):
                    x.extend(y.unbind())

    write({0: 130, 1: 64, 2: 7})
    check()
    for step in range(6):
        live = sorted(text)
        spare = [r for r in range(rows) if r not in text]
        children = spare[:3]
        parents = [int(rng.choice(live)) for _ in children]
        lens = [len(text[r][0][0]) - int(rng.integers(0, 2)) for r in parents]
        src, dst, tokens, count = tl.kv_fork(pool, _int(parents), _int(children), _int(lens))
        assert _get(count)[1] == 0
        for c in caches:
            tl.kv_copy(c, src, dst, tokens, count)
        for p, c, n in zip(parents, children, lens):
            text[c] = [tuple(x[:n] for x in layer) for layer in text[p]]
        write({r: int(rng.integers(1, 40)) for r in sorted(text)})
        check()
        ended = [int(r) for r in rng.permutation(sorted(text))[:len(text) // 2]]
        tl.kv_free(pool, _int(ended))
        for r in ended:
            del text[r]
        src, dst, count = tl.kv_compact(pool, pages)
        for c in caches:
            tl.kv_copy(c, src, dst, count=count)
        check()
        used = len({int(p) for p in _get(pool.table).flatten() if p >= 0})
        assert _get(count)[1] == used and not _get(pool.refs)[used:].any()
