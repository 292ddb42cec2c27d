"""Refusals of the page calls: the documented status before any device work (no GPU here; the addresses are never read)."""
import ctypes

import pytest
import torch

import paper_2607_04031_amd as tl
from tests.test_host_serve import BAD_CACHES, BAD_POINTERS, addr, cache, status


def pool(**kw):
    d = dict(refs=addr(0), page_table=addr(1), num_pages=1000, max_pages=30, num_rows=8, page_tokens=64)
    d.update(kw)
    return tl.KVPagesDesc(*(d[n] for n, _ in tl.KVPagesDesc._fields_))


def grow(pages=None, **kw):
    d = dict(pages=pages or pool(), rows=addr(2), lens=addr(3), n=4, missing=addr(4), stream=0)
    d.update(kw)
    tl.tl_kv_grow(**d)


def free(pages=None, **kw):
    d = dict(pages=pages or pool(), rows=addr(2), lens=addr(3), n=4, stream=0)
    d.update(kw)
    tl.tl_kv_free(**d)


def fork(pages=None, **kw):
    d = dict(pages=pages or pool(), parents=addr(2), children=addr(3), lens=addr(4), n=4, src=addr(5), dst=addr(6), tokens=addr(7), count=addr(8), stream=0)
    d.update(kw)
    tl.tl_kv_fork(**d)


def compact(pages=None, **kw):
    d = dict(pages=pages or pool(), max_moves=10, src=addr(5), dst=addr(6), count=addr(8), stream=0)
    d.update(kw)
    tl.tl_kv_compact(**d)


BAD_POOLS = [(dict(refs=None), tl.TL_EINVAL), (dict(refs=addr(0) + 2), tl.TL_EINVAL), (dict(page_table=None), tl.TL_EINVAL),
             (dict(page_table=addr(1) + 1), tl.TL_EINVAL), (dict(num_pages=0), tl.TL_EINVAL), (dict(max_pages=0), tl.TL_EINVAL),
             (dict(num_rows=0), tl.TL_EINVAL), (dict(page_tokens=32), tl.TL_EINVAL), (dict(page_tokens=96), tl.TL_EINVAL),
             (dict(page_tokens=8192), tl.TL_EINVAL), (dict(num_pages=1 << 25), tl.TL_EINVAL), (dict(max_pages=1 << 31), tl.TL_EUNSUPPORTED),
             (dict(max_pages=(1 << 25) + 1), tl.TL_EUNSUPPORTED), (dict(max_pages=1 << 25, num_rows=(1 << 15) + 1), tl.TL_EUNSUPPORTED),
             (dict(page_table=addr(0) + 3996), tl.TL_EINVAL), (dict(refs=addr(1) + 8 * 30 * 4 - 4), tl.TL_EINVAL)]


@pytest.mark.parametrize("call", [grow, free, fork, compact])
def test_bad_pools(call):
    for kw, want in BAD_POOLS:
        assert status(call, pages=pool(**kw)) == want, kw
    lib = tl.load_library()
    assert lib.tl_kv_compact(None, 1, addr(5), addr(6), addr(8), None) == tl.TL_EINVAL


def test_bad_lists():
    for kw in (dict(rows=None), dict(lens=None), dict(rows=addr(2) + 2), dict(n=-1), dict(missing=None), dict(missing=addr(4) + 1),
               dict(missing=addr(2) + 12), dict(missing=addr(0)), dict(rows=addr(1) + 4), dict(lens=addr(0) + 3996)):
        assert status(grow, **kw) == tl.TL_EINVAL, kw
    for kw in (dict(rows=None), dict(rows=addr(2) + 2), dict(n=-1), dict(rows=addr(1)), dict(lens=addr(0)), dict(lens=addr(3) + 2)):
        assert status(free, **kw) == tl.TL_EINVAL, kw
    for kw in (dict(parents=None), dict(children=None), dict(lens=None), dict(src=None), dict(dst=None), dict(tokens=None), dict(count=None),
               dict(n=-1), dict(src=addr(6) + 12), dict(tokens=addr(5) + 4), dict(count=addr(7) + 12), dict(dst=addr(2)), dict(count=addr(4)),
               dict(src=addr(0)), dict(tokens=addr(1)), dict(parents=addr(1)), dict(dst=addr(6) + 2)):
        assert status(fork, **kw) == tl.TL_EINVAL, kw
    for kw in (dict(max_moves=-1), dict(src=None), dict(dst=None), dict(count=None), dict(src=addr(6) + 36), dict(count=addr(5) + 36),
               dict(dst=addr(0)), dict(src=addr(1)), dict(count=addr(1)), dict(src=addr(5) + 1)):
        assert status(compact, **kw) == tl.TL_EINVAL, kw
    for call, kw in ((grow, dict(n=65537)), (free, dict(n=65537)), (fork, dict(n=65537)), (compact, dict(max_moves=1 << 31))):
        assert status(call, **kw) == tl.TL_EUNSUPPORTED, kw
    assert status(free, n=0, rows=None) == tl.TL_OK


def test_copy_refusals():
    def copy(cache=None, **kw):
        d = dict(cache=cache, src=addr(7), dst=addr(8), tokens=addr(9), count=addr(10), max_pairs=5, stream=0)
        d.update(kw)
        tl.tl_kv_copy(**d)
    for kw, want in BAD_CACHES + BAD_POINTERS:
        assert status(copy, cache=cache(**kw)) == want, kw
    for elem in (1, tl.TL_KV_E2M1):
        data, exps = tl.tl_kv_bytes(cache(elem_bytes=elem))
        for kw, want in [(dict(max_pairs=-1), tl.TL_EINVAL), (dict(src=None), tl.TL_EINVAL), (dict(dst=None), tl.TL_EINVAL), (dict(src=addr(7) + 2), tl.TL_EINVAL),
                         (dict(tokens=addr(9) + 1), tl.TL_EINVAL), (dict(count=addr(10) + 2), tl.TL_EINVAL), (dict(src=addr(0) + data - 4), tl.TL_EINVAL),
                         (dict(tokens=addr(1)), tl.TL_EINVAL), (dict(count=addr(2) + exps - 4), tl.TL_EINVAL), (dict(dst=addr(3)), tl.TL_EINVAL),
                         (dict(max_pairs=1 << 31), tl.TL_EUNSUPPORTED)]:
            assert status(copy, cache=cache(elem_bytes=elem), **kw) == want, kw
    assert status(copy, cache=cache(v=addr(0) + 16)) == tl.TL_EINVAL
    assert status(copy, cache=cache(), max_pairs=0, src=None, dst=None) == tl.TL_OK


def test_helpers_refuse_other_tensors():
    i32 = torch.int32
    for refs, table in ((torch.zeros(4, dtype=torch.int64), torch.zeros((2, 3), dtype=i32)), (torch.zeros(4, dtype=i32), torch.zeros((2, 3))),
                        (torch.zeros((2, 2), dtype=i32), torch.zeros((2, 3), dtype=i32)), (torch.zeros(4, dtype=i32), torch.zeros(6, dtype=i32))):
        with pytest.raises(ValueError, match="int32"):
            tl.KVPages(refs, table, 64)
    with pytest.raises(ValueError, match="device tensors"):
        tl.KVPages(torch.zeros(4, dtype=i32), torch.zeros((2, 3), dtype=i32), 64)
    with pytest.raises(ValueError, match="out holds"):
        tl._lists(3, "cpu", (torch.zeros(3, dtype=i32), torch.zeros(3, dtype=i32)), 3, 2)
    assert [x.numel() for x in tl._lists(3, "cpu", None, 3, 2)] == [3, 2]
    assert ctypes.sizeof(tl.KVPagesDesc) == 40
