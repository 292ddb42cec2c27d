"""Refusals of the serving-step entry points: the documented status before any
device work (no GPU here; the addresses are never read), and the helpers'
checks of tensors."""
import ctypes

import pytest

import paper_2607_04031_amd as tl

A = 1 << 20                # addresses far apart, 16-byte aligned


def addr(i):
    return (i + 1) << 40


def cache(**kw):
    d = dict(k=addr(0), v=addr(1), k_exp=addr(2), v_exp=addr(3), num_pages=10, page_tokens=64, kv_heads=8, head_dim=128, elem_bytes=1)
    d.update(kw)
    return tl.KVCacheDesc(*(d[n] for n, _ in tl.KVCacheDesc._fields_))


def status(call, **kw):
    try:
        call(**kw)
    except tl.TLError as e:
        return e.status
    return tl.TL_OK


BAD_CACHES = [(dict(num_pages=0), tl.TL_EINVAL), (dict(page_tokens=32), tl.TL_EINVAL), (dict(page_tokens=96), tl.TL_EINVAL),
              (dict(page_tokens=8192), tl.TL_EINVAL), (dict(kv_heads=0), tl.TL_EINVAL), (dict(kv_heads=1025), tl.TL_EINVAL),
              (dict(elem_bytes=4), tl.TL_EINVAL), (dict(num_pages=1 << 25), tl.TL_EINVAL), (dict(head_dim=96), tl.TL_EUNSUPPORTED)]


def test_kv_bytes():
    assert tl.tl_kv_bytes(cache()) == (10 * 64 * 8 * 128, 10 * 64 * 8)
    assert tl.tl_kv_bytes(cache(elem_bytes=2, head_dim=64, page_tokens=4096)) == (10 * 4096 * 8 * 64 * 2, 0)
    for kw, want in BAD_CACHES:
        assert status(tl.tl_kv_bytes, cache=cache(**kw)) == want, kw
    lib, n = tl.load_library(), ctypes.c_int64()
    assert lib.tl_kv_bytes(ctypes.byref(cache()), None, ctypes.byref(n)) == tl.TL_EINVAL
    assert lib.tl_kv_bytes(None, ctypes.byref(n), ctypes.byref(n)) == tl.TL_EINVAL


BAD_POINTERS = [(dict(k=None), tl.TL_EINVAL), (dict(v=addr(1) + 8), tl.TL_EINVAL), (dict(k_exp=None), tl.TL_EINVAL),
                (dict(v_exp=addr(3) + 4), tl.TL_EINVAL)]


def append(cache=None, rope=None, **kw):
    d = dict(Q=addr(4), ldq=64 * 128, K=addr(5), ldk=1024, V=addr(6), ldv=1024, in_dtype=tl.TL_IN_BF16, n=5, q_heads=64, slots=addr(7),
             rope=rope, Q_out=addr(8), cache=cache, stream=0)
    d.update(kw)
    tl.tl_kv_append(**d)


def rope(**kw):
    d = dict(positions=addr(9), inv_freq=addr(10), rot_dim=128, axes=1, sections=(64, 0, 0), interleaved=0)
    d.update(kw)
    return tl.RopeDesc(d["positions"], d["inv_freq"], d["rot_dim"], d["axes"], (ctypes.c_int32 * 3)(*d["sections"]), d["interleaved"])


def test_append_refusals():
    for kw, want in BAD_CACHES + BAD_POINTERS:
        assert status(append, cache=cache(**kw)) == want, kw
    for kw, want in [(dict(n=-1), tl.TL_EINVAL), (dict(q_heads=-1), tl.TL_EINVAL), (dict(in_dtype=2), tl.TL_EINVAL),
                     (dict(K=None), tl.TL_EINVAL), (dict(V=None), tl.TL_EINVAL), (dict(Q=None), tl.TL_EINVAL), (dict(Q_out=None), tl.TL_EINVAL),
                     (dict(Q=None, Q_out=None, q_heads=0, K=None, V=None), tl.TL_EINVAL), (dict(slots=None), tl.TL_EINVAL),
                     (dict(slots=addr(7) + 2), tl.TL_EINVAL), (dict(Q=addr(4) + 8), tl.TL_EINVAL), (dict(Q_out=addr(8) + 2), tl.TL_EINVAL),
                     (dict(ldk=1023), tl.TL_EINVAL), (dict(ldk=1028), tl.TL_EINVAL), (dict(ldv=1 << 31), tl.TL_EUNSUPPORTED),
                     (dict(q_heads=5000, ldq=5000 * 128), tl.TL_EUNSUPPORTED), (dict(n=1 << 30), tl.TL_EUNSUPPORTED),
                     (dict(Q_out=addr(4) + 16), tl.TL_EINVAL), (dict(Q_out=addr(0)), tl.TL_EINVAL), (dict(K=addr(2)), tl.TL_EINVAL),
                     (dict(V=addr(1) + 160), tl.TL_EINVAL)]:
        assert status(append, cache=cache(), **kw) == want, kw
    for kw in (dict(axes=0), dict(axes=4), dict(rot_dim=8), dict(rot_dim=144), dict(rot_dim=40), dict(positions=None), dict(inv_freq=addr(10) + 1),
               dict(sections=(63, 0, 0)), dict(axes=2, sections=(65, -1, 0)), dict(axes=2, sections=(32, 31, 1))):
        assert status(append, cache=cache(), rope=rope(**kw)) == tl.TL_EINVAL, kw
    assert status(append, cache=cache(), n=0, Q=None, K=None, V=None, slots=None, Q_out=None) == tl.TL_OK


def test_read_refusals():
    def read(cache=None, **kw):
        d = dict(cache=cache, slots=addr(7), n=5, K_out=addr(8), V_out=addr(9), stream=0)
        d.update(kw)
        tl.tl_kv_read(**d)
    for kw, want in BAD_CACHES + BAD_POINTERS:
        assert status(read, cache=cache(**kw)) == want, kw
    for kw, want in [(dict(n=-1), tl.TL_EINVAL), (dict(slots=None), tl.TL_EINVAL), (dict(K_out=None, V_out=None), tl.TL_EINVAL),
                     (dict(K_out=addr(8) + 2), tl.TL_EINVAL), (dict(V_out=addr(8) + 64), tl.TL_EINVAL), (dict(K_out=addr(0) + 1024), tl.TL_EINVAL),
                     (dict(V_out=addr(3)), tl.TL_EINVAL), (dict(K_out=addr(7)), tl.TL_EINVAL), (dict(n=1 << 40), tl.TL_EUNSUPPORTED)]:
        assert status(read, cache=cache(), **kw) == want, kw
    assert status(read, cache=cache(), n=0, slots=None) == tl.TL_OK


def test_keep_refusals():
    def keep(cache=None, **kw):
        d = dict(cache=cache, page_table=addr(7), max_pages=4, starts=addr(8), path=addr(9), max_path=6, counts=addr(10), num_seqs=3, stream=0)
        d.update(kw)
        tl.tl_kv_keep(**d)
    for kw, want in BAD_CACHES + BAD_POINTERS:
        assert status(keep, cache=cache(**kw)) == want, kw
    for kw, want in [(dict(num_seqs=-1), tl.TL_EINVAL), (dict(max_pages=0), tl.TL_EINVAL), (dict(max_path=0), tl.TL_EINVAL),
                     (dict(page_table=None), tl.TL_EINVAL), (dict(starts=None), tl.TL_EINVAL), (dict(path=addr(9) + 1), tl.TL_EINVAL),
                     (dict(counts=None), tl.TL_EINVAL), (dict(max_path=4097), tl.TL_EUNSUPPORTED), (dict(num_seqs=1 << 29), tl.TL_EUNSUPPORTED)]:
        assert status(keep, cache=cache(), **kw) == want, kw
    assert status(keep, cache=cache(), num_seqs=0, path=None) == tl.TL_OK


def test_attn_refusals():
    def attn(cache=None, **kw):
        d = dict(Q=addr(4), ldq=64 * 128, cache=cache, page_table=addr(7), max_pages=4, lens=addr(8), q_offsets=addr(9), mask=addr(10), mask_words=2,
                 num_seqs=3, total_q=12, max_q=6, max_len=200, q_heads=64, scale=0.1, O=addr(11), stream=0)
        d.update(kw)
        tl.tl_attn(**d)
    for kw, want in BAD_CACHES + BAD_POINTERS:
        assert status(attn, cache=cache(**kw)) == want, kw
    for kw, want in [(dict(num_seqs=-1), tl.TL_EINVAL), (dict(total_q=-1), tl.TL_EINVAL), (dict(max_q=-1), tl.TL_EINVAL), (dict(max_len=-1), tl.TL_EINVAL),
                     (dict(max_pages=0), tl.TL_EINVAL), (dict(q_heads=0), tl.TL_EINVAL), (dict(q_heads=60), tl.TL_EINVAL), (dict(scale=0.0), tl.TL_EINVAL),
                     (dict(scale=-1.0), tl.TL_EINVAL), (dict(scale=float("inf")), tl.TL_EINVAL), (dict(scale=float("nan")), tl.TL_EINVAL),
                     (dict(mask_words=0), tl.TL_EINVAL), (dict(mask=addr(10) + 2), tl.TL_EINVAL), (dict(Q=None), tl.TL_EINVAL), (dict(O=addr(11) + 8), tl.TL_EINVAL),
                     (dict(lens=None), tl.TL_EINVAL), (dict(q_offsets=None), tl.TL_EINVAL), (dict(page_table=None), tl.TL_EINVAL),
                     (dict(ldq=8191), tl.TL_EINVAL), (dict(ldq=8196), tl.TL_EINVAL), (dict(O=addr(4)), tl.TL_EINVAL), (dict(O=addr(1)), tl.TL_EINVAL),
                     (dict(O=addr(10)), tl.TL_EINVAL), (dict(O=addr(7)), tl.TL_EINVAL), (dict(ldq=1 << 31), tl.TL_EUNSUPPORTED),
                     (dict(max_len=1 << 31), tl.TL_EUNSUPPORTED), (dict(total_q=1 << 26), tl.TL_EUNSUPPORTED), (dict(mask_words=1 << 17), tl.TL_EUNSUPPORTED)]:
        assert status(attn, cache=cache(), **kw) == want, kw
    for kw in (dict(num_seqs=0, lens=None), dict(total_q=0, Q=None, O=None)):
        assert status(attn, cache=cache(), **kw) == tl.TL_OK


def test_verify_refusals():
    def verify(**kw):
        d = dict(logits=addr(0), logits_dtype=tl.TL_OUT_BF16, vocab=1000, node_offsets=addr(1), parents=addr(2), tokens=addr(3), num_seqs=4,
                 total_nodes=20, max_nodes=8, draft=addr(4), draft_dtype=tl.TL_OUT_F32, temperature=addr(5), uniform=addr(6), noise=addr(7),
                 path=addr(8), counts=addr(9), next_token=addr(10), stream=0)
        d.update(kw)
        tl.tl_verify(**d)
    for kw, want in [(dict(vocab=0), tl.TL_EINVAL), (dict(num_seqs=-1), tl.TL_EINVAL), (dict(total_nodes=-1), tl.TL_EINVAL), (dict(max_nodes=0), tl.TL_EINVAL),
                     (dict(logits_dtype=2), tl.TL_EINVAL), (dict(draft_dtype=-1), tl.TL_EINVAL), (dict(logits=None), tl.TL_EINVAL),
                     (dict(logits=addr(0) + 2), tl.TL_EINVAL), (dict(draft=addr(4) + 8), tl.TL_EINVAL), (dict(noise=None), tl.TL_EINVAL),
                     (dict(noise=addr(7) + 4), tl.TL_EINVAL), (dict(parents=None), tl.TL_EINVAL), (dict(tokens=addr(3) + 1), tl.TL_EINVAL),
                     (dict(uniform=None), tl.TL_EINVAL), (dict(temperature=None), tl.TL_EINVAL), (dict(node_offsets=None), tl.TL_EINVAL),
                     (dict(path=None), tl.TL_EINVAL), (dict(counts=addr(9) + 2), tl.TL_EINVAL), (dict(next_token=None), tl.TL_EINVAL),
                     (dict(vocab=(1 << 26) + 1), tl.TL_EUNSUPPORTED), (dict(total_nodes=1 << 27), tl.TL_EUNSUPPORTED), (dict(max_nodes=4097), tl.TL_EUNSUPPORTED)]:
        assert status(verify, **kw) == want, kw
    assert status(verify, num_seqs=0, logits=None) == tl.TL_OK


def test_helpers_refuse_other_tensors():
    import torch
    x = torch.zeros((4, 256), dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        tl._rows(x, 2, 128)                                # not on a device
    with pytest.raises(ValueError):
        tl._int32(torch.zeros(3, dtype=torch.int64))
    with pytest.raises(ValueError):
        tl._in_dtype(torch.zeros(3, dtype=torch.float16))
    with pytest.raises(ValueError):
        tl.rope(torch.zeros((1, 4), dtype=torch.int64), torch.zeros(8))
    with pytest.raises(ValueError):
        tl.rope(torch.zeros(5, dtype=torch.int32), torch.zeros(8), (4, 4))
