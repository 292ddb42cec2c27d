"""The 4-bit cache's sizes and refusals, before any device work (no GPU here; the addresses are never read), and
tl.KVCache's checks of its tensors."""
import pytest
import torch

import paper_2607_04031_amd as tl
from tests.test_host_serve import addr, append, cache, status


def four(**kw):
    return cache(elem_bytes=tl.TL_KV_E2M1, **kw)


def test_kv_bytes():
    assert tl.tl_kv_bytes(four()) == (10 * 64 * 8 * 64, 10 * 64 * 8 * 4)
    assert tl.tl_kv_bytes(four(head_dim=64, page_tokens=4096)) == (10 * 4096 * 8 * 32, 10 * 4096 * 8 * 2)
    assert status(tl.tl_kv_bytes, cache=four(head_dim=96)) == tl.TL_EUNSUPPORTED
    for elem in (0, 3, 4, -1, -2, -8, 16):
        assert status(tl.tl_kv_bytes, cache=cache(elem_bytes=elem)) == tl.TL_EINVAL


def test_refusals():
    for kw in (dict(k=None), dict(v=addr(1) + 8), dict(k_exp=None), dict(v_exp=None), dict(v_exp=addr(3) + 4)):
        assert status(append, cache=four(**kw)) == tl.TL_EINVAL, kw
    data, exps = tl.tl_kv_bytes(four())
    # outputs and inputs that end or begin inside the cache's arrays, and arrays inside one another
    for kw in (dict(K=addr(0) + data - 16), dict(V=addr(3) + exps - 16), dict(Q_out=addr(1) + data - 16), dict(slots=addr(2) + exps - 4)):
        assert status(append, cache=four(), **kw) == tl.TL_EINVAL, kw
    for kw in (dict(v=addr(0) + data - 16), dict(k_exp=addr(1) + data - 16), dict(v_exp=addr(2) + exps - 16)):
        assert status(append, cache=four(**kw)) == tl.TL_EINVAL, kw


def made(dtype=torch.uint8, elem_bytes=tl.TL_KV_E2M1, size=64 * 64 // 2, exps=64 * 2, exp_type=torch.uint8):
    k, v = (torch.zeros((1, 2, size), dtype=torch.uint8).view(dtype) for _ in range(2))
    return tl.KVCache(k, v, *(None if exps is None else torch.zeros((1, 2, exps), dtype=exp_type) for _ in range(2)), 64, 2, 64,
                      elem_bytes=elem_bytes)


@pytest.mark.parametrize("kw", [dict(dtype=torch.int8), dict(dtype=torch.float8_e4m3fn), dict(exp_type=torch.int8), dict(size=64 * 64 // 2 + 1),
                                dict(exps=64), dict(exps=None), dict(elem_bytes=2), dict(elem_bytes=4), dict(elem_bytes=None, exps=64)])
def test_other_tensors_are_refused(kw):
    with pytest.raises(ValueError) as e:
        made(**kw)
    assert "device tensors" not in str(e.value)


@pytest.mark.parametrize("kw", [dict(), dict(dtype=torch.float4_e2m1fn_x2), dict(dtype=torch.float4_e2m1fn_x2, elem_bytes=None),
                                dict(elem_bytes=None, size=64 * 64, exps=64), dict(elem_bytes=1, size=64 * 64, exps=64)])
def test_these_are_taken(kw):
    with pytest.raises(ValueError, match="device tensors"):
        made(**kw)
