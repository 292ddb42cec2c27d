"""The extension module that takes tensors to the serving-step entry points, where there is no device: it hands every call
back, and the binding's checks name what is wrong."""
import pytest
import torch

import paper_2607_04031_amd as tl


def _cache():
    k, v = (torch.zeros((1, 2, 64 * 64), dtype=torch.bfloat16) for _ in range(2))
    c = tl.KVCache.__new__(tl.KVCache)
    c.k, c.v, c.k_exp, c.v_exp = k, v, None, None
    c.page_tokens, c.kv_heads, c.head_dim, c.elem_bytes, c.num_pages = 64, 2, 64, 2, 1
    c.desc = tl.KVCacheDesc(k.data_ptr(), v.data_ptr(), None, None, 1, 64, 2, 64, 2)
    return c


def test_host_tensors_are_handed_back_and_refused():
    calls, c = tl._load_calls(), _cache()
    x, slots = torch.zeros((3, 128), dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int32)
    out = torch.zeros((3, 2, 64), dtype=torch.bfloat16)
    assert calls.kv_append(x, x, x, c.desc, slots, None, out, None) is None
    assert calls.kv_read(c.desc, slots, out, out.clone(), None) is None
    assert calls.attention(out, c.desc, slots[None], slots[:1], slots[:2], 1, 1, 0.1, None, out, None) is None
    with pytest.raises(ValueError):
        tl.kv_append(x, x, x, c, slots, None, out)
    with pytest.raises(ValueError):
        tl.kv_read(c, slots, out, out.clone())


@pytest.mark.parametrize("name,count", [("kv_append", 8), ("kv_read", 5), ("kv_keep", 6), ("attention", 11), ("verify", 13)])
def test_anything_else_is_handed_back_too(name, count):
    f = getattr(tl._load_calls(), name)
    for filler in (None, 0, "x", torch.zeros(2), object()):
        assert f(*[filler] * count) is None
    with pytest.raises(TypeError):
        f(None)


def test_rope_keeps_its_fields():
    r = tl.rope(torch.zeros((2, 5), dtype=torch.int32), torch.zeros(8), (3, 5), True)
    assert r.sections == (3, 5) and r.rot_dim == 16 and r.interleaved
    with pytest.raises(ValueError):
        r.desc      # tensors on the host have no device address
