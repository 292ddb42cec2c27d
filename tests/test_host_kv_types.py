"""tl.KVCache takes the types that the library reads: E4M3 bytes (uint8 or float8_e4m3fn) with uint8 exponents, or bfloat16.
Tensors here are on the host, which is the last thing that it refuses."""
import pytest
import torch

import paper_2607_04031_amd as tl


def made(k, v=None, k_exp=None, v_exp=None):
    size = torch.empty(0, dtype=k).element_size()
    exps = [None if size == 2 and x is None else torch.zeros((1, 2, 64), dtype=x or torch.uint8) for x in (k_exp, v_exp)]
    return tl.KVCache(torch.zeros((1, 2, 64 * 64), dtype=k), torch.zeros((1, 2, 64 * 64), dtype=v or k), *exps, 64, 2, 64)


@pytest.mark.parametrize("kw", [dict(k=torch.float16), dict(k=torch.int16), dict(k=torch.int8), dict(k=torch.float8_e5m2),
                                dict(k=torch.float8_e4m3fnuz), dict(k=torch.bool), dict(k=torch.bfloat16, v=torch.float16),
                                dict(k=torch.uint8, v=torch.int8), dict(k=torch.uint8, k_exp=torch.int8),
                                dict(k=torch.uint8, v_exp=torch.float8_e4m3fn)])
def test_other_types_are_refused(kw):
    with pytest.raises(ValueError, match="uint8"):
        made(**kw)


@pytest.mark.parametrize("k,v", [(torch.uint8, torch.uint8), (torch.float8_e4m3fn, torch.float8_e4m3fn), (torch.uint8, torch.float8_e4m3fn),
                                 (torch.bfloat16, torch.bfloat16)])
def test_these_are_taken(k, v):
    with pytest.raises(ValueError, match="device tensors"):
        made(k, v)
