"""tl_attn over entries that exist and that some rows do not see, holding any bytes: 8-bit caches' scale bytes of all ones
among them (slots that no token was written to).  Tolerance as in tests/test_gpu_attn.py."""
import numpy as np
import pytest

from tests import _serve
from tests import test_gpu_attn as base
from tests._gpu import banner

pytestmark = pytest.mark.gpu
_lib = base._lib


@pytest.mark.parametrize("D,elem", [(64, 1), (128, 1), (128, 2)])
@pytest.mark.parametrize("heads", [(2, 2), (4, 2), (8, 2), (16, 2), (12, 1)])
@pytest.mark.parametrize("tree", [True, False])
@pytest.mark.parametrize("before", [64, 1300])
def test_unwritten_entries_that_a_row_does_not_see(D, elem, heads, tree, before):
    """New tokens 7 and 9 of 12 were never written: their slots hold the pool's first bytes, all ones.  In the tree no other
    node descends from them."""
    banner(f"attn unwritten entries D={D} elem={elem} heads {heads} tree={tree} before={before}")
    n, bad = 12, (7, 9)
    mask = None
    if tree:
        mask = np.zeros((n, 1), dtype=np.uint32)
        for i in range(n):
            up = [j for j in range(i) if j not in bad]
            mask[i] = (mask[up[-1 - i % 2 if len(up) > 1 else -1]] if up else 0) | np.uint32(1 << i)
    c = base.Case(121, [before + n], [n], *heads, D, elem, 64, mask=mask)
    stale = _serve.Cache(1, heads[1], D, 64, elem)
    d = np.arange(D)
    for i in bad:
        t = before + i
        p, t = c.table[0, t // 64], t % 64
        for data, from_, at in ((c.cache.kb, stale.kb, _serve.key_at), (c.cache.vb, stale.vb, _serve.value_at)):
            data[p][:, at(t, d, D, elem)] = from_[0][:, at(t, d, D, elem)]
        c.cache.ke[p][:, _serve.key_exp_at(t)] = 0xff
        c.cache.ve[p][:, _serve.value_exp_at(t)] = 0xff
    want, size = _serve.attention(c.q, c.cache, c.table, c.lens, c.offsets, c.scale, c.mask)
    got = c.run().cpu().double().numpy()
    for i in range(n):
        if (tree and i in bad) or (not tree and i >= bad[0]):
            continue                                       # sees one
        assert np.isfinite(got[i]).all(), i
        assert (np.abs(got[i] - want[i]) <= 2.0 ** -8 * np.abs(want[i]) + 1.25 * 2.0 ** -8 * size[i]).all(), i
