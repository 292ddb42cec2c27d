"""tl_attn where a workgroup takes several pieces of tiles one after the other, and some of them hold infinities or NaNs that
others must not see.  Tolerance as in tests/test_gpu_attn.py."""
import numpy as np
import pytest

from tests import _serve
from tests import test_gpu_attn as base
from tests._gpu import banner

pytestmark = pytest.mark.gpu
_lib = base._lib


@pytest.mark.parametrize("D,elem", [(128, 1), (128, 2), (64, 1), (64, 2)])
@pytest.mark.parametrize("group", [3, 20, 40])
def test_pieces_with_and_without_odd_values_in_turn(D, elem, group):
    """200 short sequences beside a long one that has the keys split: 400 tiles of one chunk on about 360 workgroups, so that
    nearly all of them hold the end of one tile and the start of another.  Every third sequence's last token has a NaN value
    (16-bit caches an infinity too), which its chunk's masked form takes apart."""
    banner(f"attn pieces, odd values in some: D={D} elem={elem} group={group}")
    rng = np.random.default_rng(100 + group)
    lens = rng.integers(2, 60, 200)
    lens[77] = 2100
    c = base.Case(101, lens, [1] * 200, 2 * group, 2, D, elem, 64)
    odd = np.arange(0, 200, 3)
    for b in odd:
        t = int(lens[b]) - 1
        v = rng.standard_normal((2, D))
        v[0, 7] = np.nan
        if elem == 2:
            v[1, D - 2] = -np.inf
        c.cache.put(c.table[b, t // 64] * 64 + t % 64, rng.standard_normal((2, D)), v)
    q, cache = c.q_dev(), c.cache.device()
    with np.errstate(invalid="ignore"):
        want, size = _serve.attention(c.q, c.cache, c.table, c.lens, c.offsets, c.scale)
    ok = np.ones(want.shape, dtype=bool)
    ok[odd, :group, 7] = False
    if elem == 2:
        ok[odd, group:, D - 2] = False
    for _ in range(5):
        got = c.run(q=q, cache=cache).cpu().double().numpy()
        assert np.isnan(got[odd, :group, 7]).all()
        if elem == 2:
            assert (got[odd, group:, D - 2] == -np.inf).all()
        assert np.isfinite(got[ok]).all()
        assert (np.abs(got[ok] - want[ok]) <= 2.0 ** -8 * np.abs(want[ok]) + 1.25 * 2.0 ** -8 * size[ok]).all()
