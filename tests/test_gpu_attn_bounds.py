"""tl_attn with a sequence that has more new tokens than max_q says: its rows past the bound stay as they were, its others and
every other sequence's are right.  Tolerance as in tests/test_gpu_attn.py."""
import numpy as np
import pytest

import paper_2607_04031_amd as tl
from tests import _serve
from tests import test_gpu_attn as base
from tests._gpu import banner

pytestmark = pytest.mark.gpu
_lib = base._lib

# lengths, new tokens, the bound, heads: one tile of 16 rows a workgroup; the same split, few tiles of many parts; split in
# many tiles; 128-row tiles, whole and split
CASES = {"whole": ([200, 90, 64] + [30] * 13, [40, 1, 2] + [1] * 13, 2, (8, 1)),
         "few_parts": ([5000, 4000, 100], [60, 1, 2], 2, (8, 1)),
         "split": ([1500, 2300] + [40] * 20, [50, 2] + [1, 2] * 10, 2, (12, 4)),
         "wide": ([300, 130, 90], [200, 70, 3], 70, (4, 2)),
         "wide_split": ([1800, 130, 1200], [300, 70, 3], 70, (4, 2))}


@pytest.mark.parametrize("elem", [1, 2])
@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("name", list(CASES))
def test_a_sequence_above_the_bound(name, tree, elem):
    import torch
    lens, new, bound, heads = CASES[name]
    banner(f"attn bounds {name} tree={tree} elem={elem}")
    rng = np.random.default_rng(7)
    words = -(-max(new) // 32)
    c = base.Case(111, lens, new, *heads, 128, elem, 64, mask=np.concatenate([base._tree(rng, n, words) for n in new]) if tree else None)
    want, size = _serve.attention(c.q, c.cache, c.table, c.lens, c.offsets, c.scale, c.mask)
    out = torch.full((len(want), heads[0], 128), 77.0, dtype=torch.bfloat16, device="cuda")
    tl.attention(c.q_dev(), c.cache.device(), base._int(c.table), base._int(c.lens), base._int(c.offsets), bound, max(lens), c.scale,
                 mask=None if c.mask is None else base._int(c.mask), out=out)
    got = out.cpu().double().numpy()
    place = np.concatenate([np.arange(n) for n in new])
    done = place < bound
    assert (got[~done] == 77.0).all()
    assert (np.abs(got[done] - want[done]) <= 2.0 ** -8 * np.abs(want[done]) + 1.25 * 2.0 ** -8 * size[done]).all()
