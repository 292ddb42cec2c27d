"""tl_attn on both sides of the rules by which keys are split over workgroups: the number of keys, the number of tiles and
the longest sequence's bound; and single sequences, whose tiles end where workgroups do.  Tolerance as in
tests/test_gpu_attn.py."""
import numpy as np
import pytest

from tests import test_gpu_attn as base
from tests._gpu import banner

pytestmark = pytest.mark.gpu
_lib = base._lib


@pytest.mark.parametrize("elem,lens", [(1, [2048]), (1, [2049]), (2, [1536]), (2, [1537]), (1, [1025, 2048, 7]), (2, [1600, 1])])
@pytest.mark.parametrize("D", [64, 128])
def test_keys_of_a_whole_tile(elem, lens, D):
    banner(f"attn plans: {lens} keys D={D} elem={elem}")
    c = base.Case(21, lens, [1] * len(lens), 6, 2, D, elem, 64)
    c.check(c.run())
    c.check(c.run(max_len=9000))            # a loose bound: split


@pytest.mark.parametrize("heads", [(8, 1), (12, 12), (7, 7), (40, 2)])
@pytest.mark.parametrize("length,new", [(3001, 1), (2500, 4), (1300, 40)])
def test_one_sequence(heads, length, new):
    banner(f"attn plans: one sequence of {length}, {new} new, heads {heads}")
    c = base.Case(22, [length], [new], *heads, 64, 1 + length % 2, 64)
    c.check(c.run())
    c.check(c.run(max_len=100000))


@pytest.mark.parametrize("elem", [1, 2])
def test_many_tiles_of_few_rows(elem):
    banner(f"attn plans: 64 sequences, 8 heads, elem={elem}")
    rng = np.random.default_rng(5)
    lens = rng.integers(1, 60, 64)
    lens[[3, 40]] = 2100, 700
    c = base.Case(23, list(lens), [1] * 64, 16, 8, 64, elem, 64)
    c.check(c.run(max_len=4096))            # a tile per workgroup
    c.check(c.run(max_len=4097))            # split


@pytest.mark.parametrize("elem", [1, 2])
def test_many_tiles_of_trees(elem):
    banner(f"attn plans: 64 trees, 16 heads, elem={elem}")
    rng = np.random.default_rng(6)
    new = [33] * 60 + [1, 12, 33, 20]
    lens = np.array(new) + rng.integers(0, 30, 64)
    lens[[0, 50]] = 1100, 400
    mask = np.concatenate([base._tree(rng, n, 2) for n in new])
    c = base.Case(24, list(lens), new, 32, 16, 64, elem, 64, mask=mask)
    c.check(c.run(max_len=2048))            # a tile per workgroup
    c.check(c.run(max_len=2049))            # split
