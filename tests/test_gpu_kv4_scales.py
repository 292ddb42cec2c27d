"""Blocks of a 4-bit cache whose scale byte is at either end of its range: what tl_kv_read and tl_attn make of 2^-127 (of which
the values are subnormal in bf16) up to 2^127, and of pages that were not written by tl_kv_append."""
import numpy as np
import pytest

import paper_2607_04031_amd as tl
from tests import _serve, _serve4
from tests import test_gpu_attn as base
from tests._gpu import banner
from tests.test_gpu_attn4 import Case4, _near

pytestmark = pytest.mark.gpu
_lib, _int, _tree = base._lib, base._int, base._tree
ENDS = (0, 1, 2, 126, 127, 251, 252, 253, 254, 255)


class Raw(_serve4.Cache4):
    """A cache whose entries are given as codes [heads, D] and scale bytes [heads, D / 32]."""

    def put_codes(self, slot, k, ke, v, ve):
        p, t, B = slot // self.page, slot % self.page, self.D // 32
        d = np.arange(self.D)
        b, r = d // 32, d % 32
        at = (t // 16 * B + b) * 256 + t % 16 * 16 + r // 2
        self.kb[p][:, at[::2]] = k[:, ::2] | k[:, 1::2] << 4
        at = ((t // 64 * B + b) * 4 + t % 16 // 4) * 256 + r % 16 * 16 + t % 64 // 16 * 4 + t % 4
        low = r < 16
        self.vb[p][:, at[low]] = v[:, low] | v[:, ~low] << 4
        b = np.arange(B)
        self.ke[p][:, (t // 64 * B + b) * 64 + t % 16 * 4 + t % 64 // 16] = ke
        self.ve[p][:, (t // 64 * B + b) * 64 + t % 16 // 4 * 16 + t % 64 // 16 * 4 + t % 4] = ve
        self.k[slot], self.v[slot] = _bf16(_serve4.values(k, ke)), _bf16(_serve4.values(v, ve))


def _bf16(x):
    """Two significant bits, from 2^-128 on: exact in bf16 (whose least is 2^-133), but for what is 2^128 and more."""
    return np.where(np.abs(x) >= 2.0 ** 128, np.copysign(np.inf, x), x)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n", [70, 1100])
def test_read(D, n):
    """Every code under every such scale, per token and in windows; whole values, and so equal."""
    banner(f"kv4 read: scale bytes at the ends, D={D} n={n}")
    rng = np.random.default_rng(D + n)
    H, page = 2, 64
    cache = Raw(-(-n // page) + 1, H, D, page)
    for s in range(n):
        codes = [rng.permuted(np.tile(np.arange(16), (H, D // 16)), axis=1).astype(np.uint8) for _ in range(2)]
        exps = [rng.choice(ENDS, (H, D // 32)).astype(np.uint8) for _ in range(2)]
        cache.put_codes(s, codes[0], exps[0], codes[1], exps[1])
    k, v = tl.kv_read(cache.device(), _int(np.arange(n)))
    np.testing.assert_array_equal(k.cpu().double().numpy(), cache.k[:n])
    np.testing.assert_array_equal(v.cpu().double().numpy(), cache.v[:n])


class Ends(Case4):
    """A Case4 whose entries are random codes under scale bytes drawn from those given."""

    def __init__(self, seed, lens, new, Hq, H, D, page, key_exps, value_exps, mask=None):
        super().__init__(seed, lens, new, Hq, H, D, page, mask=mask)
        self.cache = Raw(self.cache.pages, H, D, page)
        for b in range(len(lens)):
            for t in range(int(lens[b])):
                codes = self.rng.integers(0, 16, (2, H, D), dtype=np.uint8)
                exps = [self.rng.choice(x, (H, D // 32)).astype(np.uint8) for x in (key_exps, value_exps)]
                self.cache.put_codes(self.table[b, t // page] * page + t % page, codes[0], exps[0], codes[1], exps[1])


@pytest.mark.parametrize("D,page", [(128, 64), (64, 128)])
@pytest.mark.parametrize("group", [2, 8, 20, 70])
@pytest.mark.parametrize("tree", [False, True])
def test_attention_over_the_smallest_scales(D, page, group, tree):
    """Values up to 6 * 2^-125, most of them subnormal in bf16, in chunks that all rows see and others, for rows of every tile
    size.  The bound of tests/test_gpu_attn.py; where the output is subnormal its rounding is half a step of 2^-133, and sums
    of 150 products in steps of 2^-149 are off by less than 150 * 2^-150 < 2^-142 (the weights are up to 2^8 times larger
    meanwhile, which only makes that less)."""
    banner(f"attn4: smallest scales D={D} group={group} tree={tree}")
    rng = np.random.default_rng(5)
    new = [3, 1, 2]
    mask = np.concatenate([_tree(rng, n, 1) for n in new]) if tree else None
    c = Ends(51, [150, 64, 9], new, 2 * group, 2, D, page, (0, 1, 125, 126), (0, 1, 2), mask=mask)
    want, size = _serve.attention(c.q, c.cache, c.table, c.lens, c.offsets, c.scale, c.mask)
    got = c.run().cpu().double().numpy()
    over = np.abs(got - want) - (2.0 ** -8 * np.abs(want) + 1.25 * 2.0 ** -8 * size + 2.0 ** -134 + 2.0 ** -142)
    assert (over <= 0).all(), f"{(over > 0).sum()} of {over.size}, {over.max() * 2.0 ** 126} * 2^-126 over"


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("group", [2, 20, 40, 70])
def test_attention_over_one_entry_is_the_entry(D, group):
    """One key: its weight is 1, and the values come back as they are, up to 6 * 2^125 and from 2^-128 on."""
    banner(f"attn4: one entry D={D} group={group}")
    for exp in (0, 1, 127, 251, 252):
        c = Ends(52 + exp, [1], [1], 2 * group, 2, D, 64, (0, 127), (exp,))
        got = c.run().cpu().double().numpy()
        want = np.repeat(c.cache.v[c.table[0, 0] * 64], group, axis=0)[None]
        np.testing.assert_array_equal(got, want)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("group", [2, 20, 40, 70])
@pytest.mark.parametrize("tree", [False, True])
def test_rows_do_not_see_others_scales(D, group, tree):
    """A new token's entry under any scale byte: rows that do not see it are within the bound of tests/test_gpu_attn.py whatever
    the byte is.  Not the same bits: a wave's rows take new maxima together, once one row's has grown by 2^8, so that what one
    row sees can move the m of another by up to 8; its weights 2^(s - m) are rounded once all the same, by half a step of
    2^-8 of themselves, whatever m is, and the sums that they are divided by move with them."""
    banner(f"attn4: scales of unseen entries D={D} group={group} tree={tree}")
    rng = np.random.default_rng(6)
    n, L, at = 6, 70, 3
    mask = _tree(rng, n, 1) if tree else None
    sees = [i >= at if mask is None else bool(int(mask[i, 0]) >> at & 1) for i in range(n)]
    unseen = [i for i in range(n) if not sees[i]]
    assert unseen and len(unseen) < n
    for exp in ENDS:
        c = Ends(53, [L], [n], 2 * group, 2, D, 64, (126,), (126, 127), mask=mask)
        t = L - n + at
        codes = np.random.default_rng(7).integers(0, 16, (2, 2, D), dtype=np.uint8)
        exps = np.full((2, D // 32), exp, dtype=np.uint8)
        c.cache.put_codes(c.table[0, t // 64] * 64 + t % 64, codes[0], exps, codes[1], exps)
        with np.errstate(invalid="ignore", over="ignore"):
            want, size = _serve.attention(c.q, c.cache, c.table, c.lens, c.offsets, c.scale, c.mask)
        _near(c.run().cpu().double().numpy()[unseen], want[unseen], size[unseen])
