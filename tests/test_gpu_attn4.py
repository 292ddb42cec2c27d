"""tl_attn over 4-bit caches against the definition in 64 bits; keys and values enter the products exactly, so that the
tolerance is that of tests/test_gpu_attn.py."""
import numpy as np
import pytest

import paper_2607_04031_amd as tl
from tests import _serve, _serve4
from tests import test_gpu_attn as base
from tests._gpu import banner

pytestmark = pytest.mark.gpu
_lib, _int, _tree = base._lib, base._int, base._tree


class Case4(base.Case):
    """A base.Case over a 4-bit cache; the pages' other bytes are all ones (scales that are NaN)."""

    def __init__(self, seed, lens, new, Hq, H, D, page, mask=None, q_sigma=1.5, spare=1):
        self.rng = rng = np.random.default_rng(seed)
        self.lens, self.new, self.Hq, self.H, self.D, self.page = np.array(lens), np.array(new), Hq, H, D, page
        need = [max(1, -(-int(x) // page)) for x in lens]
        order = rng.permutation(sum(need) + spare)
        self.table = np.full((len(lens), max(need)), -1)
        self.cache = _serve4.Cache4(sum(need) + spare, H, D, page)
        at = 0
        for b, c in enumerate(need):
            self.table[b, :c] = order[at:at + c]
            at += c
        # all tokens at once, with block scales of a wide range
        slots = [self.table[b, t // page] * page + t % page for b in range(len(lens)) for t in range(int(lens[b]))]
        for s in slots:
            scale = np.exp2(rng.integers(-2, 3, (H, D // 32))).repeat(32, axis=-1)
            self.cache.put(s, rng.standard_normal((H, D)), rng.standard_normal((H, D)) * scale)
        self.offsets = np.concatenate([[0], np.cumsum(new)])
        self.q = _serve.bf16(rng.standard_normal((int(self.offsets[-1]), Hq, D)) * q_sigma)
        self.mask, self.scale = mask, D ** -0.5


def _near(got, want, size):
    over = np.abs(got - want) - (2.0 ** -8 * np.abs(want) + 1.25 * 2.0 ** -8 * size)
    at = np.unravel_index(np.nan_to_num(over, nan=np.inf).argmax(), over.shape)
    where = f"at {at}: {got[at]}, not {want[at]}; {(~(over <= 0)).sum()} of {over.size}"     # first: the message shows values
    ok = bool((over <= 0).all())
    assert ok, where


@pytest.mark.parametrize("D,page", [(128, 64), (64, 128)])
@pytest.mark.parametrize("Hq,H", [(8, 1), (6, 2), (3, 3), (20, 1), (40, 1), (70, 1)])
def test_single_tokens(D, page, Hq, H):
    banner(f"attn4 single tokens D={D} page={page} heads {Hq}/{H}")
    c = Case4(1, [1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 200], [1] * 12, Hq, H, D, page)
    c.check(c.run())


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("new", [[2, 5, 8], [17, 1, 33], [70, 64, 65], [130, 3, 100]])
def test_chains_and_prompts(D, new):
    banner(f"attn4 causal new={new} D={D}")
    c = Case4(2, [new[0], 90 + new[1], 300], new, 4, 2, D, 64)
    c.check(c.run())
    c.check(c.run(max_q=max(new) + 50, max_len=1000))      # loose bounds


@pytest.mark.parametrize("D,Hq,H", [(128, 8, 1), (128, 4, 2), (64, 6, 6), (64, 24, 1)])
@pytest.mark.parametrize("new,lens", [([7, 1, 20], [7, 64, 200]), ([33, 64, 70], [64, 129, 90])])
def test_trees(D, Hq, H, new, lens):
    banner(f"attn4 trees new={new} lens={lens} D={D}")
    rng = np.random.default_rng(4)
    words = -(-max(new) // 32)
    c = Case4(3, lens, new, Hq, H, D, 64, mask=np.concatenate([_tree(rng, n, words) for n in new]))
    c.check(c.run())


def test_rows_that_see_nothing_and_odd_lengths():
    banner("attn4: rows that see nothing, lengths of 0, more new tokens than keys")
    rng = np.random.default_rng(6)
    m0 = _tree(rng, 5, 1)
    m0[2] = m0[4] = 0
    c = Case4(7, [5, 80, 40], [5, 3, 40], 4, 2, 128, 64, mask=np.concatenate([m0, _tree(rng, 3, 1), _tree(rng, 40, 1)]))
    out = c.run()
    c.check(out)
    assert not out[2].any() and not out[4].any()
    c = Case4(8, [0, 3, 64], [0, 0, 2], 4, 2, 64, 64)
    c.check(c.run())
    c = Case4(9, [3, 70], [5, 2], 4, 2, 128, 64)
    out = c.run()
    c.check(out)
    assert not out[0].any() and not out[1].any() and out[2].any()
    c = Case4(10, [0, 1], [1, 1], 4, 2, 128, 64)
    out = c.run()
    c.check(out)
    assert not out[0].any()


@pytest.mark.parametrize("Hq", [8, 40, 80])
def test_pages_that_are_none(Hq):
    banner(f"attn4: page ids outside the cache, {Hq} heads")
    c = Case4(11, [300, 200, 64], [1, 3, 1], Hq, 2, 128, 64)
    c.table[0, 1], c.table[0, 3], c.table[1, 0], c.table[2, 0] = -5, 10 ** 6, -1, c.cache.pages
    out = c.run()
    c.check(out)
    assert not out[4].any()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("group", [2, 8, 20])
def test_keys_that_a_row_does_not_see_contribute_nothing(D, group):
    """NaN blocks, and blocks with a scale of 2^126 and 2^127, whose larger values are infinities, that some rows see and
    others do not; rows of every tile size."""
    banner(f"attn4: NaN and infinities in unseen entries D={D} group={group}")
    rng = np.random.default_rng(12)
    n, L = 12, 76
    for mask in (None, _tree(rng, n, 1)):
        c = Case4(13, [L], [n], 2 * group, 2, D, 64, mask=mask)
        bad = L - n + 7                                    # new token 7
        p, t = c.table[0, bad // 64], bad % 64
        slot = p * 64 + t
        k, v = rng.standard_normal((2, D)), rng.standard_normal((2, D))
        k[0, 3] = np.nan
        v[1, :32] = np.repeat([1.0, 4.0, -6.0, 0.0], 8)
        v[0, 40] = np.nan
        c.cache.put(slot, k, v)
        # head 1: the block of elements 0 .. 31 times 2^126: 1, then infinity, -infinity, 0
        exp = t // 64 * 64 * (D // 32) + t % 16 // 4 * 16 + t % 64 // 16 * 4 + t % 4
        c.cache.ve[p][1, exp] = 253
        c.cache.v[slot, 1, :32] = np.repeat([2.0 ** 126, np.inf, -np.inf, 0.0], 8)
        with np.errstate(invalid="ignore"):
            want, size = _serve.attention(c.q, c.cache, c.table, c.lens, c.offsets, c.scale, c.mask)
        got = c.run().cpu().double().numpy()
        for i in range(n):
            sees = i >= 7 if mask is None else bool(int(mask[i, 0]) >> 7 & 1)
            if not sees:
                _near(got[i], want[i], size[i])
                continue
            assert np.isnan(got[i, :group]).all()          # a NaN score
            assert (got[i, group:, 8:16] == np.inf).all() and (got[i, group:, 16:24] == -np.inf).all()
            ok = np.r_[24:D]
            _near(got[i, group:][:, ok], want[i, group:][:, ok], size[i, group:][:, ok])
            # a value of 2^126 may overflow: the weights that it is summed with are up to 2^8 times what they are in the
            # end, and 2^126 2^8 is past 2^128
            some = np.isfinite(got[i, group:, :8])
            assert (got[i, group:, :8][~some] == np.inf).all()
            _near(np.where(some, got[i, group:, :8], want[i, group:, :8]), want[i, group:, :8], size[i, group:, :8])


def test_nan_values_reach_the_rows_that_see_them():
    """A NaN among the values alone: of its 32 elements, for every row that sees it, in chunks that all rows see and others."""
    banner("attn4: NaN values")
    for at in (3, 70, 130):
        c = Case4(21, [140], [12], 4, 2, 128, 64)
        v = c.rng.standard_normal((2, 128))
        v[0, 33] = np.nan
        c.cache.put(c.table[0, at // 64] * 64 + at % 64, c.rng.standard_normal((2, 128)), v)
        with np.errstate(invalid="ignore"):
            want, size = _serve.attention(c.q, c.cache, c.table, c.lens, c.offsets, c.scale)
        got = c.run().cpu().double().numpy()
        np.testing.assert_array_equal(np.isnan(got), np.isnan(want))
        ok = np.isfinite(want)
        _near(got[ok], want[ok], size[ok])


def test_long_sequences_are_split():
    import torch
    banner("attn4: long sequences")
    for group in (8, 40, 70):
        c = Case4(14, [5000, 3, 1111], [1, 2, 4], group, 1, 128, 128)
        out = c.run()
        c.check(out)
        c.check(c.run(max_len=100000))
        again = c.run()
        torch.cuda.synchronize()
        assert torch.equal(again.view(torch.int16), out.view(torch.int16))


@pytest.mark.parametrize("D,group", [(128, 3), (128, 40), (64, 20)])
def test_pieces_with_and_without_odd_values_in_turn(D, group):
    banner(f"attn4 pieces, NaNs in some: D={D} group={group}")
    rng = np.random.default_rng(100 + group)
    lens = rng.integers(2, 60, 200)
    lens[77] = 2100
    c = Case4(101, lens, [1] * 200, 2 * group, 2, D, 64)
    odd = np.arange(0, 200, 3)
    for b in odd:
        t = int(lens[b]) - 1
        v = rng.standard_normal((2, D))
        v[0, 7] = np.nan
        c.cache.put(c.table[b, t // 64] * 64 + t % 64, rng.standard_normal((2, D)), v)
    q, cache = c.q_dev(), c.cache.device()
    with np.errstate(invalid="ignore"):
        want, size = _serve.attention(c.q, c.cache, c.table, c.lens, c.offsets, c.scale)
    ok = np.ones(want.shape, dtype=bool)
    ok[odd, :group, :32] = False
    for _ in range(3):
        got = c.run(q=q, cache=cache).cpu().double().numpy()
        assert np.isnan(got[odd, :group, :32]).all() and np.isfinite(got[ok]).all()
        _near(got[ok], want[ok], size[ok])


def test_strided_queries_streams_and_graphs():
    import torch
    banner("attn4: queries inside a projection's rows, another stream, a graph replayed")
    c = Case4(16, [2300, 90, 1500], [2, 1, 3], 8, 2, 128, 64)
    wide = torch.full((6, 8 * 128 + 512), float("nan"), dtype=torch.bfloat16, device="cuda")
    wide[:, 256:256 + 1024] = c.q_dev().view(6, 1024)
    c.check(c.run(q=wide[:, 256:256 + 1024]))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        out = c.run()
    side.synchronize()
    c.check(out)
    cache, q = c.cache.device(), c.q_dev()
    table, lens, offsets = _int(c.table), _int(c.lens), _int(c.offsets)
    res = torch.empty((6, 8, 128), dtype=torch.bfloat16, device="cuda")
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        tl.attention(q, cache, table, lens, offsets, 3, 2300, c.scale, out=res)
    for step in range(3):
        c.q = _serve.bf16(np.random.default_rng(30 + step).standard_normal(c.q.shape))
        q.copy_(c.q_dev())
        res.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        c.check(res)
        assert torch.isfinite(torch.randn(1000, device="cuda").sum())


def test_cache_past_four_gigabytes():
    import torch
    banner("attn4: pages past 2^32 bytes")
    pages, H, D, page = 72000, 8, 128, 128
    cache = tl.kv_cache(pages, H, D, page, tl.TL_KV_E2M1)
    rng = np.random.default_rng(17)
    ids = [pages - 1, 34000, 70000]
    small = _serve4.Cache4(3, H, D, page)
    L = 300
    k, v = (_serve.bf16(rng.standard_normal((L, H, D))) for _ in range(2))
    for t in range(L):
        small.put(t, k[t], v[t])
    slots = [ids[t // page] * page + t % page for t in range(L)]
    tl.kv_append(None, torch.from_numpy(k.astype(np.float32)).cuda(), torch.from_numpy(v.astype(np.float32)).cuda(), cache, _int(slots))
    q = _serve.bf16(rng.standard_normal((1, 2 * H, D)))
    out = tl.attention(torch.from_numpy(q).to(torch.bfloat16).cuda(), cache, _int([ids]), _int([L]), _int([0, 1]), 1, L, D ** -0.5)
    want, size = _serve.attention(q, small, [[0, 1, 2]], [L], [0, 1], D ** -0.5)
    got = out.cpu().double().numpy()
    _near(got, want, size)


@pytest.mark.parametrize("D,G", [(128, 3), (64, 3), (128, 20)])
def test_prompts_with_a_tile_for_every_workgroup(D, G):
    """Whole tiles, the longest of all sequences and heads first: ragged lengths, among them none and fewer keys than rows, and
    a bound below some sequence's new tokens, whose rows past it are left as they are."""
    import torch
    banner(f"attn4 many prompts D={D} G={G}")
    H = 64 if G == 3 else 32
    new = [30, 25, 30, 1, 30, 0, 28, 30, 12, 30] if G == 3 else [30, 7, 25, 0, 30]
    lens = [30, 200, 64, 1, 25, 0, 129, 31, 90, 65] if G == 3 else [40, 100, 20, 0, 130]
    c = Case4(31, lens, new, H * G, H, D, 64)
    out = c.run()
    c.check(out)
    again = c.run(max_len=2000)
    torch.cuda.synchronize()
    assert torch.equal(again.view(torch.int16), out.view(torch.int16))
    res = torch.full_like(out, 7.0)
    bound = 26
    tl.attention(c.q_dev(), c.cache.device(), _int(c.table), _int(c.lens), _int(c.offsets), bound, max(lens), c.scale, out=res)
    torch.cuda.synchronize()
    for b, n in enumerate(new):
        a = int(c.offsets[b])
        assert torch.equal(res[a:a + min(n, bound)].view(torch.int16), out[a:a + min(n, bound)].view(torch.int16))
        assert (res[a + min(n, bound):a + n] == 7.0).all()
