"""tl_attn against the definition in 64 bits.

Tolerance.  Per element, with A = sum p |v| / sum p: the output's rounding to
bf16 (8 significant bits: 2^-8 of the value at most), the probabilities' rounding to bf16 (2^-8 A at most)
and the scores' fp32 error, which moves every p by less than 2^-11 of itself
(128 products of size |q k| scale, at most 16 in all here, each sum off by at
most 128 * 2^-24 of that: 2^-13; and the exponential): 2^-8 |o| + 1.25 * 2^-8 A."""
import numpy as np
import pytest

import paper_2607_04031_amd as tl
from tests import _serve
from tests._gpu import banner

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    import torch
    assert torch.cuda.is_available()
    tl.load_library()
    yield
    torch.cuda.synchronize()


def _int(x):
    import torch
    x = np.asarray(x)
    return torch.from_numpy(x.astype(np.int64)).to(torch.int32).cuda() if x.dtype != np.uint32 else \
        torch.from_numpy(x.view(np.int32).copy()).cuda()


class Case:
    """Sequences of given lengths and new tokens over pages in random order, stale bytes (NaN) everywhere else."""

    def __init__(self, seed, lens, new, Hq, H, D, elem, page, mask=None, q_sigma=1.5, spare=1):
        self.rng = rng = np.random.default_rng(seed)
        self.lens, self.new, self.Hq, self.H, self.D, self.page = np.array(lens), np.array(new), Hq, H, D, page
        need = [max(1, -(-int(x) // page)) for x in lens]
        pages = sum(need) + spare
        order = rng.permutation(pages)
        self.table = np.full((len(lens), max(need)), -1)
        at = 0
        self.cache = _serve.Cache(pages, H, D, page, elem)
        for b, c in enumerate(need):
            self.table[b, :c] = order[at:at + c]
            at += c
            for t in range(int(lens[b])):
                self.cache.put(self.table[b, t // page] * page + t % page, rng.standard_normal((H, D)), rng.standard_normal((H, D)))
        self.offsets = np.concatenate([[0], np.cumsum(new)])
        self.q = _serve.bf16(rng.standard_normal((int(self.offsets[-1]), Hq, D)) * q_sigma)
        self.mask = mask
        self.scale = D ** -0.5

    def q_dev(self):
        import torch
        return torch.from_numpy(self.q).to(torch.bfloat16).cuda()

    def run(self, max_q=None, max_len=None, q=None, cache=None, stream=None):
        out = tl.attention(self.q_dev() if q is None else q, self.cache.device() if cache is None else cache, _int(self.table),
                           _int(self.lens), _int(self.offsets), int(max(self.new)) if max_q is None else max_q,
                           int(max(self.lens)) if max_len is None else max_len, self.scale,
                           mask=None if self.mask is None else _int(self.mask), stream=stream)
        return out

    def check(self, out):
        want, size = _serve.attention(self.q, self.cache, self.table, self.lens, self.offsets, self.scale, self.mask)
        got = out.cpu().double().numpy()
        assert np.isfinite(got).all()
        over = np.abs(got - want) - (2.0 ** -8 * np.abs(want) + 1.25 * 2.0 ** -8 * size)
        assert (over <= 0).all(), f"{over.max()} over the bound, at {np.unravel_index(over.argmax(), over.shape)}"


@pytest.mark.parametrize("D,elem,page", [(128, 1, 64), (64, 1, 128), (128, 2, 128), (64, 2, 64)])
@pytest.mark.parametrize("Hq,H", [(8, 1), (6, 2), (3, 3), (20, 1), (40, 1)])
def test_single_tokens(D, elem, page, Hq, H):
    banner(f"attn single tokens D={D} elem={elem} page={page} heads {Hq}/{H}")
    c = Case(1, [1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 200], [1] * 12, Hq, H, D, elem, page)
    c.check(c.run())


@pytest.mark.parametrize("elem", [1, 2])
@pytest.mark.parametrize("new", [[2, 5, 8], [17, 1, 33], [70, 64, 65], [130, 3, 100]])
def test_chains_and_prompts(elem, new):
    banner(f"attn causal new={new} elem={elem}")
    c = Case(2, [new[0], 90 + new[1], 300], new, 4, 2, 128, elem, 64)
    c.check(c.run())
    c.check(c.run(max_q=max(new) + 50, max_len=1000))      # loose bounds


def _tree(rng, n, words):
    mask = np.zeros((n, words), dtype=np.uint32)
    for i in range(n):
        if i:
            mask[i] = mask[rng.integers(max(0, i - 6), i)]
        if i < 32 * words:
            mask[i, i // 32] |= np.uint32(1 << (i % 32))
    return mask


@pytest.mark.parametrize("D,elem,Hq,H", [(128, 1, 8, 1), (128, 2, 4, 2), (64, 1, 6, 6), (64, 2, 24, 1)])
@pytest.mark.parametrize("new,lens", [([7, 1, 20], [7, 64, 200]), ([33, 64, 70], [64, 129, 90])])
def test_trees(D, elem, Hq, H, new, lens):
    banner(f"attn trees new={new} lens={lens} D={D} elem={elem}")
    rng = np.random.default_rng(4)
    words = -(-max(new) // 32)
    c = Case(3, lens, new, Hq, H, D, elem, 64, mask=np.concatenate([_tree(rng, n, words) for n in new]))
    c.check(c.run())


def test_masks_that_leave_rows_empty_and_short_masks():
    banner("attn: rows that see nothing, masks shorter than the tree, sequences of length 0, more new tokens than keys")
    rng = np.random.default_rng(6)
    # sequence 0 is nothing but its tree; two of its rows see nothing at all
    m0 = _tree(rng, 5, 1)
    m0[2] = 0
    m0[4] = 0
    c = Case(7, [5, 80, 40], [5, 3, 40], 4, 2, 128, 1, 64, mask=np.concatenate([m0, _tree(rng, 3, 1), _tree(rng, 40, 1)]))
    out = c.run()
    c.check(out)
    assert not out[2].any() and not out[4].any()
    c = Case(8, [0, 3, 64], [0, 0, 2], 4, 2, 64, 2, 64)
    c.check(c.run())
    # a length below the new tokens: the first ones lie before the sequence and see nothing
    c = Case(9, [3, 70], [5, 2], 4, 2, 128, 1, 64)
    out = c.run()
    c.check(out)
    assert not out[0].any() and not out[1].any() and out[2].any()
    # length 0 with a query
    c = Case(10, [0, 1], [1, 1], 4, 2, 128, 1, 64)
    out = c.run()
    c.check(out)
    assert not out[0].any()


@pytest.mark.parametrize("elem", [1, 2])
def test_pages_that_are_none(elem):
    banner(f"attn: page ids outside the cache elem={elem}")
    c = Case(11, [300, 200, 64], [1, 3, 1], 8, 2, 128, elem, 64)
    c.table[0, 1], c.table[0, 3], c.table[1, 0], c.table[2, 0] = -5, 10 ** 6, -1, c.cache.pages
    out = c.run()
    c.check(out)
    assert not out[4].any()


@pytest.mark.parametrize("elem", [1, 2])
@pytest.mark.parametrize("D", [64, 128])
def test_keys_that_a_row_does_not_see_contribute_nothing(D, elem):
    """Infinities and NaNs in entries that some rows see and others do not."""
    import torch
    banner(f"attn: NaN and infinities in unseen entries D={D} elem={elem}")
    rng = np.random.default_rng(12)
    n, L = 12, 76
    for mask in (None, _tree(rng, n, 1)):
        c = Case(13, [L], [n], 4, 2, D, elem, 64, mask=mask)
        bad = L - n + 7                                    # new token 7
        slot = c.table[0, bad // 64] * 64 + bad % 64
        k, v = rng.standard_normal((2, D)), rng.standard_normal((2, D))
        k[0, 3] = np.nan
        v[0, 5], v[1, 2] = np.nan, np.nan
        if elem == 2:
            v[1, 9] = np.inf
        c.cache.put(slot, k, v)
        with np.errstate(invalid="ignore"):
            want, size = _serve.attention(c.q, c.cache, c.table, c.lens, c.offsets, c.scale, c.mask)
        got = c.run().cpu().double().numpy()
        for i in range(n):
            sees = i >= 7 if mask is None else bool(int(mask[i, 0]) >> 7 & 1)
            if not sees:
                assert np.isfinite(got[i]).all()
                assert (np.abs(got[i] - want[i]) <= 2.0 ** -8 * np.abs(want[i]) + 1.25 * 2.0 ** -8 * size[i]).all()
                continue
            assert np.isnan(got[i, :2]).all()              # a NaN score
            assert np.isnan(got[i, 2:, 2]).all()
            ok = np.ones(D, dtype=bool)
            ok[2] = False
            if elem == 2:
                assert (got[i, 2:, 9] == np.inf).all()
                ok[9] = False
            assert (np.abs(got[i, 2:, ok] - want[i, 2:, ok]) <= 2.0 ** -8 * np.abs(want[i, 2:, ok]) + 1.25 * 2.0 ** -8 * size[i, 2:, ok]).all()
    torch.cuda.synchronize()


@pytest.mark.parametrize("elem", [1, 2])
def test_long_sequences_are_split(elem):
    """Few rows over many keys: units of work, their join, and bounds far above the lengths."""
    import torch
    banner(f"attn: long sequences elem={elem}")
    c = Case(14, [5000, 3, 1111], [1, 2, 4], 8, 1, 128, elem, 128)
    out = c.run()
    c.check(out)
    c.check(c.run(max_len=100000))
    again = c.run()
    torch.cuda.synchronize()
    assert torch.equal(again.view(torch.int16), out.view(torch.int16))


def test_large_scores_and_outliers():
    """Scores of some thousands, where one key takes everything, and values of very different scales."""
    import torch
    banner("attn: large scores")
    c = Case(15, [150], [3], 4, 2, 128, 1, 64, q_sigma=1.0)
    c.q = _serve.bf16(c.q * 300)
    for t in (0, 64, 149):
        c.cache.put(c.table[0, t // 64] * 64 + t % 64, c.rng.standard_normal((2, 128)) * 2.0 ** 10, c.rng.standard_normal((2, 128)) * 1e-4)
    want, size = _serve.attention(c.q, c.cache, c.table, c.lens, c.offsets, c.scale)
    got = c.run().cpu().double().numpy()
    torch.cuda.synchronize()
    # scores up to 10^6: fp32 sums and their scaling are off by up to 10^6 * 2^-19, so only rows
    # that one key takes by more than that are compared
    for i in range(3):
        for h in range(4):
            at = [c.table[0, t // 64] * 64 + t % 64 for t in range(150 - 3 + i + 1)]
            s = np.sort(c.cache.k[at][:, h // 2] @ c.q[i, h] * c.scale)
            if s[-1] - s[-2] > 100:
                assert (np.abs(got[i, h] - want[i, h]) <= 2.0 ** -8 * np.abs(want[i, h]) + 2.0 ** -8 * size[i, h]).all()


def test_strided_queries_streams_and_graphs():
    import torch
    banner("attn: queries inside a projection's rows, another stream, a graph replayed")
    c = Case(16, [700, 90, 1500], [2, 1, 3], 8, 2, 128, 1, 64)
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
        tl.attention(q, cache, table, lens, offsets, 3, 1500, c.scale, out=res)
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
    banner("attn: pages past 2^32 bytes")
    pages, H, D, page = 36000, 8, 128, 128
    cache = tl.kv_cache(pages, H, D, page, 1)
    rng = np.random.default_rng(17)
    ids = [pages - 1, 17000, 35000]
    small = _serve.Cache(3, H, D, page, 1)
    L = 300
    k, v = rng.standard_normal((L, H, D)), rng.standard_normal((L, H, D))
    for t in range(L):
        small.put(t, k[t], v[t])
    slots = [ids[t // page] * page + t % page for t in range(L)]
    tl.kv_append(None, torch.from_numpy(k.astype(np.float32)).cuda(), torch.from_numpy(v.astype(np.float32)).cuda(), cache, _int(slots))
    q = _serve.bf16(rng.standard_normal((1, 2 * H, D)))
    out = tl.attention(torch.from_numpy(q).to(torch.bfloat16).cuda(), cache, _int([ids]), _int([L]), _int([0, 1]), 1, L, D ** -0.5)
    want, size = _serve.attention(q, small, [[0, 1, 2]], [L], [0, 1], D ** -0.5)
    got = out.cpu().double().numpy()
    # keys and values come from fp32 copies here: a rare value next to a tie may round the other way
    assert (np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + 1.5 * 2.0 ** -8 * size).all()
