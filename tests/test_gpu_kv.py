"""The paged key/value cache: tl_kv_append against the definitions (rotary
positions, scales, E4M3 and bf16 rounding, every byte of the pages), tl_kv_read
back, tl_kv_keep's moves.

Tolerances.  Without rotation nothing but one rounding happens to a value, and
bytes must be equal.  With rotation a value x cos - y sin is off by a few 2^-24
of |x| + |y| in fp32, which can move it across a rounding boundary: queries are
within half a bf16 step (8 significant bits: 2^-8 of the value at most) plus 2^-21 (|x| + |y|) of the
64-bit value, stored E4M3 values within half a step (2^-4 of the value, or half
of 2^-9 scales) plus the same, stored bf16 ones as queries."""
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


def _rows(rng, n, heads, D, bf16):
    import torch
    x = rng.standard_normal((n, heads, D)) * np.exp(rng.uniform(-3, 3, (n, heads, 1)))
    t = torch.from_numpy(x.astype(np.float32))
    return t.to(torch.bfloat16) if bf16 else t


def _int(x):
    import torch
    return torch.tensor(np.asarray(x), dtype=torch.int32).cuda()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("elem", [1, 2])
@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("n,Hq,H,page", [(1, 4, 2, 64), (67, 3, 3, 64), (150, 8, 1, 128), (5, 40, 5, 256)])
def test_append_stores_every_byte_and_reads_back(D, elem, bf16, n, Hq, H, page):
    import torch
    banner(f"kv append D={D} elem={elem} bf16={bf16} n={n} Hq={Hq} H={H} page={page}")
    rng = np.random.default_rng(n * 7 + D + elem)
    q, k, v = _rows(rng, n, Hq, D, bf16), _rows(rng, n, H, D, bf16), _rows(rng, n, H, D, bf16)
    k[0, 0] = 0.0                                          # a head of zeros
    k[-1, -1, 3], v[-1, 0, 0] = 448.0 * 2 ** 5, -1e-30     # the largest value of a scale exactly, and a tiny one
    pages = -(-n // page) + 2
    slots = rng.permutation(pages * page)[:n] if n < 10 else np.arange(37, 37 + n)
    ref = _serve.Cache(pages, H, D, page, elem)
    for i, s in enumerate(slots):
        ref.put(s, k[i].double().numpy(), v[i].double().numpy())
    # rows as column ranges of one projection
    fused = torch.cat([x.reshape(n, -1) for x in (q, k, v)], dim=1).cuda()
    a, b = Hq * D, (Hq + H) * D
    cache = _serve.Cache(pages, H, D, page, elem).device()
    out = tl.kv_append(fused[:, :a], fused[:, a:b], fused[:, b:], cache, _int(slots))
    torch.cuda.synchronize()
    assert torch.equal(out.cpu(), q.to(torch.bfloat16))
    for got, want in zip(_serve.device_bytes(cache), ref.bytes()):
        np.testing.assert_array_equal(got, want)
    ko, vo = tl.kv_read(cache, _int(np.append(slots, [-1, pages * page])))
    torch.cuda.synchronize()
    np.testing.assert_array_equal(ko.cpu().double().numpy()[:n], _serve.bf16(ref.k[slots]))
    np.testing.assert_array_equal(vo.cpu().double().numpy()[:n], _serve.bf16(ref.v[slots]))
    assert not ko[n:].any() and not vo[n:].any()           # slots outside the cache


@pytest.mark.parametrize("elem", [1, 2])
@pytest.mark.parametrize("D,rot,sections,interleaved", [(128, 128, (64,), False), (128, 128, (16, 24, 24), False),
                                                        (64, 64, (32,), True), (128, 32, (16,), False),
                                                        (128, 96, (8, 40), True), (64, 16, (0, 8, 0), False)])
def test_append_turns_queries_and_keys(elem, D, rot, sections, interleaved):
    import torch
    banner(f"kv append rope D={D} rot={rot} sections={sections} interleaved={interleaved} elem={elem}")
    n, Hq, H, page = 45, 5, 2, 64
    rng = np.random.default_rng(D + rot)
    q, k, v = (_rows(rng, n, h, D, False) for h in (Hq, H, H))
    pos = rng.integers(0, 200000, (len(sections), n))
    pos[:, 0] = 0
    pos[:, 1] = 2 ** 24 + 1
    freq = (10000.0 ** (-np.arange(rot // 2) / (rot // 2))).astype(np.float32)
    slots = rng.permutation(2 * page)[:n]
    cache = _serve.Cache(2, H, D, page, elem).device()
    rope = tl.rope(_int(pos), torch.from_numpy(freq).cuda(), sections, interleaved)
    out = tl.kv_append(q.cuda(), k.cuda(), v.cuda(), cache, _int(slots), rope)
    ko, vo = tl.kv_read(cache, _int(slots))
    torch.cuda.synchronize()
    qd, kd = q.double().numpy(), k.double().numpy()
    q64, k64 = (_serve.rotate(x, pos, freq, sections, interleaved) for x in (qd, kd))

    def slack(x):                                          # 2^-21 (|x| + |y|), at most twice the head's largest
        return 2.0 ** -20 * np.abs(x).max(-1, keepdims=True)

    got = out.cpu().double().numpy()
    assert (np.abs(got - q64) <= 2.0 ** -8 * np.abs(q64) + slack(qd)).all()
    got = ko.cpu().double().numpy()
    if elem == 2:
        assert (np.abs(got - k64) <= 2.0 ** -8 * np.abs(k64) + slack(kd)).all()
    else:
        _, e = _serve.quantise(k64)
        # an amax within rounding of 448 * 2^e may take the next scale: steps of that one
        step = np.maximum(2.0 ** -4 * np.abs(k64) * 1.0001, 2.0 ** -10 * np.exp2(e + 1.0)[..., None])
        assert (np.abs(got - k64) <= step + slack(kd)).all()
    ref = _serve.Cache(2, H, D, page, elem)
    for i, s in enumerate(slots):
        ref.put(s, k64[i], v[i].double().numpy())
    np.testing.assert_array_equal(vo.cpu().double().numpy(), _serve.bf16(ref.v[slots]))


def test_append_specials():
    """Infinities saturate, NaNs stay NaN and take no part in the maximum."""
    import torch
    D, H = 64, 1
    k = torch.ones((4, H, D))
    k[0, 0, 5] = float("inf")
    k[1, 0, 6], k[1, 0, 7] = float("nan"), 3.0
    k[2, 0, 0] = -float("inf")
    k[3] = float("nan")
    for elem in (1, 2):
        banner(f"kv append specials elem={elem}")
        cache = _serve.Cache(1, H, D, 64, elem).device()
        tl.kv_append(None, k.cuda(), k.cuda(), cache, _int([3, 2, 1, 0]))
        ko, vo = tl.kv_read(cache, _int([3, 2, 1, 0]))
        torch.cuda.synchronize()
        for o in (ko.cpu().float(), vo.cpu().float()):
            if elem == 2:
                assert torch.equal(torch.nan_to_num(o, nan=7.0), torch.nan_to_num(k, nan=7.0))
                continue
            big = 448.0 * 2.0 ** 120
            assert o[0, 0, 5] == big and o[2, 0, 0] == -big
            assert torch.isnan(o[1, 0, 6]) and o[1, 0, 7] == 3.0 and o[1, 0, 0] == 1.0
            assert torch.isnan(o[3]).all()


def test_append_skips_slots_outside_and_either_half():
    import torch
    banner("kv append: slots outside the cache, queries alone, keys alone")
    D, H, Hq, page = 128, 2, 4, 64
    rng = np.random.default_rng(3)
    q, k, v = (_rows(rng, 5, h, D, True) for h in (Hq, H, H))
    ref, cache = _serve.Cache(2, H, D, page, 1), _serve.Cache(2, H, D, page, 1).device()
    slots = [-1, 128, 5, -2 ** 31, 2 ** 31 - 1]
    ref.put(5, k[2].double().numpy(), v[2].double().numpy())
    out = tl.kv_append(q.cuda(), None, None, cache, _int(slots))
    tl.kv_append(None, k.cuda(), v.cuda(), cache, _int(slots))
    torch.cuda.synchronize()
    assert torch.equal(out.cpu(), q)
    for got, want in zip(_serve.device_bytes(cache), ref.bytes()):
        np.testing.assert_array_equal(got, want)
    # nothing to do
    tl.kv_append(q[:0].cuda(), k[:0].cuda(), v[:0].cuda(), cache, _int([]).reshape(0))
    torch.cuda.synchronize()


def test_cache_past_two_and_four_gigabytes():
    """Pages whose bytes start past 2^31 and 2^32."""
    import torch
    D, H, page = 128, 8, 128
    pages = 36000                                          # 4.7 GB of keys, and of values
    banner("kv cache of 4.7 GB: first, middle and last pages")
    cache = tl.kv_cache(pages, H, D, page, 1)
    n = 6
    slots = [0, 2 ** 31 // (H * D) + 1, 2 ** 32 // (H * D) + 65, pages * page - 1, pages * page - 100, 77]
    rng = np.random.default_rng(5)
    k, v = _rows(rng, n, H, D, True), _rows(rng, n, H, D, True)
    tl.kv_append(None, k.cuda(), v.cuda(), cache, _int(slots))
    ko, vo = tl.kv_read(cache, _int(slots))
    torch.cuda.synchronize()
    for got, x in ((ko, k), (vo, v)):
        code, e = _serve.quantise(x.double().numpy())
        np.testing.assert_array_equal(got.cpu().double().numpy(), _serve.E4M3[code] * np.exp2(e.astype(np.float64))[..., None])


@pytest.mark.parametrize("D,elem,H,page", [(128, 1, 2, 64), (64, 2, 3, 128), (64, 1, 1, 64), (128, 2, 1, 64)])
def test_keep_moves_entries(D, elem, H, page):
    import torch
    banner(f"kv keep D={D} elem={elem} H={H} page={page}")
    rng = np.random.default_rng(D + elem)
    most = 70
    starts = [0, 30, 2 * page - 3, 61, 5]
    paths = [[0], [0, 2, 3, 7, 8, 20], [0, 1, 2, 5, 6, 63], list(range(0, most)), list(range(0, 2 * most, 2))[:most]]
    B, per = len(starts), 4 * 64 // page + 3
    pages = B * per
    table = rng.permutation(pages).reshape(B, per)
    ref = _serve.Cache(pages, H, D, page, elem)
    for s in range(pages * page):
        ref.put(s, rng.standard_normal((H, D)), rng.standard_normal((H, D)))
    cache = ref.device()
    path = np.full((B, most), -1)
    for b, p in enumerate(paths):
        path[b, :len(p)] = p
    counts = [len(p) for p in paths]
    counts[1] = 5                                          # the sixth entry stays where it is
    old = _serve.Cache(pages, H, D, page, elem)
    old.kb, old.vb, old.ke, old.ve = (x.copy() for x in (ref.kb, ref.vb, ref.ke, ref.ve))
    d = np.arange(D)
    for b in range(B):
        for i in range(counts[b]):
            src, dst = starts[b] + path[b, i], starts[b] + i
            (p0, t0), (p1, t1) = (table[b, src // page], src % page), (table[b, dst // page], dst % page)
            ref.kb[p1][:, _serve.key_at(t1, d, D, elem)] = old.kb[p0][:, _serve.key_at(t0, d, D, elem)]
            ref.vb[p1][:, _serve.value_at(t1, d, D, elem)] = old.vb[p0][:, _serve.value_at(t0, d, D, elem)]
            ref.ke[p1][:, _serve.key_exp_at(t1)] = old.ke[p0][:, _serve.key_exp_at(t0)]
            ref.ve[p1][:, _serve.value_exp_at(t1)] = old.ve[p0][:, _serve.value_exp_at(t0)]
    tl.kv_keep(cache, _int(table), _int(starts), _int(path), _int(counts))
    torch.cuda.synchronize()
    for got, want in zip(_serve.device_bytes(cache), ref.bytes()):
        np.testing.assert_array_equal(got, want)


def test_keep_outside_the_table_touches_nothing():
    import torch
    banner("kv keep: pages and tokens that are none")
    cache = _serve.Cache(2, 1, 64, 64, 1, fill=0x11).device()
    before = [x.copy() for x in _serve.device_bytes(cache)]
    table = _int([[0, 7], [-1, 1], [1, 0]])
    tl.kv_keep(cache, table, _int([60, 0, -5]), _int([[0, 10], [0, 3], [0, 2]]), _int([2, 2, 2]))
    tl.kv_keep(cache, table, _int([127, 0, 0]), _int([[5, 9], [0, 0], [0, 1]]), _int([2, 0, -3]))
    torch.cuda.synchronize()
    for got, want in zip(_serve.device_bytes(cache), before):
        np.testing.assert_array_equal(got, want)


def test_streams_and_graph_replay():
    """The calls on a stream of their own, and captured in a graph that is replayed between eager work."""
    import torch
    banner("kv append / read / keep on a stream and in a graph")
    D, H, Hq, page, n = 128, 2, 8, 64, 40
    rng = np.random.default_rng(11)
    cache = _serve.Cache(3, H, D, page, 1).device()
    q, k, v = (torch.empty((n, h, D), dtype=torch.bfloat16, device="cuda") for h in (Hq, H, H))
    slots, table = _int(np.arange(50, 50 + n)), _int([[0, 1, 2]])
    q_out, ko, vo = (torch.empty((n, h, D), dtype=torch.bfloat16, device="cuda") for h in (Hq, H, H))
    side = torch.cuda.Stream()

    def work():
        tl.kv_append(q, k, v, cache, slots, None, q_out)
        tl.kv_keep(cache, table, _starts, _path, _counts)
        tl.kv_read(cache, slots, ko, vo)

    _starts, _path, _counts = _int([50]), _int([[0, 3, 4, 9]]), _int([4])
    with torch.cuda.stream(side):
        work()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        work()
    for step in range(3):
        new = [_rows(np.random.default_rng(20 + step), n, h, D, True) for h in (Hq, H, H)]
        for x, y in zip((q, k, v), new):
            x.copy_(y)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        order = np.arange(n)
        order[:4] = [0, 3, 4, 9]
        for got, x in ((ko, new[1]), (vo, new[2])):
            code, e = _serve.quantise(x.double().numpy()[order])
            np.testing.assert_array_equal(got.cpu().double().numpy(), _serve.E4M3[code] * np.exp2(e.astype(np.float64))[..., None])
        assert torch.equal(q_out.cpu(), new[0])
        torch.zeros(1000, device="cuda").sum().item()


@pytest.mark.parametrize("D,elem,bf16,H,page", [(128, 1, True, 2, 64), (64, 1, False, 3, 128), (128, 2, False, 1, 64), (64, 2, True, 5, 256)])
@pytest.mark.parametrize("start", [0, 1, 38])
def test_many_rows_at_once(D, elem, bf16, H, page, start):
    """Rows enough for the kernels that take windows of tokens: slots that
    follow one another from any start, jump inside a window, or lie outside."""
    import torch
    n, Hq = 700, 3
    banner(f"kv append / read of {n} rows D={D} elem={elem} bf16={bf16} H={H} page={page} start={start}")
    rng = np.random.default_rng(start + D)
    q, k, v = _rows(rng, n, Hq, D, bf16), _rows(rng, n, H, D, bf16), _rows(rng, n, H, D, bf16)
    pages = -(-(n + start + 200) // page) + 1
    slots = start + np.arange(n)
    slots[200:] += 50                                      # a jump
    slots[330:340] = slots[330:340][::-1]
    slots[400:403] = [-1, pages * page, -2 ** 31]
    slots[699] = 2 ** 31 - 1                               # windows that run past the end of the cache
    ref = _serve.Cache(pages, H, D, page, elem)
    for i, s in enumerate(slots):
        ref.put(s, k[i].double().numpy(), v[i].double().numpy())
    cache = _serve.Cache(pages, H, D, page, elem).device()
    out = tl.kv_append(q.cuda(), k.cuda(), v.cuda(), cache, _int(slots))
    torch.cuda.synchronize()
    assert torch.equal(out.cpu(), q.to(torch.bfloat16))
    for got, want in zip(_serve.device_bytes(cache), ref.bytes()):
        np.testing.assert_array_equal(got, want)
    inside = (slots >= 0) & (slots < pages * page)
    ko, vo = tl.kv_read(cache, _int(slots))
    torch.cuda.synchronize()
    for got, want in ((ko, ref.k), (vo, ref.v)):
        got = got.cpu().double().numpy()
        np.testing.assert_array_equal(got[inside], _serve.bf16(want[slots[inside]]))
        assert not got[~inside].any()
    only = torch.full((n, H, D), 7.0, dtype=torch.bfloat16, device="cuda")
    tl.tl_kv_read(cache, _int(slots), n, None, only)
    torch.cuda.synchronize()
    assert torch.equal(only, vo)
    # the last slots of the cache
    tail = np.arange(pages * page - 600, pages * page)
    tl.kv_append(None, k[:600].cuda(), v[:600].cuda(), cache, _int(tail))
    ko, vo = tl.kv_read(cache, _int(tail))
    torch.cuda.synchronize()
    for i, s in enumerate(tail):
        ref.put(s, k[i].double().numpy(), v[i].double().numpy())
    np.testing.assert_array_equal(ko.cpu().double().numpy(), _serve.bf16(ref.k[tail]))
    np.testing.assert_array_equal(vo.cpu().double().numpy(), _serve.bf16(ref.v[tail]))


@pytest.mark.parametrize("interleaved", [False, True])
def test_many_rows_turn_as_few_rows_do(interleaved):
    """The same rows at once and in pieces: the same bytes."""
    import torch
    n, Hq, H, D, page = 600, 5, 2, 128, 64
    banner(f"kv append of {n} rows against pieces of 100, interleaved={interleaved}")
    rng = np.random.default_rng(8)
    q, k, v = (_rows(rng, n, h, D, True).cuda() for h in (Hq, H, H))
    pos = _int(rng.integers(0, 5000, (3, n)))
    freq = torch.from_numpy((10000.0 ** (-np.arange(48) / 48)).astype(np.float32)).cuda()
    slots = _int(3 + np.arange(n))
    one, many = (_serve.Cache(10, H, D, page, 1).device() for _ in range(2))
    want = tl.kv_append(q, k, v, one, slots, tl.rope(pos, freq, (8, 16, 24), interleaved))
    got = torch.cat([tl.kv_append(q[i:i + 100], k[i:i + 100], v[i:i + 100], many, slots[i:i + 100],
                                  tl.rope(pos[:, i:i + 100].contiguous(), freq, (8, 16, 24), interleaved)) for i in range(0, n, 100)])
    torch.cuda.synchronize()
    assert torch.equal(got, want)
    for x, y in zip(_serve.device_bytes(one), _serve.device_bytes(many)):
        np.testing.assert_array_equal(x, y)
