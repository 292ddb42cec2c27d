"""The 4-bit cache: tl_kv_append against the definitions (rotary positions, the scale of 32 elements, E2M1, every byte of
the pages), tl_kv_read back, tl_kv_keep's moves.

Tolerances.  Without rotation each element is rounded once, and bytes must be equal.  With it a value is off by a few 2^-24
of |x| + |y| in fp32, which can move it across a border: stored values are within half a step (of two significant bits:
2^-2 of the value, or 1/4 of the scale; an amax next to 6 scales may take the next one, with twice that) plus 2^-20 of the
head's largest, queries within half a bf16 step plus the same."""
import numpy as np
import pytest

import paper_2607_04031_amd as tl
from tests import _serve, _serve4
from tests._gpu import banner
from tests.test_gpu_kv import _int, _lib, _rows  # noqa: F401

pytestmark = pytest.mark.gpu


def _same(cache, ref):
    for got, want in zip(_serve.device_bytes(cache), ref.bytes()):
        np.testing.assert_array_equal(got, want)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("n,Hq,H,page", [(1, 4, 2, 64), (67, 3, 3, 64), (150, 8, 1, 128), (5, 40, 5, 256)])
def test_append_stores_every_byte_and_reads_back(D, bf16, n, Hq, H, page):
    import torch
    banner(f"kv4 append D={D} bf16={bf16} n={n} Hq={Hq} H={H} page={page}")
    rng = np.random.default_rng(n * 7 + D)
    q, k, v = _rows(rng, n, Hq, D, bf16), _rows(rng, n, H, D, bf16), _rows(rng, n, H, D, bf16)
    k[0, 0, :32] = 0.0                                     # a block of zeros
    k[-1, -1, 3], v[-1, 0, 0] = 6.0 * 2 ** 5, -1e-30       # the largest value of a scale exactly, and a tiny one
    v[0, 0, 32:40] = torch.tensor([6.0, 5.0, -5.0, 2.5, 3.5, 0.25, -0.75, 1.75])      # ties
    v[0, 0, 40:64] = 0.0
    pages = -(-n // page) + 2
    slots = rng.permutation(pages * page)[:n] if n < 10 else np.arange(37, 37 + n)
    ref = _serve4.Cache4(pages, H, D, page)
    for i, s in enumerate(slots):
        ref.put(s, k[i].double().numpy(), v[i].double().numpy())
    fused = torch.cat([x.reshape(n, -1) for x in (q, k, v)], dim=1).cuda()     # rows as column ranges of one projection
    a, b = Hq * D, (Hq + H) * D
    cache = _serve4.Cache4(pages, H, D, page).device()
    out = tl.kv_append(fused[:, :a], fused[:, a:b], fused[:, b:], cache, _int(slots))
    torch.cuda.synchronize()
    assert torch.equal(out.cpu(), q.to(torch.bfloat16))
    _same(cache, ref)
    ko, vo = tl.kv_read(cache, _int(np.append(slots, [-1, pages * page])))
    torch.cuda.synchronize()
    np.testing.assert_array_equal(ko.cpu().double().numpy()[:n], ref.k[slots])
    np.testing.assert_array_equal(vo.cpu().double().numpy()[:n], ref.v[slots])
    assert not ko[n:].any() and not vo[n:].any()           # slots outside the cache


@pytest.mark.parametrize("D,rot,sections,interleaved", [(128, 128, (64,), False), (128, 128, (16, 24, 24), False),
                                                        (64, 64, (32,), True), (128, 32, (16,), False), (64, 16, (0, 8, 0), False)])
def test_append_turns_queries_and_keys(D, rot, sections, interleaved):
    import torch
    banner(f"kv4 append rope D={D} rot={rot} sections={sections} interleaved={interleaved}")
    n, Hq, H, page = 45, 5, 2, 64
    rng = np.random.default_rng(D + rot)
    q, k, v = (_rows(rng, n, h, D, False) for h in (Hq, H, H))
    pos = rng.integers(0, 200000, (len(sections), n))
    pos[:, 0], pos[:, 1] = 0, 2 ** 24 + 1
    freq = (10000.0 ** (-np.arange(rot // 2) / (rot // 2))).astype(np.float32)
    slots = rng.permutation(2 * page)[:n]
    cache = tl.kv_cache(2, H, D, page, tl.TL_KV_E2M1)
    out = tl.kv_append(q.cuda(), k.cuda(), v.cuda(), cache, _int(slots), tl.rope(_int(pos), torch.from_numpy(freq).cuda(), sections, interleaved))
    ko, vo = tl.kv_read(cache, _int(slots))
    torch.cuda.synchronize()
    qd, kd = q.double().numpy(), k.double().numpy()
    q64, k64 = (_serve.rotate(x, pos, freq, sections, interleaved) for x in (qd, kd))
    slack = lambda x: 2.0 ** -20 * np.abs(x).max(-1, keepdims=True)  # noqa: E731
    got = out.cpu().double().numpy()
    assert (np.abs(got - q64) <= 2.0 ** -8 * np.abs(q64) + slack(qd)).all()
    got = ko.cpu().double().numpy()
    _, e = _serve4.quantise(k64)
    unit = np.repeat(np.exp2(e.astype(np.float64) - 127), 32, axis=-1)
    assert (np.abs(got - k64) <= np.maximum(2.0 ** -2 * np.abs(k64) * 1.0001, 2.0 * unit / 4) + slack(kd)).all()
    ref = _serve4.Cache4(2, H, D, page)
    for i, s in enumerate(slots):
        ref.put(s, k64[i], v[i].double().numpy())
    np.testing.assert_array_equal(vo.cpu().double().numpy(), ref.v[slots])


@pytest.mark.parametrize("n", [6, 600])
def test_append_specials(n):
    """Infinities and what is past the largest scale saturate, a NaN takes its block and no other, tiny values become zeros."""
    import torch
    banner(f"kv4 append specials n={n}")
    D, H = 64, 1
    k = torch.ones((n, H, D))
    k[0, 0, 5] = float("inf")
    k[1, 0, 6], k[1, 0, 7] = float("nan"), 3.0
    k[2, 0, 40] = -float("inf")
    k[3, 0, 0] = 3.4e38
    k[4] = 2.0 ** -149
    k[5] = float("nan")
    cache = tl.kv_cache(-(-n // 64), H, D, 64, tl.TL_KV_E2M1)
    slots = _int(np.arange(n))
    tl.kv_append(None, k.cuda(), k.cuda(), cache, slots)
    ko, vo = tl.kv_read(cache, slots)
    torch.cuda.synchronize()
    big = 6.0 * 2.0 ** 125
    for o in (ko.cpu().float(), vo.cpu().float()):
        assert o[0, 0, 5] == big and o[2, 0, 40] == -big and o[3, 0, 0] == big
        assert torch.isnan(o[1, 0, :32]).all() and (o[1, 0, 32:] == 1).all()
        assert not o[4].any() and torch.isnan(o[5]).all()
        assert not o[0, 0, 6:32].any() and (o[0, 0, 32:] == 1).all()


def test_slots_outside_and_either_half():
    import torch
    banner("kv4 append: slots outside the cache, queries alone, keys alone")
    D, H, Hq, page = 128, 2, 4, 64
    rng = np.random.default_rng(3)
    q, k, v = (_rows(rng, 5, h, D, True) for h in (Hq, H, H))
    ref, cache = _serve4.Cache4(2, H, D, page), _serve4.Cache4(2, H, D, page).device()
    slots = [-1, 128, 5, -2 ** 31, 2 ** 31 - 1]
    ref.put(5, k[2].double().numpy(), v[2].double().numpy())
    out = tl.kv_append(q.cuda(), None, None, cache, _int(slots))
    tl.kv_append(None, k.cuda(), v.cuda(), cache, _int(slots))
    torch.cuda.synchronize()
    assert torch.equal(out.cpu(), q)
    _same(cache, ref)


def test_float4_tensors_make_a_cache():
    import torch
    banner("kv4: float4_e2m1fn_x2 tensors")
    made = tl.kv_cache(2, 3, 64, 64, tl.TL_KV_E2M1)
    typed = tl.KVCache(made.k.view(torch.float4_e2m1fn_x2), made.v.view(torch.float4_e2m1fn_x2), made.k_exp, made.v_exp, 64, 3, 64)
    assert typed.elem_bytes == tl.TL_KV_E2M1 and typed.num_pages == 2
    x = torch.randn((7, 3, 64), device="cuda")
    tl.kv_append(None, x, -x, typed, _int(range(7)))
    k, v = tl.kv_read(made, _int(range(7)))
    torch.cuda.synchronize()
    assert torch.equal(k, -v) and (k.float() - x).abs().max() < 1.0


def test_cache_past_two_and_four_gigabytes():
    import torch
    D, H, page = 128, 8, 128
    pages = 72000                                          # 4.7 GB of keys, and of values
    banner("kv4 cache of 4.7 GB: first, middle and last pages")
    cache = tl.kv_cache(pages, H, D, page, tl.TL_KV_E2M1)
    slots = [0, 2 ** 31 // (H * D // 2) + 1, 2 ** 32 // (H * D // 2) + 65, pages * page - 1, pages * page - 100, 77]
    rng = np.random.default_rng(5)
    k, v = _rows(rng, 6, H, D, True), _rows(rng, 6, H, D, True)
    tl.kv_append(None, k.cuda(), v.cuda(), cache, _int(slots))
    ko, vo = tl.kv_read(cache, _int(slots))
    torch.cuda.synchronize()
    for got, x in ((ko, k), (vo, v)):
        np.testing.assert_array_equal(got.cpu().double().numpy(), _serve4.values(*_serve4.quantise(x.double().numpy())))


@pytest.mark.parametrize("D,H,page", [(128, 2, 64), (64, 3, 128)])
def test_keep_moves_entries(D, H, page):
    import torch
    banner(f"kv4 keep D={D} H={H} page={page}")
    rng = np.random.default_rng(D)
    most = 200                                             # more than a batch of entries
    starts = [0, 30, 2 * page - 3, 61, 5]
    paths = [[0], [0, 2, 3, 7, 8, 20], [0, 1, 2, 5, 6, 63], list(range(0, most)), list(range(0, 2 * most, 2))[:most]]
    B, per = len(starts), 7 * 64 // page + 3
    pages = B * per
    table = rng.permutation(pages).reshape(B, per)
    start = _serve4.Cache4(pages, H, D, page)
    for x in start.bytes():
        x[...] = rng.integers(0, 255, x.shape)
    path = np.full((B, most), -1)
    for b, p in enumerate(paths):
        path[b, :len(p)] = p
    counts = [len(p) for p in paths]
    counts[1] = 5                                          # the sixth entry stays where it is
    want = _serve4.Cache4(pages, H, D, page)
    B32, d = D // 32, np.arange(D // 2)
    # of a token: its bytes of keys (byte i of the head's D / 2) and values, its exponents
    key = lambda t: (t // 16 * B32 + d // 16) * 256 + t % 16 * 16 + d % 16  # noqa: E731
    val = lambda t: ((t // 64 * B32 + d // 16) * 4 + t % 16 // 4) * 256 + d % 16 * 16 + t % 64 // 16 * 4 + t % 4  # noqa: E731
    b32 = np.arange(B32)
    ke = lambda t: (t // 64 * B32 + b32) * 64 + t % 16 * 4 + t % 64 // 16  # noqa: E731
    ve = lambda t: (t // 64 * B32 + b32) * 64 + t % 16 // 4 * 16 + t % 64 // 16 * 4 + t % 4  # noqa: E731
    for x, y in zip(want.bytes(), start.bytes()):
        x[...] = y
    for b in range(B):
        for i in range(counts[b]):
            src, dst = starts[b] + path[b, i], starts[b] + i
            (p0, t0), (p1, t1) = (table[b, src // page], src % page), (table[b, dst // page], dst % page)
            for x, y, at in zip(want.bytes(), start.bytes(), (key, val, ke, ve)):
                x[p1][:, at(t1)] = y[p0][:, at(t0)]
    cache = start.device()
    tl.kv_keep(cache, _int(table), _int(starts), _int(path), _int(counts))
    torch.cuda.synchronize()
    _same(cache, want)


def test_streams_and_graph_replay():
    import torch
    banner("kv4 append / read / keep on a stream and in a graph")
    D, H, Hq, page, n = 128, 2, 8, 64, 40
    cache = tl.kv_cache(3, H, D, page, tl.TL_KV_E2M1)
    q, k, v = (torch.zeros((n, h, D), dtype=torch.bfloat16, device="cuda") for h in (Hq, H, H))
    slots, table = _int(np.arange(50, 50 + n)), _int([[0, 1, 2]])
    q_out, ko, vo = (torch.empty((n, h, D), dtype=torch.bfloat16, device="cuda") for h in (Hq, H, H))
    starts, path, counts = _int([50]), _int([[0, 3, 4, 9]]), _int([4])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())

    def work():
        tl.kv_append(q, k, v, cache, slots, None, q_out)
        tl.kv_keep(cache, table, starts, path, counts)
        tl.kv_read(cache, slots, ko, vo)

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
            np.testing.assert_array_equal(got.cpu().double().numpy(), _serve4.values(*_serve4.quantise(x.double().numpy()[order])))
        assert torch.equal(q_out.cpu(), new[0])
        torch.zeros(1000, device="cuda").sum().item()


@pytest.mark.parametrize("D,bf16,H,page", [(128, True, 2, 64), (64, False, 3, 128), (64, True, 5, 256)])
@pytest.mark.parametrize("start", [0, 1, 38])
def test_many_rows_at_once(D, bf16, H, page, start):
    """Rows enough for the kernels that take windows of tokens."""
    import torch
    n, Hq = 1100, 3
    banner(f"kv4 append / read of {n} rows D={D} bf16={bf16} H={H} page={page} start={start}")
    rng = np.random.default_rng(start + D)
    q, k, v = _rows(rng, n, Hq, D, bf16), _rows(rng, n, H, D, bf16), _rows(rng, n, H, D, bf16)
    pages = -(-(n + start + 200) // page) + 1
    slots = start + np.arange(n)
    slots[200:] += 50                                      # a jump
    slots[330:340] = slots[330:340][::-1]
    slots[400:403] = [-1, pages * page, -2 ** 31]
    slots[-1] = 2 ** 31 - 1
    ref = _serve4.Cache4(pages, H, D, page)
    for i, s in enumerate(slots):
        ref.put(s, k[i].double().numpy(), v[i].double().numpy())
    cache = _serve4.Cache4(pages, H, D, page).device()
    out = tl.kv_append(q.cuda(), k.cuda(), v.cuda(), cache, _int(slots))
    torch.cuda.synchronize()
    assert torch.equal(out.cpu(), q.to(torch.bfloat16))
    _same(cache, ref)
    inside = (slots >= 0) & (slots < pages * page)
    ko, vo = tl.kv_read(cache, _int(slots))
    torch.cuda.synchronize()
    for got, want in ((ko, ref.k), (vo, ref.v)):
        got = got.cpu().double().numpy()
        np.testing.assert_array_equal(got[inside], want[slots[inside]])
        assert not got[~inside].any()
    only = torch.full((n, H, D), 7.0, dtype=torch.bfloat16, device="cuda")
    tl.tl_kv_read(cache, _int(slots), n, None, only)
    torch.cuda.synchronize()
    assert torch.equal(only, vo)
