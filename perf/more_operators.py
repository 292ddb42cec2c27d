"""A key/value cache held in 4 bits, attention over it, and the management of a
cache's pages, as cases to measure.

  kv4       the rows that a QKV projection left: rotary positions on queries
            and keys, keys and values written into the pages of a 4-bit cache
            (E2M1 with a power-of-two scale per token, head and 32 elements),
            and the written entries read back
  attn4     attention of the new tokens of every sequence over such pages:
            single tokens, chains, trees of drafted tokens and whole prompts
  fork      sequences go on in several ways (beams, parallel samples): a child
            shares its parent's full pages and gets a copy of the last one
  compact   pages in use move to the front of the pool, every table follows
  turnover  finished sequences give their pages back, the others get pages for
            their next tokens

`own` chooses between the plain form in torch operations and the library's
calls.  The cache tensors have the library's page layout in both.
"""
import math

import torch

own = False

# (query heads, key/value heads, head size): a Llama-3.1-70B-shaped layer, one GPU's share of it under 8-way
# tensor parallelism, a Qwen-3-30B-A3B-shaped layer, and a layer of hidden size 768
HEADS = {"dense": (64, 8, 128), "dense_tp8": (8, 1, 128), "experts": (32, 4, 128), "small": (12, 12, 64)}
BLOCK = 32                                              # elements of a head that share a scale
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)         # the values of the codes 0 .. 7; code + 8: the negative ones


def listed():
    return [
        # one token of one sequence enters the cache: launches and latency are everything
        kv4("kv4_one_token", heads="experts", n=1, src="bf16", axes=1, page=64),
        # a long prompt, from a projection that writes bf16
        kv4("kv4_prompt", heads="dense", n=8192, src="bf16", axes=1, page=128),
        # one token of one short sequence, every query head with its own key head
        attn4("attn4_one_token", heads="small", form="causal", seqs=1, new=1, length=517, page=64),
        # the ordinary decode step of a batch of sequences of different lengths
        attn4("attn4_decode_batch", heads="dense", form="causal", seqs=32, new=1, length=8192, page=64),
        # few very long sequences on one GPU of eight, a chain of five drafted tokens each
        attn4("attn4_long_chain", heads="dense_tp8", form="causal", seqs=3, new=5, length=131072, page=128),
        # prompts, each partly in the cache already
        attn4("attn4_prompt", heads="experts", form="causal", seqs=3, new=2048, length=4096, page=128),
        # one sequence is sampled in four ways
        fork("fork_one", heads="experts", seqs=1, beams=3, length=517, cache="fp8", page=64, load=50),
        # a batch of beam searches on one GPU of eight, in a pool of 16000 pages
        fork("fork_batch", heads="dense_tp8", seqs=64, beams=7, length=24000, cache="fp8", page=64, load=97),
        # a small pool after a few sequences ended
        compact("compact_small", heads="experts", seqs=5, length=700, cache="bf16", page=64, load=60),
        # half of a pool of 16000 pages is in use, in random places
        compact("compact_pool", heads="dense_tp8", seqs=64, length=12800, cache="fp8", page=64, load=50),
        # a batch of eight, two of which end
        turnover("turnover_small", seqs=8, length=1000, page=64, load=50),
        # a batch of 512 sequences, a quarter of which ends
        turnover("turnover_batch", seqs=512, length=16384, page=64, load=90),
    ]


def _named(name, case):
    return dict(case, name=name) if name else case


def kv4(name, heads, n, src, axes, page):
    return _named(name, {"kind": "kv4", "heads": heads, "n": n, "src": src, "axes": axes, "page": page})


def attn4(name, heads, form, seqs, new, length, page):
    return _named(name, {"kind": "attn4", "heads": heads, "form": form, "seqs": seqs, "new": new, "length": length, "page": page})


def fork(name, heads, seqs, beams, length, cache, page, load):
    return _named(name, {"kind": "fork", "heads": heads, "seqs": seqs, "beams": beams, "length": length, "cache": cache,
                         "page": page, "load": load})


def compact(name, heads, seqs, length, cache, page, load):
    return _named(name, {"kind": "compact", "heads": heads, "seqs": seqs, "length": length, "cache": cache, "page": page,
                         "load": load})


def turnover(name, seqs, length, page, load):
    return _named(name, {"kind": "turnover", "seqs": seqs, "length": length, "page": page, "load": load})


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("kv4", "kv4", "attn4", "attn4", "attn4", "attn4", "fork", "compact", "turnover"))
    heads, page = rng.choice(tuple(HEADS)), rng.choice((64, 128, 256))
    Hq, Hk, D = HEADS[heads]
    if kind == "kv4":
        return kv4(None, heads, _log(rng, 1, 8192), rng.choice(("bf16", "f32")), rng.choice((0, 1, 1, 3)), page)
    if kind == "attn4":
        form = rng.choice(("one", "chain", "tree", "tree", "prompt"))
        while True:
            seqs, length = _log(rng, 1, 64), _log(rng, 1, 131072)
            new = {"one": 1, "chain": rng.randint(2, 8), "tree": rng.randint(3, 64), "prompt": _log(rng, 65, 2048)}[form]
            if new <= length and seqs * length * Hk * D <= 32 * 8192 * 8 * 128 and \
                    seqs * new * length * Hq * D <= 3 * 2048 * 4096 * 32 * 128:
                return attn4(None, heads, "tree" if form == "tree" else "causal", seqs, new, length, page)
    cache, load = rng.choice(("fp8", "bf16")), rng.randint(30, 99)
    if kind == "turnover":
        return turnover(None, _log(rng, 1, 512), _log(rng, 1, 16384), page, load)
    while True:
        seqs, beams, length = _log(rng, 1, 128), rng.randint(1, 8), _log(rng, 1, 24000)
        case = fork(None, heads, seqs, beams, length, cache, page, load) if kind == "fork" else \
            compact(None, heads, seqs, length, cache, page, load)
        if _pool(case) * page * Hk * D * (1 if cache == "fp8" else 2) <= 16384 * 64 * 128:
            return case


# ---------------------------------------------------------------------------
# Inputs, from the seed alone
# ---------------------------------------------------------------------------

def _gen(seed, i):
    return torch.Generator(device="cuda").manual_seed(seed * 1013 + i)


def _host_gen(seed, i):
    return torch.Generator().manual_seed(seed * 1013 + i)


def _normal(shape, seed, i, dtype=torch.float32):
    return torch.randn(shape, generator=_gen(seed, i), device="cuda", dtype=torch.float32).to(dtype)


def _dtype(name):
    return {"f32": torch.float32, "bf16": torch.bfloat16}[name]


def _ragged(count, most, salt):
    """count sizes of [most / 4, most], the first of them the largest, the same for every seed: int64 on the host."""
    g = torch.Generator().manual_seed(most * 4099 + count * 17 + salt)
    sizes = torch.randint(max(1, most // 4), most + 1, (count,), generator=g)
    sizes[0] = most
    return sizes


def _lens(case):
    return _ragged(case["seqs"], case["length"], 2)


def _sizes(case):
    """The lengths of attn4's sequences and their new tokens, the same for every seed."""
    lens = _lens(case)
    return lens, torch.minimum(_ragged(case["seqs"], case["new"], 1), lens)


def _pages(lens, page):
    return -(-lens // page)


def _pool(case):
    """Pages of a pool of which `load` percent are in use once the pass is done (at least one of them free before it)."""
    need = int(_pages(_lens(case), case["page"]).sum())
    if case["kind"] == "fork":
        need += case["seqs"] * case["beams"]
    if case["kind"] == "turnover":
        need += 2 * case["seqs"]
    return -(-need * 100 // case["load"]) + 1


def _offsets(sizes):
    out = torch.zeros(len(sizes) + 1, dtype=torch.int64)
    out[1:] = sizes.cumsum(0)
    return out


def _dev(t):
    return t.to(torch.int32).cuda()


def _trees(seed, i, sizes, siblings):
    """A tree per sequence: the parent (an earlier node of the sequence, -1 at node 0) of every node; flat, on the host."""
    pick = torch.rand(int(sizes.sum()), generator=_host_gen(seed, i)).tolist()
    parent, at = [], 0
    for n in sizes.tolist():
        children, free = [0] * n, [0]
        for j in range(n):
            if j == 0:
                parent.append(-1)
                continue
            # the newest nodes are the likeliest parents: paths of some depth
            k = len(free) - 1 - int(pick[at + j] ** 2 * len(free))
            p = free[k]
            parent.append(p)
            children[p] += 1
            if children[p] == siblings:
                free.pop(k)
            free.append(j)
        at += n
    return torch.tensor(parent)


def _tree_mask(parent, sizes, words):
    """Bits of the nodes that each node sees (its ancestors and itself): int32 [nodes, words], on the host."""
    bits, rows, at = parent.tolist(), [], 0
    for n in sizes.tolist():
        for j in range(n):
            p = bits[at + j]
            rows.append((rows[at + p] if p >= 0 else 0) | 1 << j)
        at += n
    out = torch.tensor([[(r >> 32 * w & 0xffffffff) for w in range(words)] for r in rows], dtype=torch.int64)
    return torch.where(out >= 1 << 31, out - (1 << 32), out).to(torch.int32)


def _blocks_exponent(amax):
    """The smallest e with amax <= 6 * 2^e, kept within -126 .. 125."""
    m, e = torch.frexp(amax)
    return torch.where(amax > 0, torch.where(m <= 0.75, e - 3, e - 2), 0).clamp(-126, 125)


def _to_e2m1(x):
    """[..., elements] -> codes (uint8) and exponents [..., elements / 32]: each element times 2^-e to the nearest of
    E2M1's values, ties to the even code."""
    x = x.unflatten(-1, (-1, BLOCK))
    e = _blocks_exponent(x.abs().amax(dim=-1))
    y = (x * torch.exp2(-e.float())[..., None]).clamp(-6, 6)
    a = y.abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    a = torch.round(a / step) * step
    code = torch.where(a < 2, 2 * a, torch.where(a < 4, a + 2, a / 2 + 4)).to(torch.uint8)
    return (code | (torch.signbit(x) * 8).to(torch.uint8)).flatten(-2), e


def _key_bytes(code):
    """Codes [..., D] -> the bytes of each block of 32 elements, two neighbours a byte: [..., D / 32, 16]."""
    c = code.unflatten(-1, (-1, BLOCK // 2, 2))
    return c[..., 0] | c[..., 1] << 4


def _value_bytes(code):
    """Codes [..., D] -> the bytes of each block of 32 elements, element d and d + 16 a byte: [..., D / 32, 16]."""
    c = code.unflatten(-1, (-1, 2, BLOCK // 2))
    return c[..., 0, :] | c[..., 1, :] << 4


def _cache4(case, pages, seed):
    """A pool of 4-bit pages that holds earlier tokens: keys and values, and the exponents of their blocks, biased by 127.
    With B = D / 32 blocks of a head:
      k      [page][head][t / 16][B][t % 16][16 bytes]     k_exp  [page][head][t / 64][B][t % 16][t % 64 / 16]
      v      [page][head][t / 64][B][t % 16 / 4][d % 16][t % 64 / 16][t % 4]
      v_exp  [page][head][t / 64][B][t % 16 / 4][t % 64 / 16][t % 4]"""
    _, H, D = HEADS[case["heads"]]
    T, B, made = case["page"], HEADS[case["heads"]][2] // BLOCK, {}
    for i, name in enumerate(("k", "v")):
        code, e = _to_e2m1(_normal((pages, H, T, D), seed, 100 + i, torch.bfloat16).float())
        e = (e + 127).to(torch.uint8)
        if name == "k":
            data = _key_bytes(code).view(pages, H, T // 16, 16, B, 16).permute(0, 1, 2, 4, 3, 5)
            e = e.view(pages, H, T // 64, 4, 16, B).permute(0, 1, 2, 5, 4, 3)
        else:
            data = _value_bytes(code).view(pages, H, T // 64, 4, 4, 4, B, 16).permute(0, 1, 2, 6, 4, 7, 3, 5)
            e = e.view(pages, H, T // 64, 4, 4, 4, B).permute(0, 1, 2, 6, 4, 3, 5)
        made[name] = data.contiguous().view(pages, H, T * D // 2)
        made[name + "_exp"] = e.contiguous().view(pages, H, T * B)
    return dict(made, pages=pages, page=T, heads=H, size=D)


def _cache(case, pages, seed):
    """A pool of pages in 8 bits (any finite bytes) or bf16, whose order inside a page does not matter here."""
    _, H, D = HEADS[case["heads"]]
    T, made = case["page"], {"k_exp": None, "v_exp": None}
    for i, name in enumerate(("k", "v")):
        if case["cache"] == "bf16":
            made[name] = _normal((pages, H, T * D), seed, 100 + i, torch.bfloat16)
        else:
            made[name] = _normal((pages, H, T * D), seed, 100 + i).to(torch.float8_e4m3fn).view(torch.uint8)
            made[name + "_exp"] = torch.randint(110, 140, (pages, H, T), generator=_gen(seed, 102 + i), device="cuda",
                                                dtype=torch.uint8)
    return dict(made, pages=pages, page=T, heads=H, size=D)


def _table(lens, page, seed, pages=None, width=None):
    """Pages for every sequence, in random order over the pool: int32 [sequences, most pages] on the host."""
    need = _pages(lens, page)
    pool = torch.randperm(int(need.sum()) if pages is None else pages, generator=_host_gen(seed, 50))
    table, at = torch.full((len(lens), int(need.max()) if width is None else width), -1), 0
    for b, c in enumerate(need.tolist()):
        table[b, :c] = pool[at:at + c]
        at += c
    return table


def prepare(case, seed):
    return {"kv4": _prepare_kv4, "attn4": _prepare_attn4, "fork": _prepare_fork, "compact": _prepare_compact,
            "turnover": _prepare_turnover}[case["kind"]](case, seed)


def _prepare_kv4(case, seed):
    Hq, Hk, D = HEADS[case["heads"]]
    n, page = case["n"], case["page"]
    qkv = _normal((n, (Hq + 2 * Hk) * D), seed, 1, _dtype(case["src"]))
    qkv[:, Hq * D:(Hq + Hk) * D:37] *= 8   # some key channels are much larger than the rest
    pages = -(-n // page) + 3
    # consecutive tokens in consecutive places of pages in random order, the first one inside a page
    slots = []
    for p in torch.randperm(pages, generator=_host_gen(seed, 2)).tolist():
        slots += range(p * page, p * page + page)
    skip = int(torch.randint(0, 2 * page, (1,), generator=_host_gen(seed, 3)))
    s = {"kind": "kv4", "q": qkv[:, :Hq * D], "k": qkv[:, Hq * D:(Hq + Hk) * D], "v": qkv[:, (Hq + Hk) * D:], "n": n,
         "q_heads": Hq, "slots": _dev(torch.tensor(slots[skip:skip + n])), "cache": _cache4(case, pages, seed),
         "axes": case["axes"],
         "q_out": torch.empty((n, Hq, D), dtype=torch.bfloat16, device="cuda"),
         "k_out": torch.empty((n, Hk, D), dtype=torch.bfloat16, device="cuda"),
         "v_out": torch.empty((n, Hk, D), dtype=torch.bfloat16, device="cuda")}
    if case["axes"]:
        first = int(torch.randint(0, 4096, (1,), generator=_host_gen(seed, 4)))
        if case["axes"] == 3:   # images of 24 x 32 patches: one time, rows and columns
            pos = torch.stack([first + torch.arange(n) // 768, first + torch.arange(n) // 32 % 24,
                               first + torch.arange(n) % 32])
            s["sections"] = (D // 8, 3 * D // 16, 3 * D // 16)
        else:
            pos, s["sections"] = (first + torch.arange(n))[None], (D // 2,)
        s["positions"] = _dev(pos)
        s["inv_freq"] = (500000.0 ** (-torch.arange(0, D, 2, dtype=torch.float64) / D)).float().cuda()
    return s


def _prepare_attn4(case, seed):
    Hq, Hk, D = HEADS[case["heads"]]
    lens, new = _sizes(case)
    order = torch.randperm(len(new), generator=_host_gen(seed, 10))
    lens, new = lens[order], new[order]
    total = int(new.sum())
    s = {"kind": "attn4", "cache": _cache4(case, int(_pages(lens, case["page"]).sum()), seed),
         "table": _dev(_table(lens, case["page"], seed)), "lens": _dev(lens), "offsets": _dev(_offsets(new)),
         "total": total, "max_q": int(new.max()), "max_len": int(lens.max()), "q_heads": Hq, "scale": D ** -0.5,
         "mask": None, "seqs": case["seqs"], "q": (_normal((total, Hq, D), seed, 12) * 2).to(torch.bfloat16),
         "out": torch.empty((total, Hq, D), dtype=torch.bfloat16, device="cuda")}
    if case["form"] == "tree":
        s["mask"] = _tree_mask(_trees(seed, 13, new, 4), new, -(-case["new"] // 32)).cuda()
    return s


def _given(table, pages, **more):
    """The scheduler's view of a pool, as it comes from the host before every step: the references of every page and the
    table in one piece, and the tensors that a step works on."""
    used = table[table >= 0]
    refs = torch.zeros(pages, dtype=torch.int64).index_add_(0, used, torch.ones_like(used))
    given = _dev(torch.cat([refs, table.flatten()]))
    work_on = given.clone()
    return dict(more, given=given, tables=work_on, refs=work_on[:pages], table=work_on[pages:].view(table.shape), pages=pages)


def _ints(n):
    return torch.empty(n, dtype=torch.int32, device="cuda")


def _prepare_fork(case, seed):
    lens, page, beams = _lens(case), case["page"], case["beams"]
    lens = lens[torch.randperm(len(lens), generator=_host_gen(seed, 10))]
    B, pages = len(lens), _pool(case)
    width = int(_pages(lens, page).max()) + 4           # room for the tokens to come
    rows = torch.randperm(B * (1 + beams), generator=_host_gen(seed, 11))
    table = torch.full((len(rows), width), -1)
    table[rows[:B]] = _table(lens, page, seed, pages, width)
    n = B * beams
    return _given(table, pages, kind="fork", page=page, cache=_cache(case, pages, seed), n=n,
                  parents=_dev(rows[:B].repeat_interleave(beams)), children=_dev(rows[B:]),
                  lens=_dev(lens.repeat_interleave(beams)), out=(_ints(n), _ints(n), _ints(n), _ints(2)))


def _prepare_compact(case, seed):
    lens, page, pages = _lens(case), case["page"], _pool(case)
    lens = lens[torch.randperm(len(lens), generator=_host_gen(seed, 10))]
    table = _table(lens, page, seed, pages, int(_pages(lens, page).max()) + 4)
    most = pages // 2 + 1
    return _given(table, pages, kind="compact", page=page, cache=_cache(case, pages, seed), most=most,
                  out=(_ints(most), _ints(most), _ints(2)))


def _prepare_turnover(case, seed):
    lens, page, pages = _lens(case), case["page"], _pool(case)
    lens = lens[torch.randperm(len(lens), generator=_host_gen(seed, 10))]
    table = _table(lens, page, seed, pages, int(_pages(lens, page).max()) + 4)
    order, ended = torch.randperm(len(lens), generator=_host_gen(seed, 11)), len(lens) // 4
    more = torch.randint(1, 2 * page, (len(lens),), generator=_host_gen(seed, 12))
    return _given(table, pages, kind="turnover", page=page, ended=_dev(order[:ended]), going=_dev(order[ended:]),
                  lens=_dev((lens + more)[order[ended:]]), missing=_ints(1))


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------

def run(s):
    if "given" in s:
        s["tables"].copy_(s["given"])       # the step's tables, as the scheduler hands them over
    if own:
        return _own(s)
    return {"kv4": _plain_kv4, "attn4": _plain_attn4, "fork": _plain_fork, "compact": _plain_compact,
            "turnover": _plain_turnover}[s["kind"]](s)


def _handle(c):
    """The library's handle of the cache's tensors, which a program keeps as long as the cache."""
    import paper_2607_04031_amd as tl
    if "handle" not in c:
        four = c["k"].dtype == torch.uint8 and c["k"].numel() * 2 == c["pages"] * c["page"] * c["heads"] * c["size"]
        c["handle"] = tl.KVCache(c["k"], c["v"], c["k_exp"], c["v_exp"], c["page"], c["heads"], c["size"],
                                 elem_bytes=tl.TL_KV_E2M1 if four else None)
    return c["handle"]


def _pool_handle(s):
    """The library's handle of a pool's references and page table, which a program keeps as well."""
    import paper_2607_04031_amd as tl
    if "pool" not in s:
        s["pool"] = tl.KVPages(s["refs"], s["table"], s["page"])
    return s["pool"]


def _own(s):
    import paper_2607_04031_amd as tl
    if s["kind"] == "kv4":
        rope = tl.rope(s["positions"], s["inv_freq"], s["sections"]) if s["axes"] else None
        tl.kv_append(s["q"], s["k"], s["v"], _handle(s["cache"]), s["slots"], rope, q_out=s["q_out"])
        tl.kv_read(_handle(s["cache"]), s["slots"], s["k_out"], s["v_out"])
        return [s["q_out"], s["k_out"], s["v_out"]]
    if s["kind"] == "attn4":
        return tl.attention(s["q"], _handle(s["cache"]), s["table"], s["lens"], s["offsets"], s["max_q"], s["max_len"],
                            s["scale"], mask=s["mask"], out=s["out"])
    if s["kind"] == "fork":
        src, dst, tokens, count = tl.kv_fork(_pool_handle(s), s["parents"], s["children"], s["lens"], out=s["out"])
        tl.kv_copy(_handle(s["cache"]), src, dst, tokens, count)
        return [s["refs"], s["table"], src, dst, tokens, count] + _contents(s["cache"])
    if s["kind"] == "compact":
        src, dst, count = tl.kv_compact(_pool_handle(s), s["most"], out=s["out"])
        tl.kv_copy(_handle(s["cache"]), src, dst, count=count)
        return [s["refs"], s["table"], src, dst, count] + _contents(s["cache"])
    tl.kv_free(_pool_handle(s), s["ended"])
    tl.kv_grow(_pool_handle(s), s["going"], s["lens"], missing=s["missing"])
    return [s["refs"], s["table"], s["missing"]]


def _contents(c):
    if c["k_exp"] is None:
        return [c["k"], c["v"]]
    return [c["k"].view(torch.float8_e4m3fn), c["v"].view(torch.float8_e4m3fn), c["k_exp"], c["v_exp"]]


def _rotate(x, s):
    """Elements d and d + D / 2 of every head turned by position * inv_freq[d], the position of d's axis; angles in 64 bits."""
    D, at, angle = x.shape[-1], 0, []
    for axis, width in enumerate(s["sections"]):
        angle.append(s["positions"][axis].double()[:, None] * s["inv_freq"][at:at + width].double())
        at += width
    angle = torch.cat(angle, dim=1)[:, None]
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    a, b = x[..., :D // 2], x[..., D // 2:]
    return torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)


def _views4(c):
    """Keys, their exponents, values, their exponents with the axes that _cache4 names."""
    P, H, T, B = c["pages"], c["heads"], c["page"], c["size"] // BLOCK
    return (c["k"].view(P, H, T // 16, B, 16, 16), c["k_exp"].view(P, H, T // 64, B, 16, 4),
            c["v"].view(P, H, T // 64, B, 4, 16, 16), c["v_exp"].view(P, H, T // 64, B, 4, 16))


def _e2m1(code):
    return torch.tensor(E2M1 + tuple(-x for x in E2M1), device=code.device)[code.int()]


def _plain_kv4(s):
    c, n = s["cache"], s["n"]
    H, D, T = c["heads"], c["size"], c["page"]
    q, k, v = s["q"].float().view(n, s["q_heads"], D), s["k"].float().view(n, H, D), s["v"].float().view(n, H, D)
    if s["axes"]:
        q, k = _rotate(q, s), _rotate(k, s)
    keys, k_exp, values, v_exp = _views4(c)
    slots = s["slots"].long()
    p, t = slots // T, slots % T
    at = t % 64 // 16 * 4 + t % 4           # a value's place among the 16 of its lane
    code, e = _to_e2m1(k)
    keys[p, :, t // 16, :, t % 16] = _key_bytes(code)
    k_exp[p, :, t // 64, :, t % 16, t % 64 // 16] = (e + 127).to(torch.uint8)
    code, e = _to_e2m1(v)
    values[p, :, t // 64, :, t % 16 // 4, :, at] = _value_bytes(code)
    v_exp[p, :, t // 64, :, t % 16 // 4, at] = (e + 127).to(torch.uint8)
    kb, ke = keys[p, :, t // 16, :, t % 16], k_exp[p, :, t // 64, :, t % 16, t % 64 // 16]
    vb, ve = values[p, :, t // 64, :, t % 16 // 4, :, at], v_exp[p, :, t // 64, :, t % 16 // 4, at]
    k = _e2m1(torch.stack([kb & 15, kb >> 4], dim=-1).flatten(-2)) * torch.exp2(ke.float() - 127)[..., None]
    v = _e2m1(torch.cat([vb & 15, vb >> 4], dim=-1)) * torch.exp2(ve.float() - 127)[..., None]
    return [q.to(torch.bfloat16), k.view(n, H, D).to(torch.bfloat16), v.view(n, H, D).to(torch.bfloat16)]


def _gathered(c, table):
    """The pages of every sequence as float32 [sequences, heads, tokens, head size]: keys and values."""
    keys, k_exp, values, v_exp = _views4(c)
    N, H, L, D = table.shape[0], c["heads"], table.shape[1] * c["page"], c["size"]
    at = table.long().clamp(min=0)
    kb = keys[at].permute(0, 2, 1, 3, 5, 4, 6).reshape(N, H, L, D // BLOCK, 16)
    ke = k_exp[at].permute(0, 2, 1, 3, 6, 5, 4).reshape(N, H, L, D // BLOCK)
    vb = values[at].unflatten(-1, (4, 4)).permute(0, 2, 1, 3, 7, 5, 8, 4, 6).reshape(N, H, L, D // BLOCK, 16)
    ve = v_exp[at].unflatten(-1, (4, 4)).permute(0, 2, 1, 3, 6, 5, 7, 4).reshape(N, H, L, D // BLOCK)
    k = _e2m1(torch.stack([kb & 15, kb >> 4], dim=-1).flatten(-2)).mul_(torch.exp2(ke.float() - 127)[..., None])
    v = _e2m1(torch.cat([vb & 15, vb >> 4], dim=-1)).mul_(torch.exp2(ve.float() - 127)[..., None])
    return k.view(N, H, L, D), v.view(N, H, L, D)


def _row_places(offsets, total):
    """The sequence of each row, and its place in it."""
    rows = torch.arange(total, device=offsets.device)
    seq = (rows[:, None] >= offsets[None, 1:]).sum(dim=1)
    return seq, rows - offsets[seq]


def _plain_attn4(s):
    c, B, n, Hq, total = s["cache"], s["seqs"], s["max_q"], s["q_heads"], s["total"]
    H, D, G = c["heads"], c["size"], s["q_heads"] // c["heads"]
    k, v = _gathered(c, s["table"])
    L = k.shape[2]
    offsets, lens = s["offsets"].long(), s["lens"].long()
    seq, place = _row_places(offsets, total)
    q = torch.zeros((B, n, Hq, D), dtype=torch.float32, device="cuda")
    q[seq, place] = s["q"].float()
    q = q.view(B, n, H, G, D).permute(0, 2, 1, 3, 4).reshape(B, H, n * G, D)
    # which key each new token sees: all before the new ones, and of those its own past or its tree's bits
    start = lens - (offsets[1:] - offsets[:-1])
    key = torch.arange(L, device="cuda")
    new = key[None] - start[:, None]                                       # [B, L]: a key's place among the new tokens
    if s["mask"] is None:
        seen = new[:, None] <= torch.arange(n, device="cuda")[None, :, None]
    else:
        words = s["mask"].shape[1]
        bits = torch.zeros((B, n, words), dtype=torch.int64, device="cuda")
        bits[seq, place] = s["mask"].long()
        at = new.clamp(0, 32 * words - 1)[:, None].expand(B, n, L)
        seen = (new < 0)[:, None] | ((bits.gather(2, at // 32) >> at % 32 & 1).bool() & (new < 32 * words)[:, None])
    seen = seen & (key[None] < lens[:, None])[:, None]
    scores = torch.matmul(q, k.transpose(2, 3).contiguous()).view(B, H, n, G, L) * s["scale"]
    scores = scores.masked_fill_(~seen[:, None, :, None], float("-inf"))
    top = scores.amax(dim=-1, keepdim=True)
    p = torch.exp(scores.sub_(torch.where(top == float("-inf"), 0.0, top)))
    total_p = p.sum(dim=-1, keepdim=True)
    o = torch.matmul(p.view(B, H, n * G, L), v).view(B, H, n, G, D)
    o = torch.where(total_p > 0, o / total_p, 0.0).permute(0, 2, 1, 3, 4).reshape(B, n, Hq, D)
    return o[seq, place].to(torch.bfloat16)


def _copy_pages(c, src, dst, tokens):
    """The first tokens of pages src to pages dst, in whole groups of 64."""
    T, H = c["page"], c["heads"]
    moved = torch.arange(T // 64, device="cuda")[None] * 64 < tokens[:, None]
    pair, group = moved.nonzero(as_tuple=True)
    for name in ("k", "v", "k_exp", "v_exp"):
        if c[name] is not None:
            x = c[name].view(c["pages"], H, T // 64, -1)
            x[dst[pair], :, group] = x[src[pair], :, group]


def _listed_pairs(pairs, most, *columns):
    """The chosen rows of every column first, in order, then -1; and how many they are."""
    order = torch.argsort(~pairs, stable=True)[:most]
    count = pairs.sum()
    there = torch.arange(most, device="cuda") < count
    return [torch.where(there, x[order], -1).int() for x in columns], count


def _free_pages(refs):
    """The free pages in rising order, then the others; and how many are free."""
    return torch.argsort(refs > 0, stable=True), (refs == 0).sum()


def _plain_fork(s):
    refs, table, T = s["refs"], s["table"], s["page"]
    lens, parents, children = s["lens"].long(), s["parents"].long(), s["children"].long()
    full, last = lens // T, lens % T
    column = torch.arange(table.shape[1], device="cuda")
    rows = table[parents]
    share = (column[None] < full[:, None]) & (rows >= 0)
    free, count = _free_pages(refs)
    from_page = rows.gather(1, full.clamp(max=table.shape[1] - 1)[:, None])[:, 0]
    wants = (last > 0) & (from_page >= 0)
    place = wants.cumsum(0) - 1
    gets = wants & (place < count)
    page = torch.where(gets, free[place.clamp(0, len(free) - 1)], -1).int()
    refs.index_add_(0, torch.where(share, rows, 0).flatten(), share.int().flatten())
    refs.index_add_(0, page.clamp(min=0), gets.int())
    made = torch.where(share, rows, -1)
    made = torch.where((column[None] == full[:, None]) & gets[:, None], page[:, None], made)
    table[children] = made
    (src, dst, tokens), pairs = _listed_pairs(gets, s["n"], from_page, page, last)
    _copy_pages(s["cache"], src.long().clamp(min=0), dst.long().clamp(min=0), tokens)
    return [refs, table, src, dst, tokens, torch.stack([pairs, (wants & ~gets).sum()]).int()] + _contents(s["cache"])


def _plain_compact(s):
    refs, table, most, P = s["refs"], s["table"], s["most"], s["pages"]
    free, _ = _free_pages(refs)
    used = P - 1 - torch.argsort(refs.flip(0) == 0, stable=True)            # the pages in use in falling order, then the others
    n = (refs > 0).sum()
    k = torch.arange(most, device="cuda")
    dst, src = free[:most], used[:most]
    moves = (k < torch.minimum(n, P - n)) & (dst < src)
    (src, dst), count = _listed_pairs(moves, most, src, dst)
    a, b = src[src >= 0].long(), dst[dst >= 0].long()
    name = torch.arange(P, device="cuda", dtype=torch.int32)
    name[a] = b.int()
    refs[b] = refs[a]
    refs[a] = 0
    table.copy_(torch.where(table >= 0, name[table.clamp(min=0).long()], table))
    for x in (s["cache"][name] for name in ("k", "v", "k_exp", "v_exp")):
        if x is not None:
            x[b] = x[a]
    return [refs, table, src, dst, torch.stack([count, n]).int()] + _contents(s["cache"])


def _plain_turnover(s):
    refs, table, T = s["refs"], s["table"], s["page"]
    ended, going = s["ended"].long(), s["going"].long()
    pages = table[ended]
    refs.index_add_(0, pages.clamp(min=0).flatten(), -(pages >= 0).int().flatten())
    table[ended] = -1
    need = -(-s["lens"].long() // T)
    rows = table[going]
    wants = (torch.arange(table.shape[1], device="cuda")[None] < need[:, None]) & (rows < 0)
    free, count = _free_pages(refs)
    place = wants.flatten().cumsum(0).view(wants.shape) - 1
    gets = wants & (place < count)
    page = torch.where(gets, free[place.clamp(0, len(free) - 1)].int(), rows)
    refs.index_add_(0, page.clamp(min=0).flatten(), gets.int().flatten())
    table[going] = page
    return [refs, table, (wants & ~gets).sum().int().view(1)]


# ---------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------

def _entry_bytes(case):
    """Keys and values of one token and key head."""
    D = HEADS[case["heads"]][2]
    return D + 2 * D // BLOCK if "cache" not in case else 2 * (D + 1) if case["cache"] == "fp8" else 4 * D


def work(case):
    if case["kind"] == "kv4":
        Hq, H, D = HEADS[case["heads"]]
        n, src = case["n"], 4 if case["src"] == "f32" else 2
        # the projection's rows, the rotated queries, the cache entries written, and them read back to bf16
        return {"bytes": n * ((Hq + 2 * H) * D * src + Hq * D * 2 + 2 * H * _entry_bytes(case) + 2 * H * D * 2 + 4 * case["axes"] + 4),
                "flops": n * (Hq + H) * D * 3 if case["axes"] else n * H * D}
    if case["kind"] == "attn4":
        Hq, H, D = HEADS[case["heads"]]
        lens, new = _sizes(case)
        rows = int(new.sum())
        if case["form"] == "causal":
            seen = int((new * (lens - new) + new * (new + 1) // 2).sum())
        else:   # the tokens before the tree; of the tree, a few ancestors each
            seen = int((new * (lens - new)).sum()) + rows
        return {"bytes": int(lens.sum()) * H * _entry_bytes(case) + 4 * rows * Hq * D, "flops": 4 * seen * Hq * D}
    lens, page, pool = _lens(case), case["page"], _pool(case)
    need = int(_pages(lens, page).sum())
    if case["kind"] == "fork":
        # parents' pages, children's rows, the references, and a read and a write of every part of a page that is copied
        last = lens % page
        moved = case["beams"] * int((-(-last // 64) * 64).sum())
        return {"bytes": 4 * (need * (1 + case["beams"]) + 2 * pool) + 2 * moved * HEADS[case["heads"]][1] * _entry_bytes(case), "flops": 0}
    if case["kind"] == "compact":
        # of pages in random places, the share of the pages in use that lies behind their number
        moved = need * (pool - need) / pool * page
        return {"bytes": 4 * (2 * need + 2 * pool) + 2 * moved * HEADS[case["heads"]][1] * _entry_bytes(case), "flops": 0}
    return {"bytes": 4 * (2 * need + 2 * pool), "flops": 0}


# ---------------------------------------------------------------------------
# The definitions in 64 bits
# ---------------------------------------------------------------------------

def exact(case, seed):
    if case["kind"] == "kv4":
        return _exact_kv4(case, seed)
    if case["kind"] == "attn4":
        return _exact_attn4(case, seed)
    return None if case["kind"] == "turnover" else _exact_moved(case, seed)     # turnover: whole numbers only


def _exact_moved(case, seed):
    """The pages' contents, page by page in the order in which free pages are handed out; the whole numbers have no such value."""
    s = prepare(case, seed)
    c, T, refs, pairs = s["cache"], s["page"], s["refs"].tolist(), []
    free = [p for p, r in enumerate(refs) if r == 0]
    if case["kind"] == "fork":
        table = s["table"].tolist()
        for parent, n in zip(s["parents"].tolist(), s["lens"].tolist()):
            if n % T:
                pairs.append((table[parent][n // T], free.pop(0), -(-(n % T) // 64)))
    else:
        for a, b in zip([p for p, r in reversed(list(enumerate(refs))) if r], free):
            if b < a:
                pairs.append((a, b, T // 64))
    out = []
    for name in ("k", "v"):
        x = c[name].view(torch.float8_e4m3fn) if c["k_exp"] is not None else c[name]
        x = x.to(torch.float64).view(c["pages"], c["heads"], T // 64, -1)
        for a, b, groups in pairs:
            x[b, :, :groups] = x[a, :, :groups]
        out.append(x.view(c[name].shape))
    return [None] * (6 if case["kind"] == "fork" else 5) + out + [None] * (2 if c["k_exp"] is not None else 0)


def _exact_kv4(case, seed):
    s = prepare(case, seed)
    H, D, n = s["cache"]["heads"], s["cache"]["size"], s["n"]
    got = []
    for x, heads, turned, stored in ((s["q"], s["q_heads"], True, False), (s["k"], H, True, True), (s["v"], H, False, True)):
        x = x.double().reshape(n, heads, D)
        if turned and s["axes"]:
            axis = torch.repeat_interleave(torch.arange(len(s["sections"])), torch.tensor(s["sections"])).cuda()
            turn = s["positions"].double()[axis] * s["inv_freq"].double()[:, None]        # [D / 2, n]
            z = torch.complex(x[..., :D // 2].contiguous(), x[..., D // 2:].contiguous())
            z = z * torch.polar(torch.ones_like(turn), turn).t()[:, None]
            x = torch.cat([z.real, z.imag], dim=-1)
        if stored:
            # two significant bits, steps of 1 / 2 below 1; the scale is the least power of two that fits 6
            y = x.reshape(n, heads, D // 32, 32)
            unit = torch.exp2(torch.ceil(torch.log2(y.abs().amax(dim=-1, keepdim=True) / 6)))
            y = y / unit
            step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=1.0))) - 1)
            x = (torch.round(y / step) * step * unit).reshape(n, heads, D)
        got.append(x)
    return got


def _exact_attn4(case, seed):
    s = prepare(case, seed)
    c, Hq = s["cache"], s["q_heads"]
    H, D, T = c["heads"], c["size"], c["page"]
    G = Hq // H
    t, d = torch.arange(T, device="cuda")[:, None], torch.arange(D, device="cuda")[None]
    # the byte of an element, and the byte of its scale, in a head's block of a page
    k_at = (t // 16 * (D // 32) + d // 32) * 256 + t % 16 * 16 + d % 32 // 2
    v_at = ((t // 64 * (D // 32) + d // 32) * 4 + t % 16 // 4) * 256 + d % 16 * 16 + t % 64 // 16 * 4 + t % 4
    ke_at = (t // 64 * (D // 32) + d // 32) * 64 + t % 16 * 4 + t % 64 // 16
    ve_at = (t // 64 * (D // 32) + d // 32) * 64 + t % 16 // 4 * 16 + t % 64 // 16 * 4 + t % 4
    k_shift, v_shift = (d % 2 * 4).expand(T, D), (d % 32 // 16 * 4).expand(T, D)
    offsets, lens = s["offsets"].tolist(), s["lens"].tolist()
    out = torch.empty((s["total"], Hq, D), dtype=torch.float64, device="cuda")

    def dense(data, exps, pages, h, at, e_at, shift, L):
        code = (data[pages, h][:, at.flatten()].view(-1, T, D).int() >> shift & 15).view(-1, D)[:L]
        exponent, fraction = code >> 1 & 3, code & 1
        x = torch.where(exponent == 0, fraction * 0.5, (1 + fraction * 0.5) * torch.exp2(exponent.double() - 1))
        e = exps[pages, h][:, e_at.flatten()].view(-1, D)[:L].double() - 127
        return torch.where(code >= 8, -x, x) * torch.exp2(e)

    for b in range(s["seqs"]):
        n, L = offsets[b + 1] - offsets[b], lens[b]
        pages = s["table"][b, :-(-L // T)].long()
        i, j = torch.arange(n, device="cuda")[:, None], torch.arange(L, device="cuda")[None] - (L - n)
        if s["mask"] is None:
            seen = j <= i
        else:
            word = s["mask"][offsets[b]:offsets[b + 1]].long()
            at = j.clamp(min=0).expand(n, L)
            seen = (j < 0) | (word.gather(1, at // 32) >> (at % 32) & 1).bool()
        for h in range(H):
            k = dense(c["k"], c["k_exp"], pages, h, k_at, ke_at, k_shift, L)
            v = dense(c["v"], c["v_exp"], pages, h, v_at, ve_at, v_shift, L)
            for g in range(G):
                q = s["q"][offsets[b]:offsets[b + 1], h * G + g].double()
                z = (q @ k.t().contiguous() * s["scale"]).masked_fill(~seen, float("-inf"))
                out[offsets[b]:offsets[b + 1], h * G + g] = torch.softmax(z, dim=1) @ v
    return out
