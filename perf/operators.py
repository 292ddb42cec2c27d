"""The operators of a serving step with drafted tokens, as cases to measure.

Around the projections of a layer, a step that checks a tree (or a chain) of
drafted tokens against a paged key/value cache does four things:

  kv      the rows that a QKV projection left: rotary positions on queries and
          keys (one axis, or time, height and width), keys and values written
          into the pages (8 bits with a power-of-two scale per token and head,
          or bf16), and the written entries read back
  attn    attention of the new tokens of every sequence over its pages: single
          tokens, chains, trees of drafted tokens and whole prompts
  verify  the drafted tokens checked against the target's probabilities, from
          given random numbers: the accepted path and the token after it
  keep    the accepted path's cache entries moved to where the sequence goes on

`own` chooses between the plain form in torch operations and the library's
calls.  The cache tensors have the library's page layout in both.
"""
import math

import torch

own = False

# (query heads, key/value heads, head size): a Llama-3.1-70B-shaped layer, one GPU's share of it under 8-way
# tensor parallelism, a Qwen-3-30B-A3B-shaped layer, and a layer of hidden size 768
HEADS = {"dense": (64, 8, 128), "dense_tp8": (8, 1, 128), "experts": (32, 4, 128), "small": (12, 12, 64)}
VOCAB = (50257, 131072)
FP8_MAX = 448.0


def listed():
    return [
        # one token of one sequence enters the cache: launches and latency are everything
        kv("kv_one_token", heads="experts", n=1, src="bf16", cache="fp8", axes=1, page=64),
        # a step of 16 sequences with 32 drafted tokens each, from a projection that writes fp32
        kv("kv_tree_batch", heads="dense", n=512, src="f32", cache="fp8", axes=1, page=64),
        # a long prompt of text and images: positions along time, height and width
        kv("kv_prompt_images", heads="dense", n=8192, src="bf16", cache="fp8", axes=3, page=128),
        # one token of one short sequence, 16-bit cache, every query head with its own key head
        attn("attn_one_token", heads="small", form="causal", seqs=1, new=1, length=517, cache="bf16", page=64),
        # the ordinary decode step of a batch of sequences of different lengths
        attn("attn_decode_batch", heads="dense", form="causal", seqs=32, new=1, length=8192, cache="fp8", page=64),
        # few very long sequences on one GPU of eight, a chain of five drafted tokens each
        attn("attn_long_chain", heads="dense_tp8", form="causal", seqs=3, new=5, length=131072, cache="fp8", page=128),
        # trees of up to 64 drafted tokens over a batch of sequences
        attn("attn_tree_batch", heads="dense", form="tree", seqs=16, new=64, length=8192, cache="fp8", page=64),
        # prompts, each partly in the cache already, 16-bit cache
        attn("attn_prompt", heads="experts", form="causal", seqs=3, new=2048, length=4096, cache="bf16", page=128),
        # a chain of four tokens that a deterministic draft proposed, one sequence
        verify("verify_chain", seqs=1, nodes=5, siblings=1, vocab=50257, logits="f32", draft="none"),
        # a batch of sampled trees with the draft's own probabilities, up to three tokens tried per node
        verify("verify_tree_batch", seqs=32, nodes=24, siblings=3, vocab=131072, logits="bf16", draft="f32"),
        # the accepted tokens of one short chain stay
        keep("keep_one", heads="small", seqs=1, nodes=8, length=300, cache="bf16", page=64),
        # the accepted paths of a batch of 64-token trees stay
        keep("keep_batch", heads="dense", seqs=64, nodes=64, length=2048, cache="fp8", page=64),
    ]


def _named(name, case):
    return dict(case, name=name) if name else case


def kv(name, heads, n, src, cache, axes, page):
    return _named(name, {"kind": "kv", "heads": heads, "n": n, "src": src, "cache": cache, "axes": axes, "page": page})


def attn(name, heads, form, seqs, new, length, cache, page):
    return _named(name, {"kind": "attn", "heads": heads, "form": form, "seqs": seqs, "new": new, "length": length,
                         "cache": cache, "page": page})


def verify(name, seqs, nodes, siblings, vocab, logits, draft):
    return _named(name, {"kind": "verify", "seqs": seqs, "nodes": nodes, "siblings": siblings, "vocab": vocab,
                         "logits": logits, "draft": draft})


def keep(name, heads, seqs, nodes, length, cache, page):
    return _named(name, {"kind": "keep", "heads": heads, "seqs": seqs, "nodes": nodes, "length": length,
                         "cache": cache, "page": page})


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("kv", "attn", "attn", "attn", "verify", "verify", "keep"))
    heads, cache, page = rng.choice(tuple(HEADS)), rng.choice(("fp8", "fp8", "bf16")), rng.choice((64, 128, 256))
    Hq, Hk, D = HEADS[heads]
    if kind == "kv":
        return kv(None, heads, _log(rng, 1, 8192), rng.choice(("bf16", "f32")), cache, rng.choice((0, 1, 1, 3)), page)
    if kind == "attn":
        form = rng.choice(("one", "chain", "tree", "tree", "prompt"))
        while True:
            seqs, length = _log(rng, 1, 64), _log(rng, 1, 131072)
            new = {"one": 1, "chain": rng.randint(2, 8), "tree": rng.randint(3, 64), "prompt": _log(rng, 65, 2048)}[form]
            if new <= length and seqs * length * Hk * D <= 32 * 8192 * 8 * 128 and \
                    seqs * new * length * Hq * D <= 16 * 64 * 8192 * 64 * 128:
                return attn(None, heads, "tree" if form == "tree" else "causal", seqs, new, length, cache, page)
    if kind == "verify":
        while True:
            seqs, nodes = _log(rng, 1, 64), rng.randint(2, 64)
            vocab = rng.choice(VOCAB + (_log(rng, 1000, 131072),))
            if seqs * nodes * vocab <= 32 * 24 * 131072:
                return verify(None, seqs, nodes, rng.choice((1, 2, 3)), vocab, rng.choice(("bf16", "f32")),
                              rng.choice(("none", "bf16", "f32")))
    while True:
        seqs, nodes, length = _log(rng, 1, 64), rng.randint(2, 64), _log(rng, 64, 8192)
        if seqs * length * Hk * D <= 64 * 2048 * 8 * 128:
            return keep(None, heads, seqs, nodes, length, cache, page)


# ---------------------------------------------------------------------------
# Inputs, from the seed alone
# ---------------------------------------------------------------------------

def _gen(seed, i):
    return torch.Generator(device="cuda").manual_seed(seed * 1009 + i)


def _host_gen(seed, i):
    return torch.Generator().manual_seed(seed * 1009 + i)


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


def _sizes(case):
    """The sequences' lengths and their new tokens (or tree nodes), the same for every seed."""
    if case["kind"] == "verify":
        return None, _ragged(case["seqs"], case["nodes"], 1)
    new = _ragged(case["seqs"], case["new" if case["kind"] == "attn" else "nodes"], 1)
    lens = _ragged(case["seqs"], case["length"], 2)
    return (lens, torch.minimum(new, lens)) if case["kind"] == "attn" else (torch.maximum(lens, new), new)


def _shuffled(case, seed):
    """_sizes in another order for every seed."""
    lens, new = _sizes(case)
    order = torch.randperm(len(new), generator=_host_gen(seed, 10))
    return lens if lens is None else lens[order], new[order]


def _offsets(sizes):
    out = torch.zeros(len(sizes) + 1, dtype=torch.int64)
    out[1:] = sizes.cumsum(0)
    return out


def _dev(t):
    return t.to(torch.int32).cuda()


def _trees(seed, i, sizes, siblings):
    """A tree per sequence: the parent (an earlier node of the sequence, -1 at node 0) of every node, and its place among
    its parent's children, at most `siblings` of them; flat, on the host."""
    pick = torch.rand(int(sizes.sum()), generator=_host_gen(seed, i)).tolist()
    parent, place, at = [], [], 0
    for n in sizes.tolist():
        children, free = [0] * n, [0]
        for j in range(n):
            if j == 0:
                parent.append(-1)
                place.append(0)
                continue
            # the newest nodes are the likeliest parents: paths of some depth
            k = len(free) - 1 - int(pick[at + j] ** 2 * len(free))
            p = free[k]
            parent.append(p)
            place.append(children[p])
            children[p] += 1
            if children[p] == siblings:
                free.pop(k)
            free.append(j)
        at += n
    return torch.tensor(parent), torch.tensor(place)


def _tree_mask(parent, sizes, words):
    """Bits of the nodes that each node sees (its ancestors and itself): int32 [nodes, words], on the host."""
    bits, rows, at = parent.tolist(), [], 0
    for n in sizes.tolist():
        for j in range(n):
            p = bits[at + j]
            rows.append((rows[at + p] if p >= 0 else 0) | 1 << j)
        at += n
    out = [[(r >> 32 * w & 0xffffffff) for w in range(words)] for r in rows]
    out = torch.tensor(out, dtype=torch.int64)
    return torch.where(out >= 1 << 31, out - (1 << 32), out).to(torch.int32)


def _to_pages(x, chunk, value):
    """[pages, heads, tokens, head size] -> the cache's order of a page.  Keys: 16 tokens x one 16-byte chunk after another
    along the head; values: for every 16 of the head's elements, 16-byte chunks that hold one element of the tokens
    16 m + 4 g + i (i fastest)."""
    P, H, T, D = x.shape
    if not value:
        return x.view(P, H, T // 16, 16, D // chunk, chunk).permute(0, 1, 2, 4, 3, 5).contiguous().view(P, H, T * D)
    x = x.view(P, H, T // (4 * chunk), chunk // 4, 4, 4, D // 16, 16)
    return x.permute(0, 1, 2, 6, 4, 7, 3, 5).contiguous().view(P, H, T * D)


def _exponents(amax):
    """The smallest e with amax <= 448 * 2^e."""
    m, e = torch.frexp(amax)
    return torch.where(amax > 0, torch.where(m <= 0.875, e - 9, e - 8), 0).clamp(-126, 127)


def _cache(case, pages, seed):
    """A pool of pages that holds earlier tokens: keys, values and (8 bits) the exponents of their scales, biased by 127."""
    _, H, D = HEADS[case["heads"]]
    T, made = case["page"], {}
    for i, name in enumerate(("k", "v")):
        x = _normal((pages, H, T, D), seed, 100 + i, torch.bfloat16)
        if case["cache"] == "bf16":
            made[name], made[name + "_exp"] = _to_pages(x, 8, name == "v"), None
            continue
        e = _exponents(x.abs().amax(dim=-1).float())
        x = (x * torch.exp2(-e.float()).to(torch.bfloat16)[..., None]).to(torch.float8_e4m3fn).view(torch.uint8)
        made[name] = _to_pages(x, 16, name == "v")
        b = (e + 127).to(torch.uint8).view(pages, H, T // 64, 4, 4, 4)   # [m, g, i] of 64 tokens
        b = b.permute(0, 1, 2, 4, 3, 5) if name == "v" else b.permute(0, 1, 2, 4, 5, 3)
        made[name + "_exp"] = b.contiguous().view(pages, H, T)
    return dict(made, pages=pages, page=T, heads=H, size=D)


def _table(case, lens, seed):
    """Pages for every sequence, in random order over the pool: page table (int32 [sequences, most pages]) and their number."""
    need = -(-lens // case["page"])
    pool = torch.randperm(int(need.sum()), generator=_host_gen(seed, 50))
    table, at = torch.full((len(lens), int(need.max())), -1), 0
    for b, c in enumerate(need.tolist()):
        table[b, :c] = pool[at:at + c]
        at += c
    return table, at


def prepare(case, seed):
    if case["kind"] == "kv":
        return _prepare_kv(case, seed)
    if case["kind"] == "attn":
        return _prepare_attn(case, seed)
    if case["kind"] == "verify":
        return _prepare_verify(case, seed)
    return _prepare_keep(case, seed)


def _prepare_kv(case, seed):
    Hq, Hk, D = HEADS[case["heads"]]
    n, page, dt = case["n"], case["page"], _dtype(case["src"])
    qkv = _normal((n, (Hq + 2 * Hk) * D), seed, 1, dt)
    qkv[:, Hq * D:(Hq + Hk) * D:37] *= 8   # some key channels are much larger than the rest
    pages = -(-n // page) + 3
    # consecutive tokens in consecutive places of pages in random order, the first one inside a page
    slots, room = [], torch.randperm(pages, generator=_host_gen(seed, 2)).tolist()
    for p in room:
        slots += range(p * page, p * page + page)
    skip = int(torch.randint(0, 2 * page, (1,), generator=_host_gen(seed, 3)))
    slots = torch.tensor(slots[skip:skip + n])
    s = {"kind": "kv", "q": qkv[:, :Hq * D], "k": qkv[:, Hq * D:(Hq + Hk) * D], "v": qkv[:, (Hq + Hk) * D:], "n": n,
         "q_heads": Hq, "slots": _dev(slots), "cache": _cache(case, pages, seed), "axes": case["axes"],
         "q_out": torch.empty((n, Hq, D), dtype=torch.bfloat16, device="cuda"),
         "k_out": torch.empty((n, Hk, D), dtype=torch.bfloat16, device="cuda"),
         "v_out": torch.empty((n, Hk, D), dtype=torch.bfloat16, device="cuda")}
    if case["axes"]:
        first = int(torch.randint(0, 4096, (1,), generator=_host_gen(seed, 4)))
        time = first + torch.arange(n)
        if case["axes"] == 3:   # images of 24 x 32 patches: one time, rows and columns
            pos = torch.stack([first + torch.arange(n) // 768, first + torch.arange(n) // 32 % 24,
                               first + torch.arange(n) % 32])
            s["sections"] = (D // 8, 3 * D // 16, 3 * D // 16)
        else:
            pos, s["sections"] = time[None], (D // 2,)
        s["positions"] = _dev(pos)
        s["inv_freq"] = (500000.0 ** (-torch.arange(0, D, 2, dtype=torch.float64) / D)).float().cuda()
    return s


def _prepare_attn(case, seed):
    Hq, Hk, D = HEADS[case["heads"]]
    lens, new = _shuffled(case, seed)
    table, pages = _table(case, lens, seed)
    total = int(new.sum())
    s = {"kind": "attn", "cache": _cache(case, pages, seed), "table": _dev(table), "lens": _dev(lens),
         "offsets": _dev(_offsets(new)), "total": total, "max_q": int(new.max()), "max_len": int(lens.max()),
         "q_heads": Hq, "scale": D ** -0.5, "mask": None, "seqs": case["seqs"],
         "q": (_normal((total, Hq, D), seed, 12) * 2).to(torch.bfloat16),
         "out": torch.empty((total, Hq, D), dtype=torch.bfloat16, device="cuda")}
    if case["form"] == "tree":
        parent, _ = _trees(seed, 13, new, 4)
        s["mask"] = _tree_mask(parent, new, -(-case["new"] // 32)).cuda()
    return s


def _prepare_verify(case, seed):
    V = case["vocab"]
    _, sizes = _shuffled(case, seed)
    parent, place = _trees(seed, 21, sizes, case["siblings"])
    offsets = _offsets(sizes)
    total, B = int(offsets[-1]), case["seqs"]
    up = torch.where(parent < 0, torch.arange(total), parent + offsets[:-1].repeat_interleave(sizes)).cuda()
    logits = _normal((total, V), seed, 22, torch.float32) * 3
    guess = logits + 0.7 * _normal((total, V), seed, 23, torch.float32)   # the draft's own view of the next token
    logits, draft = logits.to(_dtype(case["logits"])), None
    if case["draft"] == "none":
        best = guess.topk(case["siblings"], dim=1).indices
        tokens = best[up, place.cuda()]
    else:
        draft = torch.softmax(guess, dim=1)
        drawn = torch.multinomial(draft, case["siblings"], replacement=True, generator=_gen(seed, 24))
        tokens, draft = drawn[up, place.cuda()], draft.to(_dtype(case["draft"]))
    temperature = 0.6 + 0.6 * torch.rand(B, generator=_host_gen(seed, 25))
    temperature[torch.rand(B, generator=_host_gen(seed, 26)) < 0.1] = 0.0   # some users decode greedily
    noise = torch.empty((B, V), device="cuda").exponential_(generator=_gen(seed, 27)).clamp_(min=1e-20)
    return {"kind": "verify", "logits": logits, "draft": draft, "offsets": _dev(offsets), "parents": _dev(parent),
            "tokens": tokens.to(torch.int32), "temperature": temperature.cuda(),
            "uniform": torch.rand(total, generator=_gen(seed, 28), device="cuda"), "noise": noise, "seqs": B,
            "total": total, "vocab": V, "max_nodes": int(sizes.max()), "siblings": case["siblings"],
            "path": torch.empty((B, int(sizes.max())), dtype=torch.int32, device="cuda"),
            "count": torch.empty(B, dtype=torch.int32, device="cuda"),
            "next": torch.empty(B, dtype=torch.int32, device="cuda")}


def _prepare_keep(case, seed):
    lens, sizes = _shuffled(case, seed)
    table, pages = _table(case, lens, seed)
    parent, _ = _trees(seed, 32, sizes, 4)
    offsets, most = _offsets(sizes).tolist(), int(sizes.max())
    path, count = torch.full((case["seqs"], most), -1), []
    ends = torch.rand(case["seqs"], generator=_host_gen(seed, 33))
    for b, n in enumerate(sizes.tolist()):
        j, way = int(ends[b] * n), []
        while j >= 0:
            way.append(j)
            j = int(parent[offsets[b] + j])
        path[b, :len(way)] = torch.tensor(way[::-1])
        count.append(len(way))
    return {"kind": "keep", "cache": _cache(case, pages, seed), "table": _dev(table), "starts": _dev(lens - sizes),
            "path": _dev(path), "count": _dev(torch.tensor(count)), "seqs": case["seqs"], "most": most}


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------

def run(s):
    if own:
        return _own(s)
    if s["kind"] == "kv":
        return _plain_kv(s)
    if s["kind"] == "attn":
        return _plain_attn(s)
    if s["kind"] == "verify":
        return _plain_verify(s)
    return _plain_keep(s)


def _handle(s):
    """The library's handle of the cache's tensors, which a program keeps as long as the cache."""
    import paper_2607_04031_amd as tl
    c = s["cache"]
    if "handle" not in c:
        c["handle"] = tl.KVCache(c["k"], c["v"], c["k_exp"], c["v_exp"], c["page"], c["heads"], c["size"])
    return c["handle"]


def _own(s):
    import paper_2607_04031_amd as tl
    if s["kind"] == "kv":
        rope = tl.rope(s["positions"], s["inv_freq"], s["sections"]) if s["axes"] else None
        tl.kv_append(s["q"], s["k"], s["v"], _handle(s), s["slots"], rope, q_out=s["q_out"])
        tl.kv_read(_handle(s), s["slots"], s["k_out"], s["v_out"])
        return [s["q_out"], s["k_out"], s["v_out"]]
    if s["kind"] == "attn":
        return tl.attention(s["q"], _handle(s), s["table"], s["lens"], s["offsets"], s["max_q"], s["max_len"],
                            s["scale"], mask=s["mask"], out=s["out"])
    if s["kind"] == "verify":
        tl.verify(s["logits"], s["offsets"], s["parents"], s["tokens"], s["temperature"], s["uniform"], s["noise"],
                  s["max_nodes"], draft=s["draft"], out=(s["path"], s["count"], s["next"]))
        return [s["path"], s["count"], s["next"]]
    tl.kv_keep(_handle(s), s["table"], s["starts"], s["path"], s["count"])
    return _cache_values(s["cache"])


def _cache_values(c):
    if c["k_exp"] is None:
        return [c["k"], c["v"]]
    return [c["k"].view(torch.float8_e4m3fn), c["v"].view(torch.float8_e4m3fn), c["k_exp"], c["v_exp"]]


def _rotate(x, s):
    """Elements d and d + D / 2 of every head turned by position * inv_freq[d], the position of d's axis."""
    D, at, angle = x.shape[-1], 0, []
    for axis, width in enumerate(s["sections"]):
        angle.append(s["positions"][axis].float()[:, None] * s["inv_freq"][at:at + width])
        at += width
    angle = torch.cat(angle, dim=1)[:, None]
    cos, sin = torch.cos(angle), torch.sin(angle)
    a, b = x[..., :D // 2], x[..., D // 2:]
    return torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)


def _key_index(c, slots):
    """Where keys of the given places lie: page, block of 16 tokens, token of the block."""
    return slots // c["page"], slots % c["page"] // 16, slots % 16


def _value_index(c, slots, chunk):
    t = slots % c["page"]
    return slots // c["page"], t // (4 * chunk), t % 16 // 4, t % (4 * chunk) // 16 * 4 + t % 4


def _views(c):
    """Keys [page, head, 16-token block, chunk, token, element], values [page, head, group, 16 elements, g, element, token]."""
    chunk = 16 // c["k"].element_size()
    T, H, D, P = c["page"], c["heads"], c["size"], c["pages"]
    return chunk, c["k"].view(P, H, T // 16, D // chunk, 16, chunk), c["v"].view(P, H, T // (4 * chunk), D // 16, 4, 16, chunk)


def _plain_kv(s):
    c, n = s["cache"], s["n"]
    H, D = c["heads"], c["size"]
    q, k, v = s["q"].float().view(n, s["q_heads"], D), s["k"].float().view(n, H, D), s["v"].float().view(n, H, D)
    if s["axes"]:
        q, k = _rotate(q, s), _rotate(k, s)
    slots = s["slots"].long()
    chunk, keys, values = _views(c)
    kp, kb, kt = _key_index(c, slots)
    vp, vg, vs, vt = _value_index(c, slots, chunk)
    if c["k_exp"] is None:
        keys[kp, :, kb, :, kt] = k.to(torch.bfloat16).view(n, H, D // chunk, chunk)
        values[vp, :, vg, :, vs, :, vt] = v.to(torch.bfloat16).view(n, H, D // 16, 16)
        k_back = keys[kp, :, kb, :, kt].view(n, H, D)
        v_back = values[vp, :, vg, :, vs, :, vt].reshape(n, H, D)
        return [q.to(torch.bfloat16), k_back, v_back]
    ke, ve = _exponents(k.abs().amax(dim=-1)), _exponents(v.abs().amax(dim=-1))
    k8 = (k * torch.exp2(-ke.float())[..., None]).to(torch.float8_e4m3fn).view(torch.uint8)
    v8 = (v * torch.exp2(-ve.float())[..., None]).to(torch.float8_e4m3fn).view(torch.uint8)
    keys[kp, :, kb, :, kt] = k8.view(n, H, D // chunk, chunk)
    values[vp, :, vg, :, vs, :, vt] = v8.view(n, H, D // 16, 16)
    T = c["page"]
    k_exp, v_exp = c["k_exp"].view(-1, H, T // 64, 16, 4), c["v_exp"].view(-1, H, T // 64, 4, 16)
    t = slots % T
    k_exp[kp, :, t // 64, t % 16, t % 64 // 16] = (ke + 127).to(torch.uint8)
    v_exp[vp, :, vg, vs, vt] = (ve + 127).to(torch.uint8)
    k8 = keys[kp, :, kb, :, kt].reshape(n, H, D).view(torch.float8_e4m3fn).float()
    v8 = values[vp, :, vg, :, vs, :, vt].reshape(n, H, D).view(torch.float8_e4m3fn).float()
    k2 = torch.exp2(k_exp[kp, :, t // 64, t % 16, t % 64 // 16].float() - 127)
    v2 = torch.exp2(v_exp[vp, :, vg, vs, vt].float() - 127)
    return [q.to(torch.bfloat16), (k8 * k2[..., None]).to(torch.bfloat16), (v8 * v2[..., None]).to(torch.bfloat16)]


def _gathered(c, table):
    """The pages of every sequence as float32 [sequences, heads, tokens, head size]: keys and values."""
    chunk, keys, values = _views(c)
    B, pages = table.shape
    T, H, D = c["page"], c["heads"], c["size"]
    at = table.long().clamp(min=0)
    k = keys[at].permute(0, 2, 1, 3, 5, 4, 6).reshape(B, H, pages * T, D)
    v = values[at].view(B, pages, H, T // (4 * chunk), D // 16, 4, 16, chunk // 4, 4)
    v = v.permute(0, 2, 1, 3, 7, 5, 8, 4, 6).reshape(B, H, pages * T, D)
    if c["k_exp"] is None:
        return k.float(), v.float()
    ke = c["k_exp"].view(-1, H, T // 64, 16, 4)[at].permute(0, 2, 1, 3, 5, 4).reshape(B, H, pages * T)
    ve = c["v_exp"].view(-1, H, T // 64, 4, 4, 4)[at].permute(0, 2, 1, 3, 5, 4, 6).reshape(B, H, pages * T)
    return (k.view(torch.float8_e4m3fn).float() * torch.exp2(ke.float() - 127)[..., None],
            v.view(torch.float8_e4m3fn).float() * torch.exp2(ve.float() - 127)[..., None])


def _row_places(offsets, total):
    """The sequence of each row, and its place in it."""
    rows = torch.arange(total, device=offsets.device)
    seq = (rows[:, None] >= offsets[None, 1:]).sum(dim=1)
    return seq, rows - offsets[seq]


def _plain_attn(s):
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


def _plain_verify(s):
    B, V, total, most = s["seqs"], s["vocab"], s["total"], s["max_nodes"]
    offsets, parents, tokens = s["offsets"].long(), s["parents"].long(), s["tokens"].long()
    seq, place = _row_places(offsets, total)
    rows = torch.arange(total, device="cuda")
    up = torch.where(parents < 0, -1, parents + offsets[seq])
    # the target's probabilities; temperature 0: all on the largest logit (the first of equal ones)
    z = s["logits"].float()
    t = s["temperature"][seq][:, None]
    top = z.amax(dim=1, keepdim=True)
    p = torch.exp((z - top) / torch.where(t > 0, t, 1.0))
    p = p / p.sum(dim=1, keepdim=True)
    ids = torch.arange(V, device="cuda")
    first = torch.where(z == top, ids, V).amin(dim=1, keepdim=True)
    p = torch.where(t > 0, p, (ids == first).float())
    # a node's rank among its parent's children, and every node's child of each rank
    same = (up[:, None] == up[None]) & (up[:, None] >= 0)
    rank = (same & (rows[None] < rows[:, None])).sum(dim=1)
    rest, mass = p.clone(), torch.ones(total, device="cuda")
    chosen = torch.zeros(total, dtype=torch.bool, device="cuda")
    open_ = torch.ones(total, dtype=torch.bool, device="cuda")             # no child accepted yet
    for r in range(s["siblings"]):
        child = ((up[None] == rows[:, None]) & (rank[None] == r))          # [node, its r-th child]
        has, c = child.any(dim=1), child.int().argmax(dim=1)
        x = tokens[c]
        left = rest[rows, x]
        q = 1.0 if s["draft"] is None else s["draft"][rows, x].float()
        ok = has & open_ & (s["uniform"][c] * q * mass < left)
        chosen = chosen | (child & ok[:, None]).any(dim=0)
        open_ = open_ & ~ok
        if s["draft"] is None:
            rest[rows, x] = torch.where(has, 0.0, left)
            mass = torch.where(has, mass - left, mass)
        else:
            less = (rest / mass.clamp(min=1e-30)[:, None] - s["draft"].float()).clamp_(min=0)
            rest = torch.where(has[:, None], less, rest)
            mass = torch.where(has, rest.sum(dim=1), mass)
    on = up < 0
    for _ in range(most):
        on = on | (chosen & (up >= 0) & on[up.clamp(min=0)])
    count = torch.zeros(B, dtype=torch.int64, device="cuda").index_add_(0, seq, on.long())
    depth = torch.cumsum(on.long(), dim=0) - 1
    depth = depth - depth[offsets[:-1]][seq]
    path = torch.full((B, most + 1), -1, dtype=torch.int64, device="cuda")
    path[seq, torch.where(on, depth, most)] = torch.where(on, place, -1)
    last = offsets[:-1] + path[torch.arange(B, device="cuda"), count - 1]
    weight = torch.where((mass[last] > 0)[:, None], rest[last], p[last]) / s["noise"]
    best = weight.amax(dim=1, keepdim=True)
    token = torch.where(weight == best, ids, V).amin(dim=1)
    return [path[:, :most].int(), count.int(), token.int()]


def _plain_keep(s):
    c = s["cache"]
    place = torch.arange(s["most"], device="cuda")[None].expand(s["seqs"], -1)
    valid = place < s["count"].long()[:, None]
    start, table = s["starts"].long()[:, None], s["table"].long()
    slot = lambda t: table.gather(1, (t // c["page"]).clamp(max=table.shape[1] - 1)) * c["page"] + t % c["page"]  # noqa: E731
    src, dst = slot(start + s["path"].long().clamp(min=0))[valid], slot(start + place)[valid]
    chunk, keys, values = _views(c)
    (p0, b0, t0), (p1, b1, t1) = _key_index(c, src), _key_index(c, dst)
    keys[p1, :, b1, :, t1] = keys[p0, :, b0, :, t0]
    (p0, g0, s0, t0), (p1, g1, s1, t1) = _value_index(c, src, chunk), _value_index(c, dst, chunk)
    values[p1, :, g1, :, s1, :, t1] = values[p0, :, g0, :, s0, :, t0]
    if c["k_exp"] is not None:
        H, T = c["heads"], c["page"]
        v_exp = c["v_exp"].view(-1, H, T // 64, 4, 16)
        v_exp[p1, :, g1, s1, t1] = v_exp[p0, :, g0, s0, t0]
        k_exp, a, b = c["k_exp"].view(-1, H, T // 64, 16, 4), src % T, dst % T
        k_exp[p1, :, b // 64, b % 16, b % 64 // 16] = k_exp[p0, :, a // 64, a % 16, a % 64 // 16]
    return _cache_values(c)


# ---------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------

def _entry_bytes(case):
    """Keys and values of one token and key head."""
    D = HEADS[case["heads"]][2]
    return 2 * (D + 1) if case["cache"] == "fp8" else 4 * D


def work(case):
    if case["kind"] == "kv":
        Hq, H, D = HEADS[case["heads"]]
        n, src = case["n"], 4 if case["src"] == "f32" else 2
        # the projection's rows, the rotated queries, the cache entries written, and them read back to bf16
        return {"bytes": n * ((Hq + 2 * H) * D * src + Hq * D * 2 + 2 * H * _entry_bytes(case) + 2 * H * D * 2 + 4 * case["axes"] + 4),
                "flops": n * (Hq + H) * D * 3 if case["axes"] else n * H * D}
    lens, new = _sizes(case)
    rows = int(new.sum())
    if case["kind"] == "verify":
        z, q = 2 if case["logits"] == "bf16" else 4, {"none": 0, "bf16": 2, "f32": 4}[case["draft"]]
        # every node's logits, the random numbers, and the draft's row where a path ends
        return {"bytes": rows * (z * case["vocab"] + 12) + case["seqs"] * (case["vocab"] * (q + 4) + 4 * case["nodes"] + 16),
                "flops": 4 * rows * case["vocab"]}
    Hq, H, D = HEADS[case["heads"]]
    if case["kind"] == "attn":
        if case["form"] == "causal":
            seen = int((new * (lens - new) + new * (new + 1) // 2).sum())
        else:   # the tokens before the tree; of the tree, a few ancestors each
            seen = int((new * (lens - new)).sum()) + rows
        return {"bytes": int(lens.sum()) * H * _entry_bytes(case) + 4 * rows * Hq * D, "flops": 4 * seen * Hq * D}
    # one read and one write of the entries of a path (about eight nodes of a tree of 64)
    moved = float(new.double().sqrt().sum())
    return {"bytes": 2 * moved * H * _entry_bytes(case) + 4 * moved, "flops": 0}


# ---------------------------------------------------------------------------
# The definitions in 64 bits
# ---------------------------------------------------------------------------

def exact(case, seed):
    return {"kv": _exact_kv, "attn": _exact_attn, "verify": _exact_none, "keep": _exact_keep}[case["kind"]](case, seed)


def _exact_none(case, seed):
    return None   # whole numbers only


def _exact_kv(case, seed):
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
        if stored and case["cache"] == "fp8":
            # E4M3: 4 significant bits, steps of 2^-9 below 2^-6; the scale is the least power of two that fits 448
            e = torch.ceil(torch.log2(x.abs().amax(dim=-1, keepdim=True) / FP8_MAX))
            y = x / torch.exp2(e)
            step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
            x = torch.round(y / step) * step * torch.exp2(e)
        got.append(x)
    return got


def _exact_attn(case, seed):
    s = prepare(case, seed)
    c, Hq = s["cache"], s["q_heads"]
    H, D, T = c["heads"], c["size"], c["page"]
    G, chunk = Hq // H, 16 // c["k"].element_size()
    t, d = torch.arange(T, device="cuda")[:, None], torch.arange(D, device="cuda")[None]
    k_at = (t // 16 * (D // chunk) + d // chunk) * 16 * chunk + t % 16 * chunk + d % chunk
    v_at = t // (4 * chunk) * (4 * chunk * D) + d // 16 * (64 * chunk) + t % 16 // 4 * (16 * chunk) + d % 16 * chunk + \
        t % (4 * chunk) // 16 * 4 + t % 4
    t = t[:, 0]
    ke_at, ve_at = t // 64 * 64 + t % 16 * 4 + t % 64 // 16, t // 64 * 64 + t % 16 // 4 * 16 + t % 64 // 16 * 4 + t % 4
    offsets, lens = s["offsets"].tolist(), s["lens"].tolist()
    out = torch.empty((s["total"], Hq, D), dtype=torch.float64, device="cuda")

    def dense(data, exps, pages, h, at, e_at, L):
        x = data[pages, h][:, at.flatten()].view(-1, D)[:L]
        if exps is None:
            return x.double()
        return x.view(torch.float8_e4m3fn).double() * torch.exp2(exps[pages, h][:, e_at].flatten()[:L].double() - 127)[:, None]

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
            k = dense(c["k"], c["k_exp"], pages, h, k_at, ke_at, L)
            v = dense(c["v"], c["v_exp"], pages, h, v_at, ve_at, L)
            for g in range(G):
                q = s["q"][offsets[b]:offsets[b + 1], h * G + g].double()
                z = (q @ k.t().contiguous() * s["scale"]).masked_fill(~seen, float("-inf"))
                out[offsets[b]:offsets[b + 1], h * G + g] = torch.softmax(z, dim=1) @ v
    return out


def _exact_keep(case, seed):
    s = prepare(case, seed)
    c = s["cache"]
    T, D = c["page"], c["size"]
    chunk = 16 // c["k"].element_size()
    k, v = c["k"].clone(), c["v"].clone()
    d = torch.arange(D, device="cuda")
    key = lambda t: (t // 16 * (D // chunk) + d // chunk) * 16 * chunk + t % 16 * chunk + d % chunk  # noqa: E731
    value = lambda t: t // (4 * chunk) * (4 * chunk * D) + d // 16 * (64 * chunk) + t % 16 // 4 * (16 * chunk) + \
        d % 16 * chunk + t % (4 * chunk) // 16 * 4 + t % 4  # noqa: E731
    table, starts, path, count = s["table"].tolist(), s["starts"].tolist(), s["path"].tolist(), s["count"].tolist()
    for b in range(s["seqs"]):
        for i in range(count[b]):
            a, z = starts[b] + path[b][i], starts[b] + i
            if a != z:
                k[table[b][z // T]][:, key(z % T)] = c["k"][table[b][a // T]][:, key(a % T)]
                v[table[b][z // T]][:, value(z % T)] = c["v"][table[b][a // T]][:, value(a % T)]
    if c["k_exp"] is None:
        return [k.double(), v.double()]
    return [k.view(torch.float8_e4m3fn).double(), v.view(torch.float8_e4m3fn).double(), None, None]
