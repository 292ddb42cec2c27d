"""Generation with drafted tokens, all products and serving operators from libtl: a small decoder with random weights.

    python examples/drafted_decode.py [--temperature T] [--tokens N] [--wide]

Every step takes one tree of guesses per sequence through the model: tl_gemm makes queries, keys and values, tl_kv_append
turns and stores them (E4M3, paged), tl_attn lets each node see the sequence and its own ancestors, tl_verify keeps the
longest path that the model agrees with and samples the token after it, tl_kv_keep moves that path's entries to where the
sequence goes on.  Guesses come from what followed a token before.  At the end the sequences are taken through the model
once more as prompts: at temperature 0 every generated token must have (nearly) the largest logit there, and the first
layer's entries, read back with tl_kv_read, must agree."""
import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

HIDDEN, LAYERS, HEADS, KV_HEADS, HEAD_DIM, MLP, VOCAB = 512, 2, 8, 2, 64, 1024, 512
PAGE = 64
MAX_NODES = 12


class Model:
    """Tile-major bf16 weights, RMS norms without gains, gated MLP."""

    def __init__(self, seed=0):
        import torch

        import paper_2607_04031_amd as tl
        g = torch.Generator().manual_seed(seed)

        def weight(n, k):
            return tl.repack((torch.randn(n, k, generator=g) * k ** -0.5).to(torch.bfloat16).cuda())

        self.embed = torch.randn(VOCAB, HIDDEN, generator=g).to(torch.bfloat16).cuda()
        self.layers = [dict(qkv=weight((HEADS + 2 * KV_HEADS) * HEAD_DIM, HIDDEN), out=weight(HIDDEN, HEADS * HEAD_DIM),
                            up=weight(2 * MLP, HIDDEN), down=weight(HIDDEN, MLP)) for _ in range(LAYERS)]
        self.head = weight(VOCAB, HIDDEN)
        self.inv_freq = (10000.0 ** (-torch.arange(HEAD_DIM // 2) / (HEAD_DIM // 2))).float().cuda()
        self.bf16 = tl.layout(out_dtype=tl.TL_OUT_BF16)
        self.fp32 = tl.layout(out_dtype=tl.TL_OUT_F32)

    def __call__(self, tokens, positions, slots, caches, table, lens, offsets, max_q, max_len, mask=None):
        """fp32 logits of the rows, whose keys and values go to 'slots' of every layer's cache."""
        import torch

        import paper_2607_04031_amd as tl
        x = self.embed[tokens.long()].float()

        def normed(x):
            return torch.nn.functional.rms_norm(x, (HIDDEN,)).to(torch.bfloat16)

        q_cols, kv_cols = HEADS * HEAD_DIM, KV_HEADS * HEAD_DIM
        rope = tl.rope(positions, self.inv_freq)
        for w, cache in zip(self.layers, caches):
            qkv = tl.gemm(normed(x), w["qkv"], q_cols + 2 * kv_cols, self.bf16)
            q = tl.kv_append(qkv[:, :q_cols], qkv[:, q_cols:q_cols + kv_cols], qkv[:, q_cols + kv_cols:], cache, slots, rope)
            o = tl.attention(q, cache, table, lens, offsets, max_q, max_len, HEAD_DIM ** -0.5, mask=mask)
            x = x + tl.gemm(o.view(-1, q_cols), w["out"], HIDDEN, self.fp32)
            gate, up = tl.gemm(normed(x), w["up"], 2 * MLP, self.bf16).float().chunk(2, dim=1)
            x = x + tl.gemm((torch.nn.functional.silu(gate) * up).to(torch.bfloat16), w["down"], HIDDEN, self.fp32)
        return tl.gemm(normed(x), self.head, VOCAB, self.fp32)


def ints(x):
    import torch
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Pages:
    """Every sequence's share of the pool, one page after another in turn, so that a sequence's pages lie apart."""

    def __init__(self, sequences, tokens):
        import paper_2607_04031_amd as tl
        self.per = -(-tokens // PAGE)
        self.table = [[p * sequences + s for p in range(self.per)] for s in range(sequences)]
        self.device = ints(self.table)
        self.caches = [tl.kv_cache(sequences * self.per, KV_HEADS, HEAD_DIM, PAGE) for _ in range(LAYERS)]

    def slot(self, s, t):
        return self.table[s][t // PAGE] * PAGE + t % PAGE


def prompt_pass(model, pages, texts):
    """All tokens of all texts into the pages: their logits."""
    offsets = [0]
    for x in texts:
        offsets.append(offsets[-1] + len(x))
    at = [(s, t) for s, x in enumerate(texts) for t in range(len(x))]
    most = max(len(x) for x in texts)
    return model(ints([texts[s][t] for s, t in at]), ints([t for _, t in at]), ints([pages.slot(s, t) for s, t in at]),
                 pages.caches, pages.device, ints([len(x) for x in texts]), ints(offsets), most, most)


def guess(seen, token, wide):
    """A tree under 'token': (tokens, parents, depths), node 0 the token itself."""
    tokens, parents, depths = [token], [-1], [0]
    for i in range(MAX_NODES):
        if i == len(tokens):
            break
        for x in seen.get(tokens[i], [])[:2 if wide else 1]:
            if len(tokens) < MAX_NODES:
                tokens.append(x)
                parents.append(i)
                depths.append(depths[i] + 1)
    return tokens, parents, depths


def generate(model, prompts, count, temperature=0.0, wide=True, seed=0):
    """(texts, pages, steps): every prompt continued by at least 'count' tokens."""
    import torch

    import paper_2607_04031_amd as tl
    gen = torch.Generator(device="cuda").manual_seed(seed)
    B = len(prompts)
    texts = [list(p) for p in prompts]
    pages = Pages(B, max(len(p) for p in prompts) + count + 2 * MAX_NODES)
    prompt_pass(model, pages, [p[:-1] for p in prompts])
    followers = [{} for _ in prompts]       # what followed a token, the last first

    def learn(s, a, b):
        known = followers[s].setdefault(a, [])
        if b in known:
            known.remove(b)
        known.insert(0, b)

    for s, p in enumerate(prompts):
        for a, b in zip(p, p[1:]):
            learn(s, a, b)
    heat = torch.full((B,), temperature, device="cuda")
    steps = 0
    while min(len(t) - len(p) for t, p in zip(texts, prompts)) < count:
        trees = [guess(followers[s], texts[s][-1], wide) for s in range(B)]
        for s in range(B):                  # one that has its tokens goes on without guesses
            if len(texts[s]) - len(prompts[s]) >= count:
                trees[s] = ([], [], [])
        starts = [len(t) - 1 for t in texts]
        offsets = [0]
        for t in trees:
            offsets.append(offsets[-1] + len(t[0]))
        tokens = ints([x for t in trees for x in t[0]])
        parents = ints([x for t in trees for x in t[1]])
        masks = []
        for _, up, _ in trees:
            for i in range(len(up)):
                masks.append((masks[len(masks) - i + up[i]] if i else 0) | 1 << i)
        lens = [a + len(t[0]) for a, t in zip(starts, trees)]
        offs = ints(offsets)
        logits = model(tokens, ints([a + d for a, t in zip(starts, trees) for d in t[2]]),
                       ints([pages.slot(s, starts[s] + i) for s, t in enumerate(trees) for i in range(len(t[0]))]),
                       pages.caches, pages.device, ints(lens), offs, MAX_NODES, max(lens), ints(masks).view(-1, 1))
        path, counts, after = tl.verify(logits, offs, parents, tokens, heat,
                                        torch.rand(offsets[-1], generator=gen, device="cuda"),
                                        torch.empty(B, VOCAB, device="cuda").exponential_(generator=gen), MAX_NODES)
        for cache in pages.caches:
            tl.kv_keep(cache, pages.device, ints(starts), path, counts)
        path, counts, after = path.tolist(), counts.tolist(), after.tolist()
        for s in range(B):
            for x in [trees[s][0][i] for i in path[s][1:counts[s]]] + after[s:s + 1] * (counts[s] > 0):
                learn(s, texts[s][-1], x)
                texts[s].append(x)
        steps += 1
    return texts, pages, steps


def check(model, prompts, texts, pages):
    """(how far generated tokens are below the largest logit of a prompt pass, at most and in its standard deviations;
    relative difference of the first layer's entries)."""
    import torch

    import paper_2607_04031_amd as tl
    fresh = Pages(len(texts), max(len(t) for t in texts))
    logits = prompt_pass(model, fresh, texts)
    short, at = 0.0, 0
    for p, t in zip(prompts, texts):
        rows = logits[at + len(p) - 1:at + len(t) - 1]
        own = rows.gather(1, torch.tensor(t[len(p):], device="cuda").view(-1, 1)).squeeze(1)
        short = max(short, ((rows.max(dim=1).values - own) / rows.std(dim=1)).max().item())
        at += len(t)
    held = [(s, i) for s, t in enumerate(texts) for i in range(len(t) - 1)]      # the last token is in no cache yet
    a, b = (tl.kv_read(p.caches[0], ints([p.slot(s, i) for s, i in held])) for p in (pages, fresh))
    off = max(((x.float() - y.float()).norm() / y.float().norm()).item() for x, y in zip(a, b))
    return short, off


def main():
    import torch
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--temperature", type=float, default=0.0)
    ap.add_argument("--tokens", type=int, default=200)
    ap.add_argument("--wide", action="store_true", help="two guesses after each token, not one")
    args = ap.parse_args()
    model = Model()
    g = torch.Generator().manual_seed(1)
    prompts = [torch.randint(0, VOCAB, (n,), generator=g).tolist() for n in (5, 70, 33, 2)]
    texts, pages, steps = generate(model, prompts, args.tokens, args.temperature, args.wide)
    made = sum(len(t) - len(p) for t, p in zip(texts, prompts))
    short, off = check(model, prompts, texts, pages)
    print(f"{made} tokens for {len(prompts)} sequences in {steps} steps; first layer's entries off by {off:.1e}"
          + (f"; chosen tokens at most {short:.3f} standard deviations below the largest logit" if args.temperature == 0 else ""))
    assert off < 0.05 and (args.temperature > 0 or short < 0.25)


if __name__ == "__main__":
    main()
