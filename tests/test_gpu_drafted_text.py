"""Generation with drafted tokens against generation without: the same text, with guesses that were kept, and a step whose
tree holds the text among wrong guesses keeps exactly that.  Where two runs may choose differently is as in
tests/test_gpu_drafted_decode.py: tokens whose logits are within a quarter of a row's standard deviation; entries of the
first layer differ by 0.05 in the norm at most."""
import pytest

from tests import test_gpu_drafted_decode as base
from tests._gpu import banner

pytestmark = pytest.mark.gpu
example = base.example
PROMPTS = [[5, 9, 2, 400, 9], [17], list(range(70))]


def _logits(example, model, text):
    import torch
    pages = example.Pages(1, len(text))
    z = example.prompt_pass(model, pages, [text])
    torch.cuda.synchronize()
    return z.double().cpu()


def test_same_text_with_guesses_that_are_kept(example, monkeypatch):
    import paper_2607_04031_amd as tl
    banner("generation with and without drafted tokens")
    model, verify, kept = example.Model(), tl.verify, []

    def watched(*args, **kw):
        out = verify(*args, **kw)
        kept.append(out[1].cpu())
        return out

    monkeypatch.setattr(tl, "verify", watched)
    runs = {}
    for wide in (False, True):
        texts, _, steps = example.generate(model, PROMPTS, 60, wide=wide)
        assert len(kept) == steps and max(int(x.max()) for x in kept) > 1      # a guess was kept, not only the token after it
        assert sum(int(x.sum()) for x in kept) == sum(len(t) - len(p) for t, p in zip(texts, PROMPTS))
        runs[wide] = texts
        kept.clear()
    monkeypatch.setattr(example, "guess", lambda seen, token, wide: ([token], [-1], [0]))
    plain, _, steps = example.generate(model, PROMPTS, 60)
    assert steps == 60 and all(len(t) - len(p) == 60 for t, p in zip(plain, PROMPTS)) and max(int(x.max()) for x in kept) == 1
    for wide, texts in runs.items():
        for p, a, b in zip(PROMPTS, plain, texts):
            same = next((i for i, (x, y) in enumerate(zip(a, b)) if x != y), None)
            if same is None:
                continue
            assert same >= len(p)
            z = _logits(example, model, a[:same])[-1]
            assert abs(z[a[same]] - z[b[same]]) < 0.25 * z.std(), (wide, same)


@pytest.mark.parametrize("before", [True, False])
def test_a_step_keeps_the_text_among_wrong_guesses(example, monkeypatch, before):
    """Two tokens of the text as a path, each beside three wrong guesses: before it (the entries kept lie apart and move) or
    after it."""
    import torch

    import paper_2607_04031_amd as tl
    banner(f"a step over a tree that holds the text, wrong guesses before={before}")
    model = example.Model()
    monkeypatch.setattr(example, "guess", lambda seen, token, wide: ([token], [-1], [0]))
    text = example.generate(model, PROMPTS, 60)[0][0]
    z = _logits(example, model, text)
    top = z.topk(2, dim=1).values
    clear = ((top[:, 0] - top[:, 1]) > 0.25 * z.std(dim=1)).tolist()
    depth = 2
    # the first place from which all of the path's rows choose clearly, and choose the text
    a = next(i for i in range(len(PROMPTS[0]), len(text) - depth - 1)
             if all(clear[i:i + depth + 1]) and z[i:i + depth + 1].argmax(1).tolist() == text[i + 1:i + depth + 2])
    tokens, parents, depths, at, want = [text[a]], [-1], [0], 0, [0]
    for k in range(1, depth + 1):
        right = text[a + k]
        wrong = [(right + i) % example.VOCAB for i in (1, 2, 3)]
        up = at
        for x in wrong + [right] if before else [right] + wrong:
            if x == right:
                at = len(tokens)
                want.append(at)
            tokens.append(x)
            parents.append(up)
            depths.append(k)
    n, ints = len(tokens), example.ints
    assert n <= example.MAX_NODES
    mask = []
    for i in range(n):
        mask.append((mask[parents[i]] if i else 0) | 1 << i)
    pages, fresh = example.Pages(1, len(text) + n), example.Pages(1, len(text))
    example.prompt_pass(model, pages, [text[:a]])
    example.prompt_pass(model, fresh, [text])
    slots = ints([pages.slot(0, a + i) for i in range(n)])
    logits = model(ints(tokens), ints([a + d for d in depths]), slots, pages.caches, pages.device, ints([a + n]), ints([0, n]), n, a + n,
                   ints(mask).view(-1, 1))
    path, counts, after = tl.verify(logits, ints([0, n]), ints(parents), ints(tokens), torch.zeros(1, device="cuda"),
                                    torch.full((n,), 0.5, device="cuda"), torch.ones((1, example.VOCAB), device="cuda"), n)
    assert counts.tolist() == [depth + 1] and path.tolist()[0][:depth + 1] == want
    assert after.tolist() == [text[a + depth + 1]]
    for cache in pages.caches:
        tl.kv_keep(cache, pages.device, ints([a]), path, counts)
    got, ref = (tl.kv_read(p.caches[0], ints([p.slot(0, a + i) for i in range(depth + 1)])) for p in (pages, fresh))
    for x, y in zip(got, ref):
        off = (x.float() - y.float()).flatten(1).norm(dim=1) / y.float().flatten(1).norm(dim=1)
        assert off.max().item() < 0.05, off
