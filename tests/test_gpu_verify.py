"""tl_verify against the walk as it is defined, in 64 bits, and against the
distribution that it must reproduce.

Decisions are whole numbers and must be equal.  The library's probabilities are
fp32, off by at most about 2^-19 of themselves here (logits of at most 30, an
exponent of at most 60 rounded to 2^-24 of that), so an input whose nearest
decision in 64 bits is closer than 2^-16 is not used: the cases' margins are
asserted, not assumed."""
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


def _dev(x, dtype):
    import torch
    return torch.from_numpy(np.ascontiguousarray(x)).to(dtype).cuda()


def _case(seed, sizes, V, siblings, draft, bf16, greedy=()):
    rng = np.random.default_rng(seed)
    total, B = sum(sizes), len(sizes)
    logits = rng.standard_normal((total, V)) * 3
    logits = _serve.bf16(logits) if bf16 else logits.astype(np.float32).astype(np.float64)
    guess = logits + 0.5 * rng.standard_normal((total, V))
    q = np.exp(guess - guess.max(1, keepdims=True))
    q /= q.sum(1, keepdims=True)
    q = _serve.bf16(q) if draft == "bf16" else q.astype(np.float32).astype(np.float64)
    parents, tokens, at = [], [], 0
    for n in sizes:
        children = {}
        for i in range(n):
            if i == 0:
                parents.append(-1)
                tokens.append(-1)
                continue
            p = int(rng.integers(max(0, i - 4), i))
            while children.get(p, 0) >= siblings:
                p = (p + 1) % i
            order = np.argsort(-guess[at + p])
            k = children.get(p, 0)
            children[p] = k + 1
            parents.append(p)
            tokens.append(int(order[k]) if draft is None else int(rng.choice(V, p=q[at + p] / q[at + p].sum())))
        at += n
    temperature = rng.uniform(0.5, 1.5, B).astype(np.float32)
    temperature[list(greedy)] = 0.0
    return dict(logits=logits, offsets=np.concatenate([[0], np.cumsum(sizes)]), parents=np.array(parents), tokens=np.array(tokens),
                temperature=temperature, uniform=rng.random(total).astype(np.float32),
                noise=np.maximum(rng.exponential(size=(B, V)), 1e-20).astype(np.float32), max_nodes=max(max(sizes), 1),
                draft=None if draft is None else q), bf16, draft


def _run(c, bf16, draft):
    import torch
    i32, f32 = torch.int32, torch.float32
    out = tl.verify(_dev(c["logits"], torch.bfloat16 if bf16 else f32), _dev(c["offsets"], i32), _dev(c["parents"], i32),
                    _dev(c["tokens"], i32), _dev(c["temperature"], f32), _dev(c["uniform"], f32), _dev(c["noise"], f32),
                    c["max_nodes"], draft=None if draft is None else _dev(c["draft"], torch.bfloat16 if draft == "bf16" else f32))
    torch.cuda.synchronize()
    return [x.cpu().numpy() for x in out]


def _check(c, bf16, draft):
    path, counts, nxt, margin = _serve.verify(**{k: (v.astype(np.float64) if k in ("temperature", "uniform", "noise") else v) for k, v in c.items()})
    assert margin > 2.0 ** -16, "the case has a decision too close to call"
    p, n, t = _run(c, bf16, draft)
    np.testing.assert_array_equal(n, counts)
    np.testing.assert_array_equal(p, path)
    np.testing.assert_array_equal(t, nxt)
    return counts


@pytest.mark.parametrize("V", [1, 2, 37, 4099, 50257])
@pytest.mark.parametrize("draft", [None, "f32", "bf16"])
@pytest.mark.parametrize("bf16", [False, True])
def test_chains(V, draft, bf16):
    banner(f"verify chains V={V} draft={draft} bf16={bf16}")
    counts = _check(*_case(V + 1, [1, 2, 6, 3], V, 1, draft, bf16, greedy=(2,)))
    assert (counts >= 1).all()


@pytest.mark.parametrize("siblings", [2, 3, 5])
@pytest.mark.parametrize("draft", [None, "f32", "bf16"])
@pytest.mark.parametrize("bf16", [False, True])
def test_trees(siblings, draft, bf16):
    banner(f"verify trees siblings={siblings} draft={draft} bf16={bf16}")
    _check(*_case(100 + siblings, [20, 1, 13, 33, 8, 64], 3001, siblings, draft, bf16, greedy=(3,)))


def test_sequences_without_nodes_and_many_sequences():
    banner("verify: empty sequences among 70")
    c = _case(7, [(i * 5) % 7 for i in range(70)], 501, 2, None, False)
    _check(*c)


def test_ties_masked_logits_and_tokens_outside():
    """Equal largest logits go to the lowest index; -infinity never wins; a
    child outside the vocabulary is not tried; a node bound below the tree."""
    banner("verify: ties, -inf, bad tokens")
    V = 1000
    c, bf16, draft = _case(9, [6, 4, 5], V, 2, None, False, greedy=(0, 1))
    c["logits"][:] = -np.inf
    c["logits"][:, 700:705] = 1.5
    c["tokens"][c["parents"] == 0] = [V, -7, 700][: 1] + [700] * (len(c["tokens"][c["parents"] == 0]) - 1)
    c["temperature"][2] = 1.0
    _check(c, bf16, draft)
    p, n, t = _run(c, bf16, draft)
    assert t[0] == 700 and t[1] == 700 and 700 <= t[2] < 705


def test_draft_that_is_the_target_accepts_everything():
    """q = p: every child is accepted whatever its random number."""
    banner("verify: the draft's distribution is the target's")
    rng = np.random.default_rng(3)
    V, n = 512, 9
    z = rng.standard_normal((n, V)).astype(np.float32).astype(np.float64)
    z[:] = z[0]
    q = np.exp(z - z.max(1, keepdims=True))
    q /= q.sum(1, keepdims=True)
    tokens = rng.choice(V, n, p=q[0])
    c = dict(logits=z, offsets=np.array([0, n]), parents=np.arange(n) - 1, tokens=tokens, temperature=np.ones(1, np.float32),
             uniform=np.full(n, 0.999, np.float32), noise=rng.exponential(size=(1, V)).astype(np.float32), max_nodes=n, draft=q)
    path, counts, _ = _run(c, False, "f32")
    assert counts[0] == n and (path[0] == np.arange(n)).all()


@pytest.mark.parametrize("draft", [None, "f32"])
def test_output_follows_the_target(draft):
    """The first token after the root (accepted or sampled) over many sequences
    follows p.  Counts of a token in N draws deviate by more than 5 standard
    deviations once in 10^6; 8 tokens are looked at."""
    banner(f"verify: distribution, draft={draft}")
    rng = np.random.default_rng(21)
    V, B, k = 8, 20000, 3
    z = rng.standard_normal(V) * 1.2
    q = np.exp(0.7 * z + 0.5 * rng.standard_normal(V))
    q /= q.sum()
    q = q.astype(np.float32).astype(np.float64)
    n = 1 + k
    tokens = rng.choice(V, (B, n), p=q / q.sum()) if draft else np.tile(np.concatenate([[0], np.argsort(-q)[:k]]), (B, 1))
    c = dict(logits=np.tile(z, (B * n, 1)), offsets=np.arange(B + 1) * n, parents=np.tile([-1] + [0] * k, B), tokens=tokens.ravel(),
             temperature=np.ones(B, np.float32), uniform=rng.random(B * n).astype(np.float32),
             noise=np.maximum(rng.exponential(size=(B, V)), 1e-20).astype(np.float32), max_nodes=n, draft=np.tile(q, (B * n, 1)))
    path, counts, nxt = _run(c, False, draft)
    first = np.where(counts > 1, tokens[np.arange(B), np.maximum(path[:, 1], 0)], nxt)
    p = np.exp(z) / np.exp(z).sum()
    got = np.bincount(first, minlength=V)
    assert (np.abs(got - B * p) <= 5 * np.sqrt(B * p * (1 - p))).all(), (got, B * p)


def test_repeats_and_graph():
    import torch
    banner("verify: the same results again, and from a replayed graph")
    c, bf16, draft = _case(31, [12, 7, 30], 9000, 3, "f32", True)
    first = _run(c, bf16, draft)
    for x, y in zip(first, _run(c, bf16, draft)):
        np.testing.assert_array_equal(x, y)
    i32, f32 = torch.int32, torch.float32
    args = [_dev(c["logits"], torch.bfloat16), _dev(c["offsets"], i32), _dev(c["parents"], i32), _dev(c["tokens"], i32),
            _dev(c["temperature"], f32), _dev(c["uniform"], f32), _dev(c["noise"], f32)]
    q = _dev(c["draft"], f32)
    out = (torch.empty((3, c["max_nodes"]), dtype=i32, device="cuda"), torch.empty(3, dtype=i32, device="cuda"), torch.empty(3, dtype=i32, device="cuda"))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        tl.verify(*args, c["max_nodes"], draft=q, out=out)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        tl.verify(*args, c["max_nodes"], draft=q, out=out)
    for step in range(3):
        c["uniform"] = np.random.default_rng(50 + step).random(len(c["uniform"])).astype(np.float32)
        args[5].copy_(_dev(c["uniform"], f32))
        for x in out:
            x.fill_(-9)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(out, _run(c, bf16, draft)):
            np.testing.assert_array_equal(x.cpu().numpy(), y)
