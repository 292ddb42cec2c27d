"""The serving-step calls with every tensor in hand go through the extension module, others through the binding's own
checks: same results, same refusals."""
import numpy as np
import pytest

import paper_2607_04031_amd as tl
from tests._gpu import banner

pytestmark = pytest.mark.gpu
D, H, HQ, PAGE, N, V = 64, 2, 6, 64, 70, 999


@pytest.fixture(scope="module", autouse=True)
def _lib():
    import torch
    assert torch.cuda.is_available()
    yield
    torch.cuda.synchronize()


def _ints(x):
    import torch
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Step:
    """One sequence of N tokens, written, attended to, verified and moved."""

    def __init__(self, elem, mask):
        import torch
        g = torch.Generator(device="cuda").manual_seed(3)
        rand = lambda *shape: torch.randn(shape, generator=g, device="cuda")  # noqa: E731
        self.qkv = rand(N, (HQ + 2 * H) * D).to(torch.bfloat16)
        self.cache = tl.kv_cache(2, H, D, PAGE, elem)
        for x in (self.cache.k, self.cache.v):
            x.zero_()
        for x in (self.cache.k_exp, self.cache.v_exp):
            if x is not None:
                x.zero_()
        self.slots, self.table, self.lens, self.offsets = _ints(np.arange(N)), _ints([[0, 1]]), _ints([N]), _ints([0, N])
        self.rope = tl.rope(_ints(np.arange(N))[None].repeat(2, 1), 0.9 ** torch.arange(24, device="cuda").float(), (8, 16))
        self.mask = _ints(np.full((N, 3), 0x155)) if mask else None
        self.logits, self.draft = rand(4, V), torch.softmax(rand(4, V), 1)
        self.parents, self.tokens, self.nodes = _ints([-1, 0, 0, 1]), _ints([0, 5, 7, 9]), _ints([0, 4])
        self.heat, self.uniform = torch.ones(1, device="cuda"), torch.rand(4, generator=g, device="cuda")
        self.noise = torch.rand((1, V), generator=g, device="cuda") + 0.01
        bf16 = lambda *shape: torch.zeros(shape, dtype=torch.bfloat16, device="cuda")  # noqa: E731
        self.q, self.k, self.v, self.o = bf16(N, HQ, D), bf16(N, H, D), bf16(N, H, D), bf16(N, HQ, D)
        self.out = (_ints([[7] * 4]), _ints([7]), _ints([7]))

    def parts(self):
        a, b = HQ * D, (HQ + H) * D
        return self.qkv[:, :a], self.qkv[:, a:b], self.qkv[:, b:]

    def native(self):
        """The extension's own status of every call, in order."""
        calls, c = tl._load_calls(), self.cache.desc
        return [calls.kv_append(*self.parts(), c, self.slots, self.rope, self.q, None),
                calls.attention(self.q, c, self.table, self.lens, self.offsets, N, N, 0.125, self.mask, self.o, None),
                calls.verify(self.logits, self.nodes, self.parents, self.tokens, self.heat, self.uniform, self.noise, 4, self.draft, *self.out, None),
                calls.kv_keep(c, self.table, _ints([N - 4]), self.out[0], self.out[1], None),
                calls.kv_read(c, self.slots, self.k, self.v, None)]

    def binding(self, stream=None):
        tl.kv_append(*self.parts(), self.cache, self.slots, self.rope, self.q, stream)
        tl.attention(self.q, self.cache, self.table, self.lens, self.offsets, N, N, 0.125, self.mask, self.o, stream)
        tl.verify(self.logits, self.nodes, self.parents, self.tokens, self.heat, self.uniform, self.noise, 4, self.draft, self.out, stream)
        tl.kv_keep(self.cache, self.table, _ints([N - 4]), self.out[0], self.out[1], stream)
        tl.kv_read(self.cache, self.slots, self.k, self.v, stream)

    def made(self):
        return [x.cpu() for x in (self.q, self.o, *self.out, self.k, self.v)]


@pytest.mark.parametrize("mask", [False, True])
@pytest.mark.parametrize("elem", [1, 2])
def test_same_results_by_either_way(elem, mask):
    import torch
    banner(f"serving calls: extension and binding, {elem} bytes an element, mask {mask}")
    one, two, three = Step(elem, mask), Step(elem, mask), Step(elem, mask)
    assert one.native() == [tl.TL_OK] * 5
    two.binding()
    three.binding(torch.cuda.current_stream())          # a given stream: the binding's own way
    assert bool(one.o.any()) and int(one.out[1]) >= 1
    for x, y, z in zip(one.made(), two.made(), three.made()):
        assert torch.equal(x, y) and torch.equal(x, z)


def test_on_the_current_stream():
    import torch
    banner("serving calls on the current stream")
    want, s = Step(1, False), Step(1, False)
    want.binding()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        s.binding()
    side.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(want.made(), s.made()))


def test_not_plain_calls_are_refused_by_the_binding():
    """Everything that the extension hands back: the binding names it, or makes what is missing."""
    import torch
    banner("serving calls: refusals")
    s = Step(1, True)
    s.binding()
    calls, c = tl._load_calls(), s.cache.desc
    q, k, v = s.parts()
    bad = {
        "slots of another type": lambda f, c: f(q, k, v, c, s.slots.long(), None, s.q, None),
        "too few slots": lambda f, c: f(q, k, v, c, s.slots[1:], None, s.q, None),
        "slots with gaps": lambda f, c: f(q, k, v, c, _ints(np.arange(2 * N))[::2], None, s.q, None),
        "slots on the host": lambda f, c: f(q, k, v, c, s.slots.cpu(), None, s.q, None),
        "keys of another type": lambda f, c: f(q, k.float(), v, c, s.slots, None, s.q, None),
        "rows with gaps": lambda f, c: f(q.t().contiguous().t(), k, v, c, s.slots, None, s.q, None),
        "a short output": lambda f, c: f(q, k, v, c, s.slots, None, s.q[1:], None),
        "an output of another type": lambda f, c: f(q, k, v, c, s.slots, None, s.q.float(), None),
        "halves": lambda f, c: f(q.half(), k.half(), v.half(), c, s.slots, None, s.q, None),
        "positions of other rows": lambda f, c: f(q[1:], k[1:], v[1:], c, s.slots[1:], s.rope, s.q[1:], None),
    }
    for name, call in bad.items():
        assert call(calls.kv_append, c) is None, name
        with pytest.raises(ValueError):
            call(tl.kv_append, s.cache)
    bad = {
        "queries of another type": dict(q=s.q.float()), "offsets of other sequences": dict(offsets=s.lens),
        "a table of other sequences": dict(table=_ints([[0, 1], [0, 1]])), "a mask of other rows": dict(mask=s.mask[1:]),
        "a mask with gaps": dict(mask=_ints(np.zeros((N, 6)))[:, ::2]), "a short output": dict(out=s.o[1:]),
        "lengths of another type": dict(lens=s.lens.long()),
    }
    for name, change in bad.items():
        a = dict(q=s.q, table=s.table, lens=s.lens, offsets=s.offsets, mask=s.mask, out=s.o)
        a.update(change)
        assert calls.attention(a["q"], c, a["table"], a["lens"], a["offsets"], N, N, 0.125, a["mask"], a["out"], None) is None, name
        with pytest.raises(ValueError):
            tl.attention(a["q"], s.cache, a["table"], a["lens"], a["offsets"], N, N, 0.125, a["mask"], a["out"])
    with pytest.raises(tl.TLError):                     # the C entry's own refusal
        tl.attention(s.q, s.cache, s.table, s.lens, s.offsets, N, N, -1.0, s.mask, s.o)
    o = tl.attention(s.q, s.cache, s.table, s.lens, s.offsets, N, N, 0.125, s.mask)      # outputs made by the call
    assert o.shape == s.q.shape
    with pytest.raises(ValueError):
        tl.verify(s.logits, s.nodes, s.parents, s.tokens, s.heat.double(), s.uniform, s.noise, 4, s.draft, s.out)
    with pytest.raises(ValueError):
        tl.verify(s.logits, s.nodes, s.parents, s.tokens, s.heat, s.uniform, s.noise, 5, s.draft, s.out)
    with pytest.raises(ValueError):
        tl.kv_keep(s.cache, s.table, _ints([0, 0]), s.out[0], s.out[1])
    with pytest.raises(ValueError):
        tl.kv_read(s.cache, s.slots, s.k[1:], s.v)
    torch.cuda.synchronize()
