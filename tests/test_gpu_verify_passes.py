"""tl_verify where the walk passes over the vocabulary: several workgroups of a sequence share a pass, some sequences
need none.  As tests/test_gpu_verify.py, with numbers that reject most drafted tokens."""
import numpy as np
import pytest

from tests import test_gpu_verify as base
from tests._gpu import banner

pytestmark = pytest.mark.gpu
_lib = base._lib

# seed, sizes, vocabulary, siblings: 16 workgroups to a sequence, 5, 3, 3 and one
CASES = {"one_sequence": (3, [24], 131072, 6), "parts_that_end_short": (1, [40, 1, 9], 40001, 4),
         "forty": (1, [5] * 40, 17000, 3), "eighty": (11, [4, 1, 3, 0] * 20, 24576, 3), "many": (2, [4] * 260, 9001, 3)}


def _rejecting(name, draft, bf16):
    seed, sizes, V, siblings = CASES[name]
    c, bf16, draft = base._case(seed, sizes, V, siblings, draft, bf16, greedy=(0,) if len(sizes) > 1 else ())
    c["uniform"] = (1 - (1 - c["uniform"].astype(np.float64)) * 0.3).astype(np.float32)
    return c, bf16, draft


@pytest.mark.parametrize("name", list(CASES))
@pytest.mark.parametrize("draft,bf16", [("f32", True), ("bf16", False)])
def test_shared_passes(name, draft, bf16):
    banner(f"verify passes {name} draft={draft} bf16={bf16}")
    c, bf16, draft = _rejecting(name, draft, bf16)
    base._check(c, bf16, draft)


def test_repeats_are_equal_and_graphs_replay():
    """Which workgroup takes a part differs from call to call; results do not."""
    import torch
    import paper_2607_04031_amd as tl
    banner("verify passes: repeats and a graph")
    c, bf16, draft = _rejecting("forty", "f32", True)
    i32, f32 = torch.int32, torch.float32
    args = [base._dev(c["logits"], torch.bfloat16), base._dev(c["offsets"], i32), base._dev(c["parents"], i32), base._dev(c["tokens"], i32),
            base._dev(c["temperature"], f32), base._dev(c["uniform"], f32), base._dev(c["noise"], f32), c["max_nodes"]]
    q = base._dev(c["draft"], f32)
    out = tl.verify(*args, draft=q)
    want = [x.cpu() for x in out]
    for _ in range(20):
        for x in out:
            x.fill_(-7)
        tl.verify(*args, draft=q, out=out)
        assert all(torch.equal(x.cpu(), y) for x, y in zip(out, want))
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        tl.verify(*args, draft=q, out=out)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        tl.verify(*args, draft=q, out=out)
    for step in range(4):
        for x in out:
            x.fill_(-7)
        args[5].copy_(base._dev(c["uniform"], f32) if step % 2 == 0 else torch.zeros_like(args[5]))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        if step % 2 == 0:
            assert all(torch.equal(x.cpu(), y) for x, y in zip(out, want))
        else:
            assert bool((out[1] >= 2).any())    # a uniform number of 0 accepts what has any weight


@pytest.mark.parametrize("draft,bf16", [(None, False), ("f32", True), ("bf16", False)])
def test_more_nodes_than_are_held(draft, bf16):
    """Paths past node 256, whose numbers are read as the walk comes to them: every token accepted, then some rejected."""
    banner(f"verify long paths draft={draft} bf16={bf16}")
    c, bf16, draft = base._case(31, [400, 5, 290], 97, 1, draft, bf16)
    c["uniform"][:] = 0.0
    counts = base._check(c, bf16, draft)
    c["uniform"][c["offsets"][0] + 300:c["offsets"][1]] = 0.97
    fewer = base._check(c, bf16, draft)
    assert counts[0] == 400 and 300 <= fewer[0] < 400
