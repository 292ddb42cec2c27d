"""The example of generation with drafted tokens, small: a step's operators together.  A generated token may lie below the
largest logit of the prompt pass only by what the two passes differ: rows are grouped differently, so that sums round
differently before bf16 and E4M3, 2^-4 of a value at most there and in the mean far less: a quarter of the logits' standard
deviation is far above that and far below the next best token's place among 512.  The first layer's entries differ by
bf16's rounding of a projection, and where that crosses a tie by one E4M3 step, 2^-3: 0.05 in the norm at most."""
import importlib.util
import os

import pytest

from tests._gpu import banner

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "drafted_decode.py")
    spec = importlib.util.spec_from_file_location("drafted_decode", path)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


@pytest.mark.parametrize("wide", [False, True])
def test_drafts_change_the_steps_and_not_the_text(example, wide):
    banner(f"generation with drafted tokens wide={wide}")
    model = example.Model()
    prompts = [[5, 9, 2, 400, 9], [17], list(range(70))]
    texts, pages, steps = example.generate(model, prompts, 60, wide=wide)
    for p, t in zip(prompts, texts):
        assert t[:len(p)] == p and len(t) - len(p) >= 60 and all(0 <= x < example.VOCAB for x in t)
    short, off = example.check(model, prompts, texts, pages)
    assert short < 0.25 and off < 0.05
    assert steps <= 60


def test_sampling_with_drafts(example):
    banner("generation with drafted tokens, sampled")
    model = example.Model()
    prompts = [[5, 9, 2], [17, 3]]
    texts, pages, steps = example.generate(model, prompts, 30, temperature=0.5)
    _, off = example.check(model, prompts, texts, pages)
    assert off < 0.05
    again, _, _ = example.generate(model, prompts, 30, temperature=0.5)
    assert again == texts
