"""The serving step over a cache of 8 bits as examples/drafted_actions.py runs it."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.parametrize("seed,drafts", [(0, 3), (1, 6), (2, 1)])
def test_sampling_over_eight_bits(seed, drafts):
    import drafted_actions
    said, passes = drafted_actions.sample(30, seed, drafts)
    assert len(said) == 30 and all(0 <= t < 128 for t in said) and len(set(said)) > 5
    assert passes <= 31
    assert drafted_actions.sample(30, seed, drafts) == (said, passes)  # the same seed


@pytest.mark.parametrize("seed,drafts", [(0, 3), (1, 6), (2, 1)])
def test_sampling_takes_fewer_passes_than_tokens(seed, drafts):
    # the prompt's pass gives the first token; if no draft were accepted, every other token would take a pass of its own
    import drafted_actions
    said, passes = drafted_actions.sample(30, seed, drafts)
    assert passes < 30


def test_greedy_steps_over_eight_bits_follow_those_over_sixteen():
    # the first tokens of both: the logits of a prompt, whose rows see each other in 16 bits, are the same; a step's are near
    import drafted_actions as ex
    import torch
    tokens, h, w = ex.encode(3)
    one, eight = ex.Backbone(tokens.shape[1], 3), ex.QuantisedBackbone(tokens.shape[1], 3)
    assert one.prompt(tokens, h, w) == eight.prompt(tokens, h, w)
    cu, slots, pos, mask = one.plan(3, ex._i32(-1, 0, 0))
    _, _, _, _ = eight.plan(3, ex._i32(-1, 0, 0))
    x = one.embed[torch.tensor([5, 7, 9], device="cuda")]
    a, _, _ = one.forward(x, cu, pos, "tree", mask)
    b, _, _ = eight.forward(x, cu, pos, "tree", mask)
    # (codes are off by up to 2^-4 of a value, 2^-4 / sqrt(3) of it in the mean, of keys and values alike and in two layers)
    assert (a - b).norm() <= 0.1 * a.norm()
