"""The language backbone's operators together, as examples/drafted_actions.py uses them: encoder tokens into the paged
cache, trees of drafts verified in one pass, accepted rows written into their slots."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.parametrize("seed,drafts", [(0, 4), (1, 7), (2, 1)])
def test_trees_say_what_single_tokens_say(seed, drafts):
    import drafted_actions
    said, found, passes_one, passes_tree = drafted_actions.decode(30, seed, drafts)
    assert found == said
    assert len(set(said)) > 5  # (not one token over and over)
    assert passes_tree < passes_one if drafts > 1 else passes_tree <= passes_one


def test_cache_holds_what_single_tokens_would_have_written():
    # the accepted rows' keys and values, wherever their pages are, equal those of decoding one at a time
    import drafted_actions as ex
    import torch
    tokens, h, w = ex.encode(3)
    one, tree = ex.Backbone(tokens.shape[1], 3), ex.Backbone(tokens.shape[1], 3)
    said = [one.prompt(tokens, h, w)]
    assert tree.prompt(tokens, h, w) == said[0]
    for _ in range(6):
        said += one.step(said[-1:], [-1])
    # a chain of right drafts with a wrong branch at every depth
    nodes, parents = [said[0]], [-1]
    at = 0
    for d in range(1, 6):
        nodes += [(said[d] + 1) % 128, said[d]]
        parents += [at, at]
        at = len(nodes) - 1
    assert tree.step(nodes, parents) == said[1:]
    assert tree.length == one.length
    pos = torch.arange(one.length, device="cuda")
    rows = lambda b, c: c[:, b.table[0][pos // ex.PAGE].long(), pos % ex.PAGE].float()
    for a, b in ((rows(one, one.k_cache), rows(tree, tree.k_cache)), (rows(one, one.v_cache), rows(tree, tree.v_cache))):
        # the same arithmetic but for the shape of the projections and the joining of sums: bf16 roundings that differ
        # in the last place, through two layers
        assert (a - b).abs().max() <= 2.0 ** -4 * a.abs().max() and (a - b).norm() <= 2.0 ** -7 * a.norm()
