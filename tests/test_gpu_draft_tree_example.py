"""The example that runs rotation, prompt attention, tree attention and the cache's step together."""

import os
import sys

import pytest

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def test_drafts_do_not_change_what_is_generated():
    """With a budget that evicts nothing, greedy decoding with drafts gives the tokens that it gives without any, in
    fewer passes."""
    import torch
    import draft_tree as ex
    model = ex.ToyModel(vocab=64, seed=3)
    prompt = torch.randint(0, 64, (150,), generator=torch.Generator().manual_seed(5)).tolist()
    with_drafts, passes, lengths = ex.generate(model, prompt, 80, budget=400)
    without, one_by_one, same = ex.generate(model, prompt, 80, budget=400, depth=0)
    assert with_drafts == without and one_by_one == 79
    assert passes < one_by_one
    assert lengths == same == [150 + 79] * 2


def test_the_budget_holds():
    import draft_tree as ex
    tokens, passes, lengths = ex.main(["--budget", "96", "--tokens", "60"])
    assert len(tokens) == 60 and 0 < passes <= 59 and lengths == [96, 96]
