"""The example that runs rollouts, log-probabilities and both losses together."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


def test_tuning_under_a_constraint_raises_the_reward():
    from examples import tune_constrained_policy as example
    history, tokens, seen, table = example.run(rounds=8, batch=64, seed=3, verbose=False)
    assert all(math.isfinite(h) for h in history)
    assert history[-1] > history[0] + 0.05, history
    # every drawn token is allowed in the state before it
    live = tokens >= 0
    assert bool((table.delta[seen[live].long(), tokens[live].long()] >= 0).all())
    assert torch.equal(live, live.cummin(1).values), "tokens behind the end of an answer"
