"""The example policy: renderer, embedding, scores and optimiser in one training loop.

The rewards of an update are shares of 2048 steps, whose mean has a standard deviation of at most sqrt(0.25 / 2048) = 0.011; a policy
that learns steps forward more often than the untrained one did by ten of those at least."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.parametrize("bits", [32, 8])
def test_policy_learns_from_frames(bits):
    import torch
    import depth_policy
    rewards, policy = depth_policy.train(envs=128, steps=16, updates=24, lr=2e-3, state_bits=bits, seed=1)
    assert sum(rewards[-3:]) / 3 > rewards[0] + 0.11, rewards
    assert all(torch.isfinite(p).all() for p in policy.parameters())
