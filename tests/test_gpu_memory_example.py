"""The example policy with a memory: it runs, every weight has a gradient, and whole rollouts give what its steps gave."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def test_policy_with_a_memory_runs():
    import math

    import torch
    import depth_policy
    rewards, policy = depth_policy.train(envs=48, steps=10, updates=3, seed=2, memory=True, report=lambda s: None)
    assert len(rewards) == 3 and all(math.isfinite(r) for r in rewards)
    for name, p in policy.named_parameters():
        assert torch.isfinite(p).all() and p.grad is not None and torch.isfinite(p.grad).all() and (p.grad != 0).any(), name


def test_rollouts_give_what_steps_gave():
    import torch
    import depth_policy
    torch.manual_seed(4)
    policy = depth_policy.Policy(memory=True).cuda()
    depth, previous = torch.rand((6, 20, 64, 64), device="cuda") * 5, torch.randint(0, depth_policy.MOVES + 1, (6, 20), device="cuda")
    starts, states = previous == depth_policy.MOVES, policy.memory.start(6)
    with torch.no_grad():
        logits, value = policy(depth, previous, starts, policy.memory.start(6))
        for t in range(20):
            one, v = policy(depth[:, t], previous[:, t], starts[:, t], states)
            # float32 sums of up to 2048 terms, taken in another order by products of other sizes, through norms and twenty steps: 2^-24 times
            # 4096 roundings of numbers of size one, most of which cancel
            assert (one - logits[:, t]).abs().max() < 2.0 ** -12 and (v - value[:, t]).abs().max() < 2.0 ** -12
