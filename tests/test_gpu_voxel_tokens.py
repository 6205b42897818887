"""The example that runs the token operators together: the loss falls, and stepping through the ring gives the packed form's results."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def test_training_lowers_the_loss_and_steps_match():
    import voxel_tokens
    _, losses, state, starts = voxel_tokens.train(20, 1200, log=lambda *_: None)
    assert all(v == v and v < 1e4 for v in losses) and losses[-1] < 0.7 * losses[0]
    # two bf16 results of the same sums: each rounded once (half a step) and made of probabilities rounded once, of values up to `size`
    size = float(voxel_tokens.split_heads(state["w"])[2].abs().max())
    assert voxel_tokens.generate(state, starts, log=lambda *_: None) <= 4 * size * torch.finfo(torch.bfloat16).eps / 2
