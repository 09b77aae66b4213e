"""The example block end to end: single tokens continue a prompt, a training
step's gradients lower the loss, and agree with differences of the loss."""
import os
import sys

import pytest
import torch

from conftest import ROOT

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(ROOT, "examples"))


def test_tokens_continue_the_prompt():
    """In fp32 both ways differ by roundings alone: the 8-bit rounding of the
    norm is that of the same rows, so nearly every q is equal; one that is not
    moves its row by a step of 2^-4 in one of 256 products."""
    from mixer_block import Block, serve
    block = Block(256, dtype=torch.float32)
    got, want = serve(block, [40, 1, 0, 130], 5)
    assert torch.isfinite(got).all()
    assert (got - want).norm() <= 1e-3 * want.norm()


def test_training_lowers_the_loss():
    from mixer_block import Block
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(2 * 96, 128, generator=g, device="cuda").to(torch.bfloat16)
    h = torch.randn(2 * 96, 128, generator=g, device="cuda")
    block = Block(128)
    losses = [float(block.train(x, h, torch.roll(x.float(), 1, 0), 2, 5.0)) for _ in range(6)]
    assert all(b < a for a, b in zip(losses, losses[1:])), losses
