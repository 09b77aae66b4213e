"""The example block's training step: the gradients that it subtracts, against
the whole block in 64 bits through automatic differentiation and against
differences of its loss.

In fp32 each of under 20 operations in a row sums at most 200 terms, off by
200 u of their magnitudes; with terms ten times their sum that is 2.4e-3 of a
gradient's size, where a wrong factor or a missing path gives far more.  The
loss in 64 bits, differenced over 2e-4 of each weight's scale, is off by 1e-7."""
import os
import sys

import pytest
import torch

from conftest import ROOT
from seq_reference import conv1d, equal_starts, scan

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(ROOT, "examples"))

WEIGHTS = ["w_out", "w_x", "w_dt", "w_in", "conv_w", "conv_b", "A", "D", "dt_bias", "norm_w"]


def loss_of(block, weights, x, h, target, sequences):
    w_out, w_x, w_dt, w_in, conv_w, conv_b, A, D, dt_bias, norm_w = weights
    t, starts, n, r = x.shape[0], equal_starts(x.shape[0], sequences), block.states, block.rank
    v = x + h
    y = v / (v.square().mean(1, keepdim=True) + 1e-5).sqrt() * norm_w
    u, z = (y @ w_in).chunk(2, 1)
    u = conv1d(u, conv_w, conv_b, starts)[0]
    low = u @ w_x
    B, C = low[:, r:r + n].reshape(t, 1, n), low[:, r + n:].reshape(t, 1, n)
    s = scan(u, low[:, :r] @ w_dt, A, B, C, D, z, dt_bias, starts)[0]
    return (s @ w_out - target).square().mean()


def test_gradients_of_a_training_step():
    from mixer_block import Block
    t, width, sequences, rate = 70, 48, 2, 1e6
    block = Block(width, states=5, taps=3, dtype=torch.float32)
    g = torch.Generator().manual_seed(6)
    x, h, target = (torch.randn(t, width, generator=g) for _ in range(3))
    before = [getattr(block, name).double().cpu() for name in WEIGHTS]
    loss = float(block.train(x.cuda(), h.cuda(), target.cuda(), sequences, rate))
    got = [(b - getattr(block, name).double().cpu()) / rate for b, name in zip(before, WEIGHTS)]

    ins = (x.double(), h.double(), target.double(), sequences)
    leaves = [b.clone().requires_grad_() for b in before]
    want = loss_of(block, leaves, *ins)
    assert abs(loss - want.item()) <= 1e-4 * want.item()
    for name, a, b in zip(WEIGHTS, got, torch.autograd.grad(want, leaves)):
        # the subtraction from the weight leaves its rounding over the rate
        slack = 2.0 ** -24 * before[WEIGHTS.index(name)].norm() / rate
        assert (a - b).norm() <= 2.4e-3 * b.norm() + slack, name

    along = [b.square().mean().sqrt().clamp(min=0.1) * torch.randn(b.shape, generator=g, dtype=torch.float64) for b in before]
    step = 1e-4
    moved = [float(loss_of(block, [b + s * d for b, d in zip(before, along)], *ins)) for s in (step, -step)]
    assert abs((moved[0] - moved[1]) / (2 * step) - sum((a * d).sum() for a, d in zip(got, along))) <= 2.4e-3 * sum((a * d).abs().sum() for a, d in zip(got, along))
