"""The example's hybrid layers end to end: single tokens continue prompts that
came in parts, and a training step's gradients agree with both layers in 64
bits through automatic differentiation and with differences of the loss.

In fp32 each of under 20 operations in a row sums at most 200 terms, off by
200 u of their magnitudes; with terms ten times their sum that is 2.4e-3 of a
gradient's size, where a wrong factor or a missing path gives far more.  The
loss in 64 bits, differenced over 2e-4 of each weight's scale, is off by 1e-7."""
import os
import sys

import pytest
import torch

from conftest import ROOT
from hybrid_reference import angles, attend, qk, recurrence
from seq_reference import conv1d, equal_starts

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(ROOT, "examples"))
F32 = torch.float32


def _layers(width, dtype=F32):
    from hybrid_block import Attention, Recurrence
    return [Recurrence(width, dtype=dtype), Attention(width, heads=4, kv_heads=2, window=20, sinks=2, dtype=dtype), Recurrence(width, dtype=dtype, seed=5)]


@pytest.mark.parametrize("dtype", [F32, torch.bfloat16], ids=str)
def test_tokens_continue_the_prompt(dtype):
    """Both ways run the same operations on the same rows, in fp32 with sums of
    other orders: 1e-3 covers the 2.4e-3 / 2 of the module's bound for values.
    In bf16 some 30 roundings of 2^-8, half of them of random sign in a product
    of many, leave a few percent."""
    from hybrid_block import serve
    got, want = serve(_layers(64, dtype), [40, 3, 0, 130], 0.4, 25)
    assert torch.isfinite(got).all()
    assert (got.float() - want.float()).norm() <= (1e-3 if dtype == F32 else 0.06) * want.float().norm()


def _loss(layers, weights, x, h, target, sequences):
    t = x.shape[0]
    starts, weights = equal_starts(t, sequences), iter(weights)
    for layer in layers:
        v = x + h
        if hasattr(layer, "lam"):
            w_out, w_gates, w_in, conv_w, conv_b, lam, norm_w = (next(weights) for _ in range(7))
        else:
            w_out, w_qkv, wq, wk, norm_w = (next(weights) for _ in range(5))
        y, h = v / (v.square().mean(1, keepdim=True) + 1e-5).sqrt() * norm_w, v
        if hasattr(layer, "lam"):
            u = conv1d(y @ w_in, conv_w, conv_b, starts, silu=False)[0]
            r, i = (u @ w_gates).chunk(2, 1)
            s = recurrence(u, r, i, lam, 8.0, starts)[0]
        else:
            hq, kv, d = layer.heads, layer.kv, layer.dim
            q, k, v = (p.reshape(t, -1, d) for p in (y @ w_qkv).split([hq * d, kv * d, kv * d], 1))
            angle, _ = angles(torch.arange(t) % (t // sequences), layer.freqs.cpu())
            q, k = qk(q, wq, angle, d, False, 1e-6), qk(k, wk, angle, d, False, 1e-6)
            heads = [torch.cat([attend(q[lo:hi, n], k[lo:hi, n // (hq // kv)], v[lo:hi, n // (hq // kv)], 0, layer.window, layer.sinks, d ** -0.5)[0]
                                for lo, hi in zip(starts, starts[1:])]) for n in range(hq)]
            s = torch.cat(heads, 1)
        x = s @ w_out
    return (x + h - target).square().mean()


def test_gradients_of_a_training_step():
    from hybrid_block import gradients
    t, width, sequences = 80, 64, 2
    layers = _layers(width)
    g = torch.Generator().manual_seed(6)
    x, h, target = (torch.randn(t, width, generator=g) for _ in range(3))
    loss, dx, grads = gradients(layers, x.cuda(), h.cuda(), target.cuda(), sequences)
    got = [dx.double().cpu()] + [d.double().cpu() for _, d in grads]
    at = [x.double()] + [w.double().cpu() for w, _ in grads]

    def value(v):
        return _loss(layers, v[1:], v[0], h.double(), target.double(), sequences)

    leaves = [v.clone().requires_grad_() for v in at]
    want = value(leaves)
    assert abs(float(loss) - want.item()) <= 1e-4 * want.item()
    for n, (a, b) in enumerate(zip(got, torch.autograd.grad(want, leaves))):
        assert (a - b).norm() <= 2.4e-3 * b.norm(), n

    along = [v.square().mean().sqrt().clamp(min=0.1) * torch.randn(v.shape, generator=g, dtype=torch.float64) for v in at]
    step = 1e-4
    moved = [float(value([v + s * d for v, d in zip(at, along)])) for s in (step, -step)]
    assert abs((moved[0] - moved[1]) / (2 * step) - sum((a * d).sum() for a, d in zip(got, along))) <= 2.4e-3 * sum((a * d).abs().sum() for a, d in zip(got, along))


def test_the_script_runs():
    from hybrid_block import main
    main()
