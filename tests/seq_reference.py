"""Plain 64-bit forms of the sequence operators for the tests, on the CPU and
differentiable: loops over sequences and tokens, straight from the formulas.

``starts`` is a list of first rows (sequences + 1 values); rows outside of
[starts[0], starts[-1]) are zero in the results.
"""
import torch

U32, U16 = 2.0 ** -24, 2.0 ** -8      # unit roundoffs of float32 and bfloat16


def out_round(dtype):
    """Unit roundoff of an output's type (on top of the fp32 computation)."""
    return U16 if dtype == torch.bfloat16 else U32


def equal_starts(tokens, sequences):
    return [i * (tokens // sequences) for i in range(sequences + 1)]


def conv1d(x, w, bias, starts, init=None, silu=True):
    """y, final states and the sums in front of the activation."""
    taps = w.shape[1]
    s = torch.zeros_like(x)
    finals = []
    rows = [None] * x.shape[0]
    for b, (lo, hi) in enumerate(zip(starts, starts[1:])):
        head = init[b] if init is not None else x.new_zeros(taps - 1, x.shape[1])
        line = torch.cat((head, x[lo:hi]))
        for i in range(hi - lo):
            rows[lo + i] = (line[i:i + taps] * w.t()).sum(0) + (bias if bias is not None else 0)
        finals.append(line[hi - lo:])
    s = torch.stack([r if r is not None else x.new_zeros(x.shape[1]) for r in rows]) if rows else s
    y = s * torch.sigmoid(s) if silu else s
    return y, torch.stack(finals), s


def gradients(fn, inputs, weights):
    """Gradients of sum(weights * outputs) for the inputs that are given."""
    leaves = [None if v is None else v.detach().clone().requires_grad_() for v in inputs]
    outs = fn(*leaves)
    total = sum((o * w).sum() for o, w in zip(outs, weights) if w is not None)
    got = iter(torch.autograd.grad(total, [v for v in leaves if v is not None], allow_unused=True))
    return [None if v is None else next(got) for v in leaves]


def scan(x, dt, A, B, C, D, z, dt_bias, starts, init=None, softplus=True):
    """y and the final states of the selective scan.  B and C are T x G x N."""
    t, d = x.shape
    per = d // B.shape[1]
    s = dt if dt_bias is None else dt + dt_bias
    s = torch.logaddexp(s, torch.zeros_like(s)) if softplus else s
    rows, finals = [None] * t, []
    for b, (lo, hi) in enumerate(zip(starts, starts[1:])):
        h = init[b] if init is not None else x.new_zeros(d, A.shape[1])
        for i in range(lo, hi):
            bm, cm = B[i].repeat_interleave(per, 0), C[i].repeat_interleave(per, 0)
            h = torch.exp(s[i][:, None] * A) * h + (s[i] * x[i])[:, None] * bm
            rows[i] = (h * cm).sum(1)
        finals.append(h)
    y = torch.stack([r if r is not None else x.new_zeros(d) for r in rows]) if t else x
    if D is not None:
        y = y + D * x
    if z is not None:
        y = y * z * torch.sigmoid(z)
    return y, torch.stack(finals)
