"""Plain 64-bit forms of the operators of hybrid layers for the tests, on the
CPU, straight from the formulas, and the bounds of the kernels' fp32 errors
that follow along a recurrence.

``starts`` is a list of first rows (sequences + 1 values); rows outside of
[starts[0], starts[-1]) are zero in the results.
"""
import torch

from seq_reference import U32


def gates(x, r, i, lam, c):
    """L = log a, a, m = sqrt(1 - a^2) and s(i) x."""
    log_a = -c * torch.logaddexp(lam, torch.zeros_like(lam)) * torch.sigmoid(r)
    return log_a, torch.exp(log_a), torch.sqrt(-torch.expm1(2 * log_a)), torch.sigmoid(i) * x


def recurrence(x, r, i, lam, c, starts, init=None):
    """y and the final states, differentiable."""
    _, a, m, sx = gates(x, r, i, lam, c)
    b = m * sx
    rows, finals = [None] * x.shape[0], []
    for q, (lo, hi) in enumerate(zip(starts, starts[1:])):
        h = init[q] if init is not None else x.new_zeros(x.shape[1])
        for t in range(lo, hi):
            h = a[t] * h + b[t]
            rows[t] = h
        finals.append(h)
    zero = x.new_zeros(x.shape[1])
    return torch.stack([zero if v is None else v for v in rows]) if rows else x, torch.stack(finals)


# Relative errors of the gates, in units of 2^-24: the logistic function and
# the rate c softplus(lam) are products of a few correctly or nearly correctly
# rounded functions, so L is off by at most 10; exp(L) by 10 |L| + 2 and the
# product a h by one more; m by 16 (its series is off by 5e-8, the subtraction
# by 24 where it is used, and the root halves both); b = m s(i) x by 24.
def decay_error(log_a):
    return (12 * log_a.abs() + 4) * U32


INPUT_ERROR = 24 * U32


def recurrence_errors(x, r, i, lam, c, starts, init, dy=None, d_final=None):
    """Bounds of the errors of y and the final states, and of the gradients
    for dy and d_final: the errors of each step carried along by |a|, twice
    (once for the rows, once for the composed pairs of a chunk)."""
    log_a, a, m, sx = gates(x, r, i, lam, c)
    b, da = m * sx, decay_error(log_a)
    t, d = x.shape
    h, eh, before, ebefore = (torch.zeros(t, d, dtype=torch.float64) for _ in range(4))
    efinal = []
    for q, (lo, hi) in enumerate(zip(starts, starts[1:])):
        v = init[q] if init is not None else torch.zeros(d, dtype=torch.float64)
        e = torch.zeros(d, dtype=torch.float64)
        for k in range(lo, hi):
            before[k], ebefore[k] = v, e
            e = a[k] * e + 2 * (da[k] * (a[k] * v).abs() + INPUT_ERROR * b[k].abs())
            v = a[k] * v + b[k]
            e = e + 2 * U32 * v.abs()
            h[k], eh[k] = v, e
        efinal.append(e)
    out = {"y": eh, "final": torch.stack(efinal)}
    if dy is None:
        return out
    g, eg = torch.zeros(t, d, dtype=torch.float64), torch.zeros(t, d, dtype=torch.float64)
    einit = []
    for q, (lo, hi) in enumerate(zip(starts, starts[1:])):
        v = d_final[q] if d_final is not None else torch.zeros(d, dtype=torch.float64)
        e = torch.zeros(d, dtype=torch.float64)
        for k in range(hi - 1, lo - 1, -1):
            v = v + dy[k]
            e = e + 2 * U32 * v.abs()
            g[k], eg[k] = v, e
            e = a[k] * e + 2 * da[k] * (a[k] * v).abs()
            v = a[k] * v
        einit.append(e)
    s, sr = torch.sigmoid(i), torch.sigmoid(r)
    out["dx"] = m * s * eg + 40 * U32 * (g * m * s).abs()
    out["di"] = (x * s * (1 - s)).abs() * (m * eg + 40 * U32 * (g * m).abs()) + 4 * U32 * (g * m * x * s).abs()
    t1, t2 = (a * log_a * before).abs(), (a * a * sx * torch.where(m > 0, log_a / m, 0.0)).abs()
    e = (t1 + t2) * (eg + (60 * U32 + da) * g.abs()) + (g * a * log_a).abs() * ebefore
    out["dr"] = (1 - sr) * e + 4 * U32 * g.abs() * (t1 + t2)
    ratio = torch.sigmoid(lam) / torch.logaddexp(lam, torch.zeros_like(lam))
    out["dlam"] = (e.sum(0) + (t + 40) * U32 * (g.abs() * (t1 + t2)).sum(0)) * ratio
    out["d_init"] = torch.stack(einit)
    return out


def angles(positions, freqs):
    """Angles (T x 1 x R/2) in 64 bits, and how far fp32's cosine of what is
    left behind the whole turns may be off: the turns have a product's error in
    64 bits, the rest is rounded to fp32 (2^-26 turns) and so is the cosine."""
    a = positions.double()[:, None, None] * freqs.double()
    return a, a.abs() * 2.0 ** -51 + 2 * 3.1416 * 2.0 ** -26 + 4 * U32


def pairs(x, rot, near):
    if near:
        return x[..., 0:rot:2], x[..., 1:rot:2], x[..., rot:]
    return x[..., :rot // 2], x[..., rot // 2:rot], x[..., rot:]


def joined(a, b, rest, near):
    return torch.cat((torch.stack((a, b), -1).flatten(-2) if near else torch.cat((a, b), -1), rest), -1)


def rotated(u, angle, rot, near, back=False):
    a, b, rest = pairs(u, rot, near)
    c, s = torch.cos(angle), torch.sin(angle) * (-1 if back else 1)
    return joined(a * c - b * s, b * c + a * s, rest, near)


def qk(x, w, angle, rot, near, eps):
    return rotated(x / (x.square().mean(-1, keepdim=True) + eps).sqrt() * w, angle, rot, near)


def visible(n, m, past, window, sinks):
    """Which of the keys 0 .. m-1 the queries past .. past+n-1 see: n x m."""
    i, j = torch.arange(past, past + n)[:, None], torch.arange(m)[None]
    return (j <= i) & ((j > i - window) | (j < sinks))


def attend(q, k, v, past, window, sinks, scale):
    """One head of one sequence, keys from position 0: y, the log of the sums
    of the exponentials, and the bound of y's fp32 error for weights that are
    rounded to a type of unit roundoff u: a function of u."""
    seen = visible(q.shape[0], k.shape[0], past, window, sinks)
    s = (q @ k.t() * scale).masked_fill(~seen, -float("inf"))
    w = torch.softmax(s, 1)
    # a score is a sum of D products; weights carry its error twice (their own and the sum's)
    size = torch.where(seen, q.abs() @ k.abs().t() * scale, 0.0).amax(1, keepdim=True)
    rel = 2 * (q.shape[1] + 8) * U32 * size + (seen.sum(1, keepdim=True) + 24) * U32
    wv = w @ v.abs()
    return w @ v, torch.logsumexp(s, 1), (lambda u: (rel + u) * wv), (rel + 8 * U32 * (1 + s.amax(1, keepdim=True).abs())).flatten()


def ring_row(p, window, sinks):
    return p if p < sinks else sinks + (p - sinks) % window


def attend_gradients(q, k, v, dy, window, sinks, scale, u):
    """Gradients of one head of one sequence and the bounds of the kernels'
    errors, for operands (weights, ds, the kept y) rounded to unit roundoff u:
    [(dq, bound), (dk, bound), (dv, bound)]."""
    n, d = q.shape
    seen = visible(n, n, 0, window, sinks)
    w = torch.softmax((q @ k.t() * scale).masked_fill(~seen, -float("inf")), 1)
    y, dp = w @ v, dy @ v.t()
    delta = (dy * y).sum(1, keepdim=True)
    ds = torch.where(seen.sum(1, keepdim=True) == 1, torch.zeros_like(w), w * (dp - delta))
    size = torch.where(seen, q.abs() @ k.abs().t() * scale, 0.0).amax(1, keepdim=True)
    rel = 3 * (d + 8) * U32 * size + (seen.sum(1, keepdim=True) + 32) * U32      # of a weight: its score's, and lse's
    edp = (d + 8) * U32 * (dy.abs() @ v.abs().t())
    ey = (rel + u) * (w @ v.abs()) + (u + U32) * y.abs()
    edelta = (dy.abs() * ey).sum(1, keepdim=True) + (d + 8) * U32 * (dy * y).abs().sum(1, keepdim=True)
    eds = w * (rel * (dp - delta).abs() + edp + edelta)
    eds = torch.where(seen.sum(1, keepdim=True) == 1, torch.zeros_like(w), eds + u * (ds.abs() + eds))
    more = (n + 16) * U32
    return [(scale * ds @ k, scale * (eds + more * ds.abs()) @ k.abs()), (scale * ds.t() @ q, scale * (eds + more * ds.abs()).t() @ q.abs()),
            (w.t() @ dy, ((rel + u + more) * w).t() @ dy.abs())]
