"""Window attention in bfloat16 on the GPU: outputs lose no more than their own
rounding.  Next to the exact value rounded once, whose error is taken from the
64-bit result itself, the kernels' fp32 sums and operands in two bfloat16 parts
(off by 2^-16) add under 2^-13 of the summed terms, which for windows up to 64 are at
most some ten times the result: 1/50 of a rounding's 2^-9, and as independent
errors add as squares under 1/1000 of the root mean square; 1.03 leaves room for
the sample (20000 values or more, each error's square spread by less than its size)."""
import pytest
import torch

import paper_2306_14320_amd as P
from hybrid_reference import attend, attend_gradients
from test_gpu_seq_attention import Case

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16 = torch.bfloat16


def _ratio(got, exact):
    """The root mean square error in units of the exact value's rounding."""
    own = (exact.to(BF16).double() - exact).square().mean().sqrt()
    return float((got.double().cpu() - exact).square().mean().sqrt() / own)


def _exact(c, dy, rows):
    """dq, dk and dv in 64 bits of the sequences of (lo, hi) in rows."""
    per = c.h // c.kv
    q, k, v, dy = (t.double().cpu() for t in (c.q, c.k, c.v, dy))
    dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    for lo, hi in rows:
        for h in range(c.h):
            (a, _), (b, _), (d, _) = attend_gradients(q[lo:hi, h], k[lo:hi, h // per], v[lo:hi, h // per], dy[lo:hi, h], c.window, c.sinks, c.scale, 0.0)
            dq[lo:hi, h] = a
            dk[lo:hi, h // per] += b
            dv[lo:hi, h // per] += d
    return dq, dk, dv


@pytest.mark.parametrize("heads", [(2, 2), (4, 1)], ids=["2q2k", "4q1k"])
@pytest.mark.parametrize("dim", [64, 256])
@pytest.mark.parametrize("window, sinks", [(2, 0), (4, 0), (8, 1), (16, 0), (500, 0)])
def test_queries_gradients_where_few_keys_are_seen(window, sinks, dim, heads):
    """delta from the kept y carries that y's rounding, which is as large as dq
    itself where a row sees a few keys: small windows, and the first rows of
    every sequence."""
    c = Case(BF16, *heads, dim, window, sinks, [0, 300, 600], None, 0)
    dy = torch.randn(c.tokens, c.h, dim, generator=torch.Generator().manual_seed(7)).to(BF16).to(DEV)
    lse = torch.empty(c.tokens, c.h, device=DEV)
    y = c.run(lse=lse)
    got = P.window_attention_backward(dy, c.q, c.k, c.v, y, lse, c.desc, seq_starts=c.sp)
    exact = _exact(c, dy, [(0, 300), (300, 600)])[0]
    few = list(range(600)) if window < 64 else [t for t in range(600) if t % 300 < 63]
    assert _ratio(got.dq[few], exact[few]) <= 1.03


@pytest.mark.parametrize("heads", [(4, 2), (64, 64)], ids=["4q2k", "64q64k"])
@pytest.mark.parametrize("dim, window, sinks", [(32, 20, 0), (64, 100, 3), (96, 33, 1), (128, 300, 4), (256, 50, 0)])
def test_outputs_and_keys_gradients(dim, window, sinks, heads):
    """Tiles of 32 keys for their gradients, and with 64 heads of 128."""
    c = Case(BF16, *heads, dim, window, sinks, [0, 250, 420], None, 0)
    dy = torch.randn(c.tokens, c.h, dim, generator=torch.Generator().manual_seed(7)).to(BF16).to(DEV)
    lse = torch.empty(c.tokens, c.h, device=DEV)
    y = c.run(lse=lse)
    got = P.window_attention_backward(dy, c.q, c.k, c.v, y, lse, c.desc, seq_starts=c.sp)
    heads = range(c.h) if c.h < 8 else range(0, c.h, 16)
    if c.h == c.kv:
        keep = list(heads)
        c.q, c.k, c.v, dy, c.h, c.kv = c.q[:, keep], c.k[:, keep], c.v[:, keep], dy[:, keep], len(keep), len(keep)
        y, got = y[:, keep], [g[:, keep] for g in got]
    exact = torch.zeros(c.tokens, c.h, dim, dtype=torch.float64)
    for lo, hi in ((0, 250), (250, 420)):
        for h in range(c.h):
            kh = h // (c.h // c.kv)
            exact[lo:hi, h] = attend(*(t.double().cpu() for t in (c.q[lo:hi, h], c.k[lo:hi, kh], c.v[lo:hi, kh])), 0, window, sinks, c.scale)[0]
    dq, dk, dv = _exact(c, dy, [(0, 250), (250, 420)])
    rows = slice(0, 420)
    assert _ratio(y[rows], exact[rows]) <= 1.03
    assert _ratio(got[1][rows], dk[rows]) <= 1.03
    assert _ratio(got[2][rows], dv[rows]) <= 1.03


@pytest.mark.parametrize("heads, dim, window", [((4, 1), 64, 60), ((16, 4), 128, 200), ((8, 1), 256, 2000)])
def test_steps(heads, dim, window):
    (h, kv), n = heads, 24
    g = torch.Generator().manual_seed(dim)
    q, k, v = (torch.randn(n, m, dim, generator=g).to(BF16) for m in (h, kv, kv))
    caches = [torch.randn(n, window, kv, dim, generator=g).to(BF16) for _ in range(2)]
    past = torch.arange(window + 3, window + 3 + n, dtype=torch.int32)
    args = [t.to(DEV) for t in (q, k, v)]
    y = P.window_attention_step(*args, *(c.to(DEV) for c in caches), past.to(DEV), P.window_attention_desc_for(*args, window))
    exact = torch.zeros(n, h, dim, dtype=torch.float64)
    for b in range(n):
        for c, new in zip(caches, (k, v)):
            c[b, int(past[b]) % window] = new[b]
        for head in range(h):
            exact[b, head] = attend(q[b:b + 1, head].double(), *(c[b, :, head // (h // kv)].double() for c in caches), window - 1, window, 0, dim ** -0.5)[0][0]
    assert _ratio(y, exact) <= 1.03
