"""The short causal convolution, its gradients and its step on the GPU against
the plain 64-bit form.

Bounds, per output, from the roundings of the fp32 computation (u = 2^-24) and
the output's own rounding:
- the sum in front of the activation, s, has W products and W sums:
  |ds| <= (W + 1) u S with S = sum |w x| + |bias|;
- SiLU multiplies an error of s by at most 1.1 and adds its own: exp's argument
  is rounded (|s| u relative), exp, 1 + e, the reciprocal and the product add
  at most 8 u: |dy| <= 1.1 |ds| + (8 + 2 |s|) u |y|;
- its slope's derivative is at most 0.5: |dg| <= |dy| (0.5 |ds| + (12 + 4 |s|) u);
- gradients sum n products of g: |d| <= sum |factor| |dg| + (n + 2) u sum |factor g|.
"""
import numpy as np
import pytest
import torch

import paper_2306_14320_amd as P
from seq_reference import U32, conv1d, equal_starts, gradients, out_round

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16

# (dtype, channels, taps, starts or (tokens, sequences), states, silu, bias, aligned rows)
CASES = [
    (F32, 1, 4, (1, 1), False, True, True, True),
    (F32, 5, 4, (3, 1), True, True, True, False),             # shorter than a tile, scalar loads
    (BF16, 64, 4, (64, 2), False, True, True, True),
    (BF16, 520, 4, (100, 1), True, True, True, True),         # two groups of channels, the last with one vector
    (BF16, 1030, 3, (77, 7), True, True, False, False),
    (F32, 260, 2, [0, 0, 1, 3, 3, 40, 41, 90], True, True, True, True),     # empty and one-token sequences
    (BF16, 72, 4, [5, 5, 6, 8, 70, 133], True, False, True, True),          # rows in front that no sequence holds
    (F32, 33, 8, [2, 4, 9, 60], True, True, True, False),     # sequences shorter than the filter
    (BF16, 136, 1, [0, 17, 50], False, True, True, True),     # one tap: no state
    (F32, 128, 5, [0, 130, 300], False, True, True, True),
    (F32, 64, 6, (48, 3), True, False, False, True),
    (BF16, 16, 7, [3, 3, 3, 20], True, True, True, True),
]
IDS = ["%s-d%d-w%d-%d" % (str(c[0])[6:], c[1], c[2], i) for i, c in enumerate(CASES)]


class Case:
    def __init__(self, dtype, d, w, rows, states, silu, bias, aligned, seed=0):
        g = torch.Generator().manual_seed(1000 + seed)
        if isinstance(rows, tuple):
            self.tokens, self.seqs = rows
            self.starts, self.dense = equal_starts(*rows), True
        else:
            self.starts, self.dense = rows, False
            self.tokens, self.seqs = rows[-1] + 3, len(rows) - 1     # three rows behind the last sequence
        self.dtype, self.d, self.w_, self.silu = dtype, d, w, silu

        def normal(*shape, scale=1.0):
            return (torch.randn(shape, generator=g, dtype=torch.float64) * scale).to(dtype)

        self.ld = 2 * d + (0 if aligned else 3)
        self.wide = normal(self.tokens, self.ld)
        self.x = self.wide[:, :d]
        self.taps = normal(d, w, scale=w ** -0.5)
        self.bias = normal(d) if bias else None
        self.init = normal(self.seqs, w - 1, d) if states else None
        self.dy = normal(self.tokens, d)
        self.d_final = normal(self.seqs, w - 1, d) if states else None
        self.lo, self.hi = self.starts[0], self.starts[-1]
        self.outside = [t for t in range(self.tokens) if not self.lo <= t < self.hi]
        # rows outside hold NaN: they must reach nothing
        self.wide[self.outside] = float("nan")
        self.dy[self.outside] = float("nan")

    def dev(self, t):
        return None if t is None else t.to(DEV)

    def call(self):
        x = self.wide.to(DEV)[:, :self.d]
        desc = P.causal_conv1d_desc_for(x, self.taps, self.seqs, silu=self.silu)
        assert desc.ld_x == (self.ld if self.tokens > 1 else self.d)
        kw = dict(bias=self.dev(self.bias), initial_state=self.dev(self.init),
                  seq_starts=None if self.dense else torch.tensor(self.starts, dtype=torch.int32, device=DEV))
        return x, self.taps.to(DEV), desc, kw

    def clean(self, t):
        t = t.clone()
        t[self.outside] = 0
        return t.double()

    def sums(self):
        """s and S: the sum and the sum of magnitudes."""
        args = [None if v is None else v.double() for v in (self.taps, self.bias)]
        init = None if self.init is None else self.init.double()
        s = conv1d(self.clean(self.x), args[0], args[1], self.starts, init, False)[2]
        big = conv1d(self.clean(self.x).abs(), args[0].abs(), None if args[1] is None else args[1].abs(), self.starts,
                     None if init is None else init.abs(), False)[2]
        return s, big


def guarded(shape, dtype, extra=256):
    """A tensor with a guard band behind it, all NaN."""
    n = int(np.prod(shape))
    buf = torch.full((n + extra,), float("nan"), dtype=dtype, device=DEV)
    return buf[:n].view(shape), buf[n:]


def within(got, ref, bound, what):
    err = (got.double().cpu() - ref).abs()
    assert torch.isfinite(got.cpu()).all(), what
    assert (err <= bound + 1e-30).all(), "%s: error %.3g at bound %.3g" % (what, *max(zip(err.flatten().tolist(), bound.flatten().tolist()), key=lambda p: p[0] - p[1]))


@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_forward(case):
    c = Case(*case)
    x, w, desc, kw = c.call()
    y, guard = guarded((c.tokens, c.d), c.dtype)
    final, fguard = guarded((c.seqs, c.w_ - 1, c.d), c.dtype)
    P.causal_conv1d(x, w, desc, y=y, final_state=final, **kw)
    torch.cuda.synchronize()
    init = None if c.init is None else c.init.double()
    ref, ref_final, s = conv1d(c.clean(c.x), c.taps.double(), None if c.bias is None else c.bias.double(), c.starts, init, c.silu)
    _, big = c.sums()
    ds = (c.w_ + 1) * U32 * big
    bound = 1.1 * ds + (8 + 2 * s.abs()) * U32 * ref.abs() if c.silu else ds
    bound = bound + out_round(c.dtype) * (ref.abs() + bound)
    within(y[c.lo:c.hi], ref[c.lo:c.hi], bound[c.lo:c.hi], "y")
    assert torch.isnan(y[c.outside]).all(), "wrote a row that no sequence holds"
    assert torch.isnan(guard).all() and torch.isnan(fguard).all(), "wrote past an output"
    assert torch.equal(final.double().cpu(), ref_final), "the final state is a copy"


@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_backward(case):
    c = Case(*case)
    x, w, desc, kw = c.call()
    got = P.causal_conv1d_backward(c.dy.to(DEV), x, w, desc, d_final_state=c.dev(c.d_final), **kw)
    again = P.causal_conv1d_backward(c.dy.to(DEV), x, w, desc, d_final_state=c.dev(c.d_final), **kw)
    torch.cuda.synchronize()
    for a, b in zip(got, again):
        assert (a is None) == (b is None)
        if a is not None and a is not got.dx:
            assert torch.equal(a, b), "two calls differ"
    assert torch.equal(got.dx[c.lo:c.hi], again.dx[c.lo:c.hi])

    dbl = [None if v is None else v.double() for v in (c.taps, c.bias, c.init)]
    ref = gradients(lambda x, w, b, i: conv1d(x, w, b, c.starts, i, c.silu)[:2], [c.clean(c.x)] + dbl,
                    [c.clean(c.dy), None if c.d_final is None else c.d_final.double()])
    # magnitudes: the same sums over absolute values, with the error of g in the place of g
    s, big = c.sums()
    dy = c.clean(c.dy).abs()
    sig = torch.sigmoid(s)
    slope = (sig * (1 + s * (1 - sig))).abs() if c.silu else torch.ones_like(s)
    dg = dy * (0.5 * (c.w_ + 1) * U32 * big + (12 + 4 * s.abs()) * U32) if c.silu else torch.zeros_like(s)

    def linear(g, final):   # the gradients are linear in g: the same formulas with magnitudes
        return gradients(lambda x, w, b, i: conv1d(x, w, b, c.starts, i, False)[:2],
                         [c.clean(c.x).abs()] + [None if v is None else v.abs() for v in dbl], [g, final])

    final = None if c.d_final is None else c.d_final.double().abs()
    errs = linear(dg, None if final is None else torch.zeros_like(final))
    mags = linear(dy * slope + dg, final)
    n = c.tokens
    for name, value, r, e, m, terms, dtype in [
            ("dx", got.dx, ref[0], errs[0], mags[0], c.w_, c.dtype), ("dw", got.dw, ref[1], errs[1], mags[1], n, F32),
            ("dbias", got.dbias, ref[2], errs[2], mags[2], n, F32), ("d_initial_state", got.d_initial_state, ref[3], errs[3], mags[3], c.w_, c.dtype)]:
        assert (value is None) == (r is None), name
        if value is None or value.numel() == 0:
            continue
        bound = e + (terms + 2) * U32 * m
        bound = bound + out_round(dtype) * (r.abs() + bound)
        if name == "dx":
            value, r, bound = value[c.lo:c.hi], r[c.lo:c.hi], bound[c.lo:c.hi]
        within(value, r, bound, name)


def test_gradient_against_differences():
    """The fp32 gradients along a random direction against central differences
    of the 64-bit form.  With step h the difference is off by at most
    h^2/6 times a third derivative (under 2 times sum |.|) plus 2^-52 sum|.| / h:
    h = 1e-5 leaves 1e-9 of the sums' magnitude; the fp32 gradients are off by
    less than 1e-5 of it (300 roundings)."""
    c = Case(F32, 24, 4, [0, 2, 19, 19, 40], True, True, True, True, seed=3)
    x, w, desc, kw = c.call()
    got = P.causal_conv1d_backward(c.dy.to(DEV), x, w, desc, d_final_state=c.dev(c.d_final), **kw)
    inputs = [c.clean(c.x), c.taps.double(), c.bias.double(), c.init.double()]
    g = torch.Generator().manual_seed(5)
    dirs = [torch.randn(v.shape, generator=g, dtype=torch.float64) for v in inputs]

    def value(step):
        y, final, _ = conv1d(*[v + step * d for v, d in zip(inputs[:3], dirs[:3])], c.starts, inputs[3] + step * dirs[3])
        return (y * c.clean(c.dy)).sum() + (final * c.d_final.double()).sum()

    grads = [c.clean(got.dx.cpu())] + [v.double().cpu() for v in got[1:]]
    along = sum((v * d).sum() for v, d in zip(grads, dirs))
    big = sum((v * d).abs().sum() for v, d in zip(grads, dirs))
    assert abs((value(1e-5) - value(-1e-5)) / 2e-5 - along) <= 2e-5 * big


@pytest.mark.parametrize("dtype,d,w,requests,aligned", [(BF16, 2048, 4, 5, True), (F32, 37, 3, 9, False), (F32, 64, 1, 3, True), (BF16, 8, 8, 1, True)])
def test_step_walks_a_sequence(dtype, d, w, requests, aligned):
    """Tokens one by one through the step give the prompt call's outputs (the
    same products and sums in the same order: the same bits) and final state."""
    tokens = 11
    g = torch.Generator().manual_seed(7)
    ld = d if aligned else d + 1
    x = torch.randn(tokens, requests, ld, generator=g).to(dtype).to(DEV)[:, :, :d]
    taps, bias = torch.randn(d, w, generator=g).to(dtype).to(DEV), torch.randn(d, generator=g).to(dtype).to(DEV)
    pool = torch.randn(requests + 2, w - 1, d, generator=g).to(dtype).to(DEV)
    slots = (torch.randperm(requests + 2, generator=g)[:requests]).to(torch.int32).to(DEV)
    before = pool.clone()
    rows = x.transpose(0, 1).reshape(requests * tokens, d).contiguous()
    desc = P.causal_conv1d_desc_for(rows, taps, requests)
    final = torch.empty(requests, w - 1, d, dtype=dtype, device=DEV)
    y = P.causal_conv1d(rows, taps, desc, bias=bias, initial_state=before[slots.long()].contiguous(), final_state=final).view(requests, tokens, d)
    step = P.causal_conv1d_desc_for(x[0], taps)
    for t in range(tokens):
        got = P.causal_conv1d_step(x[t], taps, pool, step, bias=bias, slots=slots)
        assert torch.equal(got, y[:, t]), t
    assert torch.equal(pool[slots.long()], final)
    idle = [i for i in range(requests + 2) if i not in slots.tolist()]
    assert torch.equal(pool[idle], before[idle]), "a slot that no request names moved"


def test_step_leaves_requests_without_a_slot():
    d, w = 64, 4
    x = torch.randn(4, d, device=DEV)
    taps = torch.randn(d, w, device=DEV)
    pool = torch.randn(3, w - 1, d, device=DEV)
    before = pool.clone()
    desc = P.causal_conv1d_desc_for(x, taps)
    y = P.causal_conv1d_step(x, taps, pool, desc, slots=torch.tensor([-1, 2, 3, -2 ** 31], dtype=torch.int32, device=DEV))
    assert torch.equal(y[[0, 2, 3]], torch.zeros(3, d, device=DEV))
    assert torch.equal(pool[:2], before[:2]) and not torch.equal(pool[2], before[2])
    assert (y[1] != 0).any()


def test_zero_tokens_copy_the_state():
    x = torch.empty(0, 32, device=DEV)
    taps = torch.randn(32, 4, device=DEV)
    init = torch.randn(2, 3, 32, device=DEV)
    final = torch.empty_like(init)
    desc = P.causal_conv1d_desc_for(x, taps, 2)
    assert P.causal_conv1d(x, taps, desc, initial_state=init, final_state=final).shape == (0, 32)
    assert torch.equal(final, init)
    g = P.causal_conv1d_backward(x, x, taps, desc, initial_state=init, d_final_state=final)
    assert torch.equal(g.dw, torch.zeros(32, 4, device=DEV)) and torch.equal(g.d_initial_state, final)


def test_starts_out_of_range_stay_in_bounds():
    """seq_starts lives on the device, so the host cannot refuse it: values
    outside of the rows are taken as the nearest row."""
    x = torch.randn(40, 32, device=DEV)
    taps = torch.randn(32, 4, device=DEV)
    desc = P.causal_conv1d_desc_for(x, taps, 3)
    y, guard = guarded((40, 32), F32)
    P.causal_conv1d(x, taps, desc, y=y, seq_starts=torch.tensor([-7, 12, 30, 1 << 30], dtype=torch.int32, device=DEV))
    want = P.causal_conv1d(x, taps, desc, seq_starts=torch.tensor([0, 12, 30, 40], dtype=torch.int32, device=DEV))
    assert torch.equal(y, want) and torch.isnan(guard).all()


def test_other_stream_and_graph():
    """A call on a stream of its own, and one captured in a graph and replayed
    with new inputs between eager work."""
    d, w, tokens = 256, 4, 50
    x, taps, bias = torch.randn(tokens, d, device=DEV), torch.randn(d, w, device=DEV), torch.randn(d, device=DEV)
    desc = P.causal_conv1d_desc_for(x, taps, 2)
    want = P.causal_conv1d(x, taps, desc, bias=bias)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = P.causal_conv1d(x, taps, desc, bias=bias, stream=side)
    side.synchronize()
    assert torch.equal(got, want)
    dy, y = torch.randn_like(x), torch.empty_like(x)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        P.causal_conv1d(x, taps, desc, bias=bias, y=y)
        grads = P.causal_conv1d_backward(dy, x, taps, desc, bias=bias)
    for i in range(3):
        x.copy_(torch.randn_like(x))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, P.causal_conv1d(x, taps, desc, bias=bias)), i
        for a, b in zip(grads, P.causal_conv1d_backward(dy, x, taps, desc, bias=bias)):
            assert a is b is None or torch.equal(a, b), i
