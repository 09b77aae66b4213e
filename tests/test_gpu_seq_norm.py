"""The root-mean-square norm with the residual's addition on the GPU against
the formulas in 64 bits.

Bounds (u = 2^-24, D channels, h as the call kept it):
- h: one rounding of a sum, to its type;
- mean(h^2): D + 1 roundings, all terms positive: (D + 2) u relative, half of
  it in r; the division and the root add 2 u, the two products 2 u: y is off
  by at most ((D + 2) / 2 + 6) u |y|, and its own rounding;
- the scale of a block: the same, and a division's u; q is y / scale rounded to
  3 bits of mantissa: half a step is 2^-4 |y/scale|, or 2^-10 below 2^-6;
- dx = r (g - h k) + dres, k = r^2 mean(g h): the sum has D terms of either
  sign, so k is off by (D + 8) u r^2 mean|g h| (and that much from r);
- dw: T terms, each off by ((D + 2) / 2 + 6) u and a rounding.
"""
import numpy as np
import pytest
import torch

import paper_2306_14320_amd as P
from seq_reference import U32, gradients, out_round

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16
EPS = 1e-5

# (dtype, residual's type or None, tokens, channels, block, spare elements between rows of x)
CASES = [
    (BF16, BF16, 1, 1, 0, 0), (F32, F32, 3, 7, 0, 2), (BF16, F32, 5, 64, 16, 0), (F32, BF16, 4, 512, 512, 8),
    (BF16, BF16, 2, 520, 0, 8), (BF16, F32, 7, 2048, 128, 0), (F32, F32, 2, 2049, 0, 0), (BF16, BF16, 3, 4096, 64, 1),
    (BF16, F32, 2, 5001, 0, 0), (F32, F32, 3, 8192, 256, 0), (BF16, BF16, 2, 16384, 128, 0), (BF16, None, 3, 320, 32, 0),
    (F32, None, 1300, 96, 0, 3),
]
IDS = ["%s-%s-%dx%d-b%d" % (str(c[0])[6:], str(c[1])[6:], c[2], c[3], c[4]) for c in CASES]


def _inputs(dtype, rdtype, tokens, d, block, spare):
    g = torch.Generator().manual_seed(tokens * 100003 + d)
    x = torch.randn(tokens, d + spare, generator=g).to(dtype).to(DEV)[:, :d]
    res = None if rdtype is None else (2 * torch.randn(tokens, d, generator=g)).to(rdtype).to(DEV)
    w = (1 + 0.2 * torch.randn(d, generator=g)).to(DEV)
    desc = P.rms_norm_desc_for(tokens, d, dtype, rdtype, EPS, block=0, ld_x=d + spare)
    desc8 = P.rms_norm_desc_for(tokens, d, dtype, rdtype, EPS, block=block, ld_x=d + spare)
    return x, res, w, desc, desc8


def _ref(h, w):
    h = h.double().cpu()
    return h / (h.square().mean(1, keepdim=True) + EPS).sqrt() * w.double().cpu()


def _within(got, ref, bound, what):
    err = (got.double().cpu() - ref).abs()
    assert (err <= bound + 1e-30).all(), (what, float((err - bound).max()))


def _guarded(shape, dtype, extra=512):
    n = int(np.prod(shape))
    buf = torch.full(((n + extra) * dtype.itemsize,), 255, dtype=torch.uint8, device=DEV)
    return buf.view(dtype)[:n].view(shape), buf[n * dtype.itemsize:]


@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_forward(case):
    x, res, w, desc, _ = _inputs(*case)
    shape = (case[2], case[3])
    y, guard = _guarded(shape, x.dtype)
    h, hguard = _guarded(shape, case[1] or x.dtype)
    P.add_rms_norm(x, w, desc, residual=res, y=y, h=h)
    torch.cuda.synchronize()
    assert (guard == 255).all() and (hguard == 255).all(), "wrote past an output"
    want = x.float() + (0 if res is None else res.float())
    assert torch.equal(h, want.to(h.dtype))
    ref = _ref(h, w)
    _within(y, ref, (((case[3] + 2) / 2 + 6) * U32 + out_round(x.dtype)) * 1.01 * ref.abs(), "y")
    if res is not None:      # the sum in place gives the same
        y2, h2 = P.add_rms_norm(x, w, desc, residual=res, h=res)
        assert h2 is res and torch.equal(res, h) and torch.equal(y2, y)
    else:
        y2, h2 = P.add_rms_norm(x, w, desc)
        assert h2 is x and torch.equal(y2, y)


@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_fp8(case):
    x, res, w, _, desc = _inputs(*case)
    t, d, block = case[2], case[3], case[4] or case[3]
    q, guard = _guarded((t, d), torch.float8_e4m3fn)
    scales, sguard = _guarded((t, d // block), F32)
    _, _, h = P.add_rms_norm_fp8(x, w, desc, residual=res, q=q, scales=scales)
    torch.cuda.synchronize()
    assert (guard == 255).all() and (sguard == 255).all(), "wrote past an output"
    ref = _ref(h, w)
    rel = ((d + 2) / 2 + 8) * U32
    top = ref.reshape(t, -1, block).abs().amax(2) / 448
    _within(scales, top, 1.01 * rel * top, "scales")
    exact = ref / top.repeat_interleave(block, 1)
    value = q.cpu().double()
    assert torch.isfinite(value).all()
    _within(value, exact, (exact.abs() * (2.0 ** -4 + 3 * rel)).clamp(min=2.0 ** -10), "q")
    # the largest value of a block is 448 or, by the division's rounding, next to it
    assert (value.reshape(t, -1, block).abs().amax(2) == 448).all()


def test_fp8_of_zeros_and_nan():
    x = torch.zeros(3, 256, device=DEV)
    x[1, 7] = float("nan")
    x[2] = 1
    w = torch.ones(256, device=DEV)
    for block in (0, 64):
        q, scales, _ = P.add_rms_norm_fp8(x, w, P.rms_norm_desc_for(3, 256, F32, block=block))
        assert (scales[:2] == 1).all() and (q[0].float() == 0).all() and torch.isnan(q[1].float()).all()
        assert (q[2].float() == 448).all()


@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_backward(case):
    _, res, w, desc, _ = _inputs(*case)
    t, d = case[2], case[3]
    g = torch.Generator().manual_seed(9)
    hd = case[1] or case[0]
    h = (1.5 * torch.randn(t, d, generator=g)).to(hd).to(DEV)
    dy = torch.randn(t, d, generator=g).to(case[0]).to(DEV)
    dres = None if res is None else torch.randn(t, d, generator=g).to(hd).to(DEV)
    dx, dw = P.add_rms_norm_backward(dy, h, w, desc, d_residual=dres)
    dx2, dw2 = P.add_rms_norm_backward(dy, h, w, desc, d_residual=dres)
    assert torch.equal(dx, dx2) and torch.equal(dw, dw2), "two calls differ"
    hh, ww, dd = h.double().cpu(), w.double().cpu(), dy.double().cpu()
    rr = torch.zeros_like(hh) if dres is None else dres.double().cpu()
    ref = gradients(lambda a, b: ((a / (a.square().mean(1, keepdim=True) + EPS).sqrt() * b), a), [hh, ww], [dd, rr])
    r = 1 / (hh.square().mean(1, keepdim=True) + EPS).sqrt()
    gw = (dd * ww).abs()
    k = r * r * (gw * hh.abs()).mean(1, keepdim=True)
    bound = (2 * (d + 2) + 20) * U32 * r * (gw + hh.abs() * k) + 2 * U32 * rr.abs()
    _within(dx, ref[0], bound + out_round(hd) * (ref[0].abs() + bound), "dx")
    _within(dw, ref[1], (t + (d + 2) / 2 + 10) * U32 * (dd * hh * r).abs().sum(0), "dw")
    if dres is not None:      # in place of the residual's gradient
        again = dres.clone()
        P.add_rms_norm_backward(dy, h, w, desc, d_residual=again, dx=again)
        assert torch.equal(again, dx)


def test_gradient_against_differences():
    """Central differences of the 64-bit form with step 1e-5 are off by about
    1e-10 of the terms' size; the fp32 gradients by under 300 roundings."""
    t, d = 6, 200
    g = torch.Generator().manual_seed(2)
    h, w, dy, ch, cw = (torch.randn(s, generator=g, dtype=torch.float64) for s in ((t, d), (d,), (t, d), (t, d), (d,)))
    desc = P.rms_norm_desc_for(t, d, F32, F32, EPS)
    dx, dw = P.add_rms_norm_backward(dy.float().to(DEV), h.float().to(DEV), w.float().to(DEV), desc)
    h, w, dy = h.float().double(), w.float().double(), dy.float().double()

    def value(s):
        a, b = h + s * ch, w + s * cw
        return (a / (a.square().mean(1, keepdim=True) + EPS).sqrt() * b * dy).sum()

    dx, dw = dx.double().cpu(), dw.double().cpu()
    assert abs((value(1e-5) - value(-1e-5)) / 2e-5 - (dx * ch).sum() - (dw * cw).sum()) <= 2e-5 * ((dx * ch).abs().sum() + (dw * cw).abs().sum())


def test_zero_tokens_stream_and_graph():
    w = torch.ones(64, device=DEV)
    none = torch.empty(0, 64, device=DEV)
    desc = P.rms_norm_desc_for(0, 64, F32)
    assert P.add_rms_norm(none, w, desc)[0].shape == (0, 64)
    assert torch.equal(P.add_rms_norm_backward(none, none, w, desc)[1], torch.zeros(64, device=DEV))
    x, res = torch.randn(9, 64, device=DEV), torch.randn(9, 64, device=DEV)
    desc = P.rms_norm_desc_for(9, 64, F32, block=32)
    side = torch.cuda.Stream()
    want = P.add_rms_norm_fp8(x, w, desc, residual=res)
    side.wait_stream(torch.cuda.current_stream())
    got = P.add_rms_norm_fp8(x, w, desc, residual=res, stream=side)
    side.synchronize()
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(got, want))
    plain = P.rms_norm_desc_for(9, 64, F32)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, h = P.add_rms_norm(x, w, plain, residual=res)
        dx, dw = P.add_rms_norm_backward(y, h, w, plain)
    for i in range(3):
        x.copy_(torch.randn_like(x))
        graph.replay()
        torch.cuda.synchronize()
        y2, h2 = P.add_rms_norm(x, w, plain, residual=res)
        dx2, dw2 = P.add_rms_norm_backward(y2, h2, w, plain)
        assert all(torch.equal(a, b) for a, b in ((y, y2), (h, h2), (dx, dx2), (dw, dw2))), i
