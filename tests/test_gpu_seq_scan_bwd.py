"""The gradients of the selective scan on the GPU against the plain 64-bit
form's (through automatic differentiation), and against differences.

Bounds (u = 2^-24; k and the states' magnitudes H and errors E as in
test_gpu_seq_scan.py; kp = (12 + 2 |z|) u for p = dy silu(z), 0 without gate).
The gradient of the state obeys the same kind of recurrence from the end, with
magnitudes G_t = |C p| + a_{t+1} G_{t+1} and errors
    F_t = a F_{t+1} + a G_{t+1} (|s A| k + 6 u) + |C p| (kp + 3 u) + u G_t,
and the outputs are sums of products of these: each adds its factors' errors
and one rounding per term (N states, D channels, T rows).
"""
import pytest
import torch

import paper_2306_14320_amd as P
from seq_cases import BF16, DEV, F32, SCAN, SCAN_IDS, ScanCase
from seq_reference import U32, gradients, out_round, scan
from test_gpu_seq_scan import state_errors, within

pytestmark = pytest.mark.gpu


def bounds(c):
    """Bounds of every gradient before its own rounding, as a dict."""
    x, dt, A, B, C, D, z, bias, init = c.doubles()
    t, d, n, groups = c.tokens, c.d, c.n, c.groups
    per = d // groups
    s, H, E, _ = state_errors(c)
    v = dt if bias is None else dt + bias
    k = (18 + 2 * v.abs()) * U32
    bm, cm = B.abs().repeat_interleave(per, 1), C.abs().repeat_interleave(per, 1)
    dy = c.clean(c.dy)
    zz = torch.zeros_like(x) if z is None else z
    kp = torch.zeros_like(x) if z is None else (12 + 2 * zz.abs()) * U32
    p = dy.abs() if z is None else (dy * z * torch.sigmoid(z)).abs()
    a = torch.exp(s[:, :, None] * A)
    sa = (s[:, :, None] * A).abs()
    G, F = torch.zeros_like(H), torch.zeros_like(H)
    Hp, Ep = torch.zeros_like(H), torch.zeros_like(H)
    di = torch.zeros(c.seqs, d, n, dtype=torch.float64)
    for b, (lo, hi) in enumerate(zip(c.starts, c.starts[1:])):
        g = torch.zeros(d, n, dtype=torch.float64) if c.d_final is None else c.d_final[b].double().abs()
        f = torch.zeros_like(g)
        for i in range(hi - 1, lo - 1, -1):
            put = cm[i] * p[i][:, None]
            f = f + put * (kp[i][:, None] + 3 * U32)
            g = g + put
            f = f + U32 * g
            G[i], F[i] = g, f
            f = a[i] * (f + g * (sa[i] * k[i][:, None] + 6 * U32))
            g = a[i] * g
            if i > lo:
                Hp[i], Ep[i] = H[i - 1], E[i - 1]
            elif init is not None:
                Hp[i] = init[b].abs()
        di[b] = f
    U = (bm * G).sum(2)
    EU = (bm * F).sum(2) + (n + 3) * U32 * U
    skip = torch.zeros_like(x) if D is None else D.expand_as(x).abs()
    out = {"dx": EU * s + U * s * k + skip * p * kp + 3 * U32 * (U * s + skip * p)}
    Q = a * G * Hp
    EQ = a * (F * Hp + G * Ep) + Q * (sa * k[:, :, None] + 8 * U32)
    ds = (A.abs() * Q).sum(2) + x.abs() * U
    eds = (A.abs() * EQ).sum(2) + (n + 5) * U32 * (A.abs() * Q).sum(2) + x.abs() * EU + 2 * U32 * ds
    if c.softplus:
        sig = torch.sigmoid(v)
        eds, ds = eds * sig + ds * sig * (14 + 4 * v.abs()) * U32, ds * sig
    out["ddt"] = eds
    out["dA"] = (s[:, :, None] * EQ + Q * s[:, :, None] * (k[:, :, None] + (t + 4) * U32)).sum(0)
    inn = (s * x).abs()[:, :, None]
    out["dB"] = (inn * F + G * inn * (k[:, :, None] + (per + 6) * U32)).reshape(t, groups, per, n).sum(2)
    out["dC"] = (p[:, :, None] * E + H * p[:, :, None] * (kp[:, :, None] + (per + 6) * U32)).reshape(t, groups, per, n).sum(2)
    out["dD"] = (p * x.abs() * (kp + (t + 3) * U32)).sum(0)
    if z is not None:
        pre = (cm * H).sum(2) + skip * x.abs()
        epre = (cm * E).sum(2) + (n + 4) * U32 * pre
        sig = torch.sigmoid(zz)
        out["dz"] = dy.abs() * sig * (1 + zz.abs()) * (epre + pre * (16 + 4 * zz.abs()) * U32)
    out["ddt_bias"] = (eds + (t + 2) * U32 * ds).sum(0)
    out["d_initial_state"] = di + U32 * di
    return out


NAMES = ("dx", "ddt", "dA", "dB", "dC", "dD", "dz", "ddt_bias", "d_initial_state")


def reference(c):
    x, dt, A, B, C, D, z, bias, init = c.doubles()
    got = gradients(lambda x, dt, A, B, C, D, z, bias, init: scan(x, dt, A, B, C, D, z, bias, c.starts, init, c.softplus),
                    (x, dt, A, B, C, D, z, bias, init), [c.clean(c.dy), None if c.d_final is None else c.d_final.double()])
    return dict(zip(("dx", "ddt", "dA", "dB", "dC", "dD", "dz", "ddt_bias", "d_initial_state"), got))


@pytest.mark.parametrize("case", SCAN, ids=SCAN_IDS)
def test_backward(case):
    c = ScanCase(*case)
    args, desc, kw = c.device()
    d_final = None if c.d_final is None else c.d_final.to(DEV)
    need = P.im2win_selective_scan_backward_workspace_bytes(desc)
    ws = torch.full((need + 256,), 255, dtype=torch.uint8, device=DEV)
    got = P.selective_scan_backward(c.dy.to(DEV), *args, desc, d_final_state=d_final, workspace=ws[:need], **kw)
    torch.cuda.synchronize()
    assert (ws[need:] == 255).all(), "wrote past the workspace"
    ref, bound = reference(c), bounds(c)
    for name in NAMES:
        value, r = getattr(got, name), ref[name]
        assert (value is None) == (r is None), name
        if value is None:
            continue
        b = bound[name] + out_round(value.dtype) * (r.abs() + bound[name])
        if name in ("dx", "ddt", "dB", "dC", "dz"):
            value, r, b = value[c.lo:c.hi], r[c.lo:c.hi], b[c.lo:c.hi]
        within(value, r, b, name)
    again = P.selective_scan_backward(c.dy.to(DEV), *args, desc, d_final_state=d_final, **kw)
    for name in NAMES:
        a, b = getattr(got, name), getattr(again, name)
        if a is not None:
            rows = slice(c.lo, c.hi) if name in ("dx", "ddt", "dB", "dC", "dz") else slice(None)
            assert torch.equal(a[rows], b[rows]), "two calls differ: " + name


def test_outputs_stay_in_bounds():
    """Through the C entry: guard bands behind every output, and rows that no
    sequence holds stay as they were."""
    c = ScanCase(*SCAN[4])
    (x, dt, A, B, C), desc, kw = c.device()
    shapes = dict(dx=((c.tokens, c.d), c.dtype), ddt=((c.tokens, c.d), c.dtype), dA=((c.d, c.n), F32),
                  dB=((c.tokens, c.groups, c.n), c.dtype), dC=((c.tokens, c.groups, c.n), c.dtype), dD=((c.d,), F32),
                  dz=((c.tokens, c.d), c.dtype), ddt_bias=((c.d,), F32), d_initial_state=((c.seqs, c.d, c.n), F32))
    bufs = {}
    for name, (shape, dtype) in shapes.items():
        n = torch.Size(shape).numel()
        bufs[name] = (torch.full((n + 128,), float("nan"), dtype=dtype, device=DEV), n, shape)
    need = P.im2win_selective_scan_backward_workspace_bytes(desc)
    ws = torch.empty(need, dtype=torch.uint8, device=DEV)
    dy, d_final = c.dy.to(DEV), c.d_final.to(DEV)
    P.im2win_selective_scan_backward(desc, dy.data_ptr(), x.data_ptr(), dt.data_ptr(), A.data_ptr(), B.data_ptr(), C.data_ptr(),
                                     kw["D"].data_ptr(), kw["z"].data_ptr(), kw["dt_bias"].data_ptr(), kw["seq_starts"].data_ptr(),
                                     kw["initial_state"].data_ptr(), d_final.data_ptr(), *[bufs[n][0].data_ptr() for n in NAMES],
                                     ws.data_ptr(), need, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    want = P.selective_scan_backward(dy, x, dt, A, B, C, desc, d_final_state=d_final, **kw)
    for name in NAMES:
        buf, n, shape = bufs[name]
        assert torch.isnan(buf[n:]).all(), name
        value, other = buf[:n].view(shape), getattr(want, name)
        if shape[0] == c.tokens:
            assert torch.isnan(value[c.outside]).all(), name
            value, other = value[c.lo:c.hi], other[c.lo:c.hi]
        assert torch.equal(value, other), name


def test_against_differences():
    """Central differences of the 64-bit form along a random direction, step
    1e-5: off by about 1e-9 of the terms' size; the fp32 gradients by their
    bounds, under 2e-5 of it at 60 rows."""
    c = ScanCase(F32, 20, 16, 2, [0, 3, 40, 40, 60], True, True, True, True, True, seed=11)
    args, desc, kw = c.device()
    got = P.selective_scan_backward(c.dy.to(DEV), *args, desc, d_final_state=c.d_final.to(DEV), **kw)
    inputs = c.doubles()
    g = torch.Generator().manual_seed(4)
    dirs = [torch.randn(v.shape, generator=g, dtype=torch.float64) for v in inputs]
    for v in (0, 1, 3, 4, 6):
        dirs[v][c.outside] = 0

    def value(step):
        at = [v + step * d for v, d in zip(inputs, dirs)]
        y, final = scan(*at[:8], c.starts, at[8], True)
        return (y * c.clean(c.dy)).sum() + (final * c.d_final.double()).sum()

    order = (got.dx, got.ddt, got.dA, got.dB, got.dC, got.dD, got.dz, got.ddt_bias, got.d_initial_state)
    terms = []
    for v, d in zip(order, dirs):
        v = v.double().cpu()
        if v.shape[0] == c.tokens:
            v[c.outside] = 0
        terms.append(v * d)
    along, big = sum(v.sum() for v in terms), sum(v.abs().sum() for v in terms)
    assert abs((value(1e-5) - value(-1e-5)) / 2e-5 - along) <= 2e-5 * big


def test_zero_tokens_and_graph():
    A = -torch.ones(8, 4, device=DEV)
    x, B = torch.empty(0, 8, device=DEV), torch.empty(0, 1, 4, device=DEV)
    init = torch.randn(3, 8, 4, device=DEV)
    desc = P.selective_scan_desc_for(x, x, A, B, B, sequences=3)
    g = P.selective_scan_backward(x, x, x, A, B, B, desc, initial_state=init, d_final_state=init)
    assert torch.equal(g.d_initial_state, init) and (g.dA == 0).all()
    c = ScanCase(BF16, 64, 16, 1, (300, 1), True, True, True, True, True)
    args, desc, kw = c.device()
    dy = c.dy.to(DEV)
    graph = torch.cuda.CUDAGraph()
    P.selective_scan_backward(dy, *args, desc, **kw)
    with torch.cuda.graph(graph):
        got = P.selective_scan_backward(dy, *args, desc, **kw)
    for i in range(3):
        args[0].copy_(torch.randn_like(args[0]))
        graph.replay()
        torch.cuda.synchronize()
        want = P.selective_scan_backward(dy, *args, desc, **kw)
        for name in NAMES:
            assert torch.equal(getattr(got, name), getattr(want, name)), (i, name)


def test_starts_out_of_range_stay_in_bounds():
    c = ScanCase(F32, 32, 16, 1, (200, 4), False, True, True, True, True)
    args, desc, kw = c.device()
    dy = c.dy.to(DEV)
    kw["seq_starts"] = torch.tensor([-9, 50, 100, 150, 1 << 30], dtype=torch.int32, device=DEV)
    got = P.selective_scan_backward(dy, *args, desc, **kw)
    kw["seq_starts"] = torch.tensor([0, 50, 100, 150, 200], dtype=torch.int32, device=DEV)
    want = P.selective_scan_backward(dy, *args, desc, **kw)
    assert all(a is b is None or torch.equal(a, b) for a, b in zip(got, want))
