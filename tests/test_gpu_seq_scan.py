"""The selective scan and its step on the GPU against the plain 64-bit form.

Bounds (u = 2^-24).  The step size s has a relative error of at most 16 u +
2 |v| u from softplus (v the sum in front of it; exp's argument, exp, the
reciprocal, the series); so has exp(s A) |s A| times that, plus the rounded
product s A and exp's own 2 u.  With H the recurrence of magnitudes (H_t = a_t
H_{t-1} + |s x B|), the state's error e obeys
    e_t <= a_t e_{t-1} + a_t H_{t-1} (|s A| k_t + 4 u) + |s x B| (k_t + 3 u) + u H_t,
k_t = (18 + 2 |v|) u.  A chunked run reads states through one more such decay
per chunk (|S A| summed instead of one by one): its error is that of the
factors it replaces plus (chunk rows + 4) u |S A| exp(-|S A|) <= (rows + 4) u
of H, at most once per chunk of 64 rows or more, which 2 u H per row covers.
y adds N + 4 roundings of sum |C| H, D x, and the gate's (12 + 2 |z|) u.
"""
import pytest
import torch

import paper_2306_14320_amd as P
from seq_cases import BF16, DEV, F32, SCAN, SCAN_IDS, ScanCase
from seq_reference import U32, out_round, scan

pytestmark = pytest.mark.gpu


def state_errors(c):
    """Magnitudes H and errors e of the states after each row, T x D x N, and
    those of the final states."""
    x, dt, A, B, C, D, z, bias, init = c.doubles()
    v = dt if bias is None else dt + bias
    s = torch.logaddexp(v, torch.zeros_like(v)) if c.softplus else v
    k = (18 + 2 * v.abs()) * U32
    per = c.d // c.groups
    H = torch.zeros(c.tokens, c.d, c.n, dtype=torch.float64)
    E = torch.zeros_like(H)
    ends = []
    for b, (lo, hi) in enumerate(zip(c.starts, c.starts[1:])):
        h = torch.zeros(c.d, c.n, dtype=torch.float64) if init is None else init[b].abs()
        e = torch.zeros_like(h)
        for i in range(lo, hi):
            sa = s[i][:, None] * A
            a, ki = torch.exp(sa), k[i][:, None]
            new = (s[i] * x[i]).abs()[:, None] * B[i].repeat_interleave(per, 0).abs()
            e = a * e + a * h * (sa.abs() * ki + 6 * U32) + new * (ki + 3 * U32)
            h = a * h + new
            e = e + U32 * h
            H[i], E[i] = h, e
        ends.append((h, e))
    return s, H, E, ends


def y_bound(c, ref, H, E):
    x, dt, A, B, C, D, z, bias, init = c.doubles()
    per = c.d // c.groups
    cm = C.abs().repeat_interleave(per, 1)
    skip = 0 if D is None else (D * x).abs()
    bound = (cm * E).sum(2) + (c.n + 4) * U32 * ((cm * H).sum(2) + skip)
    if z is not None:
        gate = (z * torch.sigmoid(z)).abs()
        bound = bound * gate + (12 + 2 * z.abs()) * U32 * gate * ((cm * H).sum(2) + skip)
    return bound + out_round(c.dtype) * (ref.abs() + bound)


def within(got, ref, bound, what):
    got = got.double().cpu()
    assert torch.isfinite(got).all(), what
    err = (got - ref).abs() - bound
    assert (err <= 1e-30).all(), "%s is %.3g over its bound (%.3g of it)" % (what, err.max(), ((got - ref).abs() / (bound + 1e-30)).max())


@pytest.mark.parametrize("case", SCAN, ids=SCAN_IDS)
def test_forward(case):
    c = ScanCase(*case)
    args, desc, kw = c.device()
    buf = torch.full((c.tokens * c.d + 256,), float("nan"), dtype=c.dtype, device=DEV)
    y = buf[:c.tokens * c.d].view(c.tokens, c.d)
    fbuf = torch.full((c.seqs * c.d * c.n + 256,), float("nan"), device=DEV)
    final = fbuf[:-256].view(c.seqs, c.d, c.n)
    need = P.im2win_selective_scan_workspace_bytes(desc)
    ws = torch.full((need + 256,), 255, dtype=torch.uint8, device=DEV)     # all NaN, and a guard band
    P.selective_scan(*args, desc, y=y, final_state=final, workspace=ws[:need] if need else None, **kw)
    torch.cuda.synchronize()
    ref, ref_final = scan(*c.doubles()[:8], c.starts, c.doubles()[8], c.softplus)
    _, H, E, ends = state_errors(c)
    bound = y_bound(c, ref, H, E)
    within(y[c.lo:c.hi], ref[c.lo:c.hi], bound[c.lo:c.hi], "y")
    within(final, ref_final, torch.stack([e for _, e in ends]), "final_state")
    assert torch.isnan(y[c.outside]).all(), "wrote a row that no sequence holds"
    assert torch.isnan(buf[c.tokens * c.d:]).all() and torch.isnan(fbuf[-256:]).all() and (ws[need:] == 255).all()
    again = torch.empty_like(final)
    y2 = P.selective_scan(*args, desc, final_state=again, **kw)
    assert torch.equal(y2[c.lo:c.hi], y[c.lo:c.hi]) and torch.equal(again, final), "two calls differ"


@pytest.mark.parametrize("case", SCAN, ids=SCAN_IDS)
def test_step_walks_the_sequences(case):
    """The rows of each sequence one by one through the step, against the same
    bounds as the scan over all of them."""
    c = ScanCase(*case)
    (x, dt, A, B, C), _, kw = c.device()
    z, D, bias = kw["z"], kw["D"], kw["dt_bias"]
    longest = min(40, max(b - a for a, b in zip(c.starts, c.starts[1:])))
    pool = torch.randn(c.seqs + 2, c.d, c.n, device=DEV)
    spare = pool[[0, c.seqs + 1]].clone()
    pool[1:-1] = 0 if c.init is None else c.init.to(DEV)
    ref, _ = scan(*c.doubles()[:8], c.starts, c.doubles()[8], c.softplus)
    _, H, E, _ = state_errors(c)
    bound = y_bound(c, ref, H, E)
    for i in range(longest):
        at = [lo + i if lo + i < hi else -1 for lo, hi in zip(c.starts, c.starts[1:])]
        rows = torch.tensor([max(r, c.lo) for r in at], device=DEV)
        slots = torch.tensor([b + 1 if r >= 0 else -1 for b, r in enumerate(at)], dtype=torch.int32, device=DEV)
        ins = [v[rows] for v in (x, dt, B, C)]
        zi = None if z is None else z[rows]
        desc = P.selective_scan_desc_for(ins[0], ins[1], A, ins[2], ins[3], zi, softplus=c.softplus)
        y = P.selective_scan_step(ins[0], ins[1], A, ins[2], ins[3], pool, desc, D=D, z=zi, dt_bias=bias, slots=slots)
        for b, r in enumerate(at):
            if r >= 0:
                within(y[b], ref[r], bound[r], (i, b))
            else:
                assert (y[b] == 0).all()
    assert torch.equal(pool[[0, c.seqs + 1]], spare), "a slot that no request names moved"


def test_step_state_matches_the_reference():
    """The states that the step leaves, for sizes with and without whole
    vectors, against one token of the recurrence in 64 bits."""
    for d, n, groups in ((64, 16, 1), (33, 5, 3), (48, 24, 2), (16, 64, 1)):
        g = torch.Generator().manual_seed(d)
        x, dt = (torch.randn(7, d, generator=g).to(DEV) for _ in range(2))
        B, C = (torch.randn(7, groups, n, generator=g).to(DEV) for _ in range(2))
        A = (-torch.rand(d, n, generator=g) - 0.1).to(DEV)
        pool = torch.randn(9, d, n, generator=g).to(DEV)
        slots = torch.tensor([8, 0, 3, -1, 5, 9, 1], dtype=torch.int32, device=DEV)
        before = pool.clone()
        desc = P.selective_scan_desc_for(x, dt, A, B, C)
        P.selective_scan_step(x, dt, A, B, C, pool, desc, slots=slots)
        for i, slot in enumerate(slots.tolist()):
            if not 0 <= slot < 9:
                continue
            s = torch.nn.functional.softplus(dt[i].double())[:, None]
            decay, put = torch.exp(s * A.double()), s * x[i].double()[:, None] * B[i].double().repeat_interleave(d // groups, 0)
            want = decay * before[slot].double() + put
            tol = 40 * U32 * ((decay * before[slot].double()).abs() * (1 + (s * A.double()).abs()) + put.abs())
            assert ((pool[slot].double() - want).abs() <= tol).all(), (d, n, i)
        for slot in (2, 4, 6, 7):
            assert torch.equal(pool[slot], before[slot])


def test_infinite_and_empty():
    """Zero tokens copy the states; a decay of exactly zero (an infinite step)
    forgets the past."""
    A = -torch.ones(8, 4, device=DEV)
    x = torch.empty(0, 8, device=DEV)
    B = torch.empty(0, 1, 4, device=DEV)
    init = torch.randn(3, 8, 4, device=DEV)
    final = torch.full_like(init, float("nan"))
    desc = P.selective_scan_desc_for(x, x, A, B, B, sequences=3)
    assert P.selective_scan(x, x, A, B, B, desc, initial_state=init, final_state=final).shape == (0, 8)
    assert torch.equal(final, init)
    P.selective_scan(x, x, A, B, B, desc, final_state=final)
    assert (final == 0).all()
    x, B = torch.ones(2, 8, device=DEV), torch.ones(2, 1, 4, device=DEV)
    dt = torch.full((2, 8), 200.0, device=DEV)
    desc = P.selective_scan_desc_for(x, dt, A, B, B)
    final = torch.empty(1, 8, 4, device=DEV)
    y = P.selective_scan(x, dt, A, B, B, desc, initial_state=init[:1].contiguous() * 1e30, final_state=final)
    assert torch.equal(final, torch.full_like(final, 200.0)) and torch.equal(y, torch.full_like(y, 800.0))


def test_starts_out_of_range_stay_in_bounds():
    c = ScanCase(F32, 32, 16, 1, (200, 4), False, True, True, True, True)
    args, desc, kw = c.device()
    kw["seq_starts"] = torch.tensor([-9, 50, 100, 150, 1 << 30], dtype=torch.int32, device=DEV)
    buf = torch.full((200 * 32 + 256,), float("nan"), device=DEV)
    y = buf[:200 * 32].view(200, 32)
    P.selective_scan(*args, desc, y=y, **kw)
    kw["seq_starts"] = torch.tensor([0, 50, 100, 150, 200], dtype=torch.int32, device=DEV)
    assert torch.equal(y, P.selective_scan(*args, desc, **kw)) and torch.isnan(buf[200 * 32:]).all()


def test_other_stream_and_graph():
    c = ScanCase(BF16, 64, 16, 1, (300, 1), True, True, True, True, True)
    args, desc, kw = c.device()
    want = P.selective_scan(*args, desc, **kw)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = P.selective_scan(*args, desc, stream=side, **kw)
    side.synchronize()
    assert torch.equal(got, want)
    final = torch.empty(1, 64, 16, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = P.selective_scan(*args, desc, final_state=final, **kw)
    other = torch.empty_like(final)
    for i in range(3):
        args[0].copy_(torch.randn_like(args[0]))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, P.selective_scan(*args, desc, final_state=other, **kw)) and torch.equal(final, other), i
