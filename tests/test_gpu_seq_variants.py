"""Sizes that reach the kernels' variants for large problems: pairs of channels
beside the carry kernel, longer stripes of the convolution's gradients, and two
requests a workgroup in the scan's step.  Which variant a case takes is read off
the workspace, whose size follows from the chunks or stripes, and asserted.

The references are those of seq_reference.py (the convolution's without its loop
over rows), in 64 bits, on the device where the CPU would take minutes; bounds
as in the files for small sizes."""
import pytest
import torch

import paper_2306_14320_amd as P
from seq_cases import BF16, DEV, F32, ScanCase
from seq_reference import U32, gradients, out_round, scan
from test_gpu_seq_conv1d import Case
from test_gpu_seq_scan import state_errors, within, y_bound
from test_gpu_seq_scan_bwd import NAMES, bounds, reference

pytestmark = pytest.mark.gpu


def up(n):
    return (n + 15) // 16 * 16


# ---------------------------------------------------------------------------
# the scan in pairs of channels, with the carry kernel
# ---------------------------------------------------------------------------
CARRY = [
    (F32, 2047, 16, 1, (2100, 1), True, True, True, True, True),
    (BF16, 895, 7, 1, [2, 700, 701, 701, 2900, 4697], True, True, True, True, False),
    (F32, 2048, 24, 4, (2100, 1), False, True, True, True, True),
    (BF16, 1000, 16, 1, [0, 4200, 4201, 4300], True, False, True, True, True),
]
CARRY_IDS = ["d%d-n%d-g%d" % c[1:4] for c in CARRY]


class DeviceCase(ScanCase):
    """The 64-bit values on the device."""

    def __init__(self, *case):
        super().__init__(*case)
        self.d_final = None if self.d_final is None else self.d_final.to(DEV)

    def clean(self, v):
        return super().clean(v).to(DEV)

    def doubles(self):
        return tuple(None if v is None else v.to(DEV) for v in super().doubles())

    def carry_bytes(self, chunks):
        states = 4 * (2 if self.n <= 8 else 4 if self.n <= 16 else 6)
        return up(chunks * self.d * states * 4), up(chunks * self.d * 4), up(chunks * 4), states

    def chunks(self, desc, backward):
        """The chunks that the workspace is for; None if no number of them is (of pairs of channels, backwards)."""
        for chunks in range(1, self.tokens + 1):
            carry, span, flags, states = self.carry_bytes(chunks)
            if not backward:
                if carry + span + flags == P.im2win_selective_scan_workspace_bytes(desc):
                    return chunks
                continue
            blocks = -(-(self.d // self.groups) // 128)
            if 3 * carry + 3 * span + flags + up(blocks * self.tokens * self.groups * 2 * states * 4) == P.im2win_selective_scan_backward_workspace_bytes(desc):
                return chunks

    def looks_back(self, chunks, depth):
        return chunks <= depth * self.seqs and (self.dense or chunks <= 4 * depth)


@pytest.mark.timeout(300)
@pytest.mark.parametrize("case", CARRY, ids=CARRY_IDS)
def test_scan_of_pairs_with_carries(case):
    c = DeviceCase(*case)
    args, desc, kw = c.device()
    assert c.tokens * c.d >= 1 << 22 and not c.looks_back(c.chunks(desc, False), 32)
    final = torch.empty(c.seqs, c.d, c.n, device=DEV)
    y = P.selective_scan(*args, desc, final_state=final, **kw)
    with torch.device(DEV):
        ref, ref_final = scan(*c.doubles()[:8], c.starts, c.doubles()[8], c.softplus)
        _, H, E, ends = state_errors(c)
        bound = y_bound(c, ref, H, E)
    within(y[c.lo:c.hi], ref[c.lo:c.hi].cpu(), bound[c.lo:c.hi].cpu(), "y")
    within(final, ref_final.cpu(), torch.stack([e for _, e in ends]).cpu(), "final_state")


@pytest.mark.timeout(300)
@pytest.mark.parametrize("case", CARRY, ids=CARRY_IDS)
def test_scan_gradients_of_pairs_with_carries(case):
    c = DeviceCase(*case)
    args, desc, kw = c.device()
    chunks = c.chunks(desc, True)
    assert chunks and not c.looks_back(chunks, 16)
    got = P.selective_scan_backward(c.dy.to(DEV), *args, desc, d_final_state=c.d_final, **kw)
    with torch.device(DEV):
        ref, bound = reference(c), bounds(c)
    for name in NAMES:
        value, r = getattr(got, name), ref[name]
        assert (value is None) == (r is None), name
        if value is None:
            continue
        b = bound[name] + out_round(value.dtype) * (r.abs() + bound[name])
        if name in ("dx", "ddt", "dB", "dC", "dz"):
            value, r, b = value[c.lo:c.hi], r[c.lo:c.hi], b[c.lo:c.hi]
        within(value, r.cpu(), b.cpu(), name)


# ---------------------------------------------------------------------------
# the convolution's gradients in stripes of more than 8 rows
# ---------------------------------------------------------------------------
STRIPES = [
    (16, (F32, 3, 2, [1, 5, 5, 20001], True, True, True, False)),
    (16, (BF16, 1025, 4, (8200, 2), False, True, True, True)),
    (32, (BF16, 9, 3, [0, 11, 13, 40001], True, True, True, False)),
    (64, (F32, 5, 4, [2, 3, 3, 30010, 65600], True, True, True, True)),
    (64, (BF16, 8, 8, (65600, 5), False, False, False, True)),
]


def conv_of_rows(x, w, bias, starts, init, silu):
    """y, final states and the sums in front of the activation, all rows at a time."""
    taps = w.shape[1]
    heads = init if init is not None else x.new_zeros(len(starts) - 1, taps - 1, x.shape[1])
    line = torch.cat([v for b, (lo, hi) in enumerate(zip(starts, starts[1:])) for v in (heads[b], x[lo:hi])])
    at = torch.cat([torch.arange(lo, hi) - starts[0] + b * (taps - 1) for b, (lo, hi) in enumerate(zip(starts, starts[1:]))])     # of a row's first tap
    s = sum(line[at + k] * w[:, k] for k in range(taps)) + (bias if bias is not None else 0)
    s = torch.cat((x.new_zeros(starts[0], x.shape[1]), s, x.new_zeros(x.shape[0] - starts[-1], x.shape[1])))
    ends = [hi - starts[0] + b * (taps - 1) for b, hi in enumerate(starts[1:])]
    return s * torch.sigmoid(s) if silu else s, torch.stack([line[e:e + taps - 1] for e in ends]), s


@pytest.mark.timeout(300)
@pytest.mark.parametrize("stripe,case", STRIPES, ids=["%d-d%d-w%d" % (s, c[1], c[2]) for s, c in STRIPES])
def test_conv_gradients_in_stripes(stripe, case):
    c = Case(*case)
    x, w, desc, kw = c.call()
    parts = -(-c.tokens // (4 * stripe))
    assert P.im2win_causal_conv1d_backward_workspace_bytes(desc) == parts * (c.w_ + 1) * c.d * 4
    got = P.causal_conv1d_backward(c.dy.to(DEV), x, w, desc, d_final_state=c.dev(c.d_final), **kw)
    dbl = [None if v is None else v.double() for v in (c.taps, c.bias, c.init)]
    mag = [None if v is None else v.abs() for v in dbl]
    ref = gradients(lambda x, w, b, i: conv_of_rows(x, w, b, c.starts, i, c.silu)[:2], [c.clean(c.x)] + dbl,
                    [c.clean(c.dy), None if c.d_final is None else c.d_final.double()])
    s = conv_of_rows(c.clean(c.x), dbl[0], dbl[1], c.starts, dbl[2], False)[2]
    big = conv_of_rows(c.clean(c.x).abs(), mag[0], mag[1], c.starts, mag[2], False)[2]
    dy, sig = c.clean(c.dy).abs(), torch.sigmoid(s)
    slope = (sig * (1 + s * (1 - sig))).abs() if c.silu else torch.ones_like(s)
    dg = dy * (0.5 * (c.w_ + 1) * U32 * big + (12 + 4 * s.abs()) * U32) if c.silu else torch.zeros_like(s)
    final = None if c.d_final is None else c.d_final.double().abs()

    def linear(g, f):
        return gradients(lambda x, w, b, i: conv_of_rows(x, w, b, c.starts, i, False)[:2], [c.clean(c.x).abs()] + mag, [g, f])

    errs, mags = linear(dg, None if final is None else torch.zeros_like(final)), linear(dy * slope + dg, final)
    for name, r, e, m, terms, dtype in [("dx", ref[0], errs[0], mags[0], c.w_, c.dtype), ("dw", ref[1], errs[1], mags[1], c.tokens, F32),
                                        ("dbias", ref[2], errs[2], mags[2], c.tokens, F32), ("d_initial_state", ref[3], errs[3], mags[3], c.w_, c.dtype)]:
        value = getattr(got, name)
        assert (value is None) == (r is None), name
        if value is None:
            continue
        bound = e + (terms + 2) * U32 * m
        bound = bound + out_round(dtype) * (r.abs() + bound)
        if name == "dx":
            value, r, bound = value[c.lo:c.hi], r[c.lo:c.hi], bound[c.lo:c.hi]
        within(value, r, bound, name)


# ---------------------------------------------------------------------------
# single tokens, two requests a workgroup
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("dtype,requests,d,n,groups", [(F32, 515, 512, 16, 1), (BF16, 601, 520, 24, 2), (F32, 901, 300, 5, 3), (BF16, 517, 512, 32, 1)])
def test_steps_in_pairs(dtype, requests, d, n, groups):
    """An odd number of requests, every ninth without a slot, against one token
    of the recurrence; |error| of the state as in test_gpu_seq_scan.py."""
    assert requests % 2 and requests // 2 * -(-d * 4 // 256) >= 2048
    g = torch.Generator().manual_seed(requests)
    x, dt, z = (torch.randn(requests, d, generator=g).to(dtype).to(DEV) for _ in range(3))
    B, C = (torch.randn(requests, groups, n, generator=g).to(dtype).to(DEV) for _ in range(2))
    A, D, bias = (-0.2 - 3 * torch.rand(d, n, generator=g)).to(DEV), torch.randn(d, generator=g).to(DEV), (torch.randn(d, generator=g) - 1).to(DEV)
    pool = torch.randn(requests + 3, d, n, generator=g).to(DEV)
    slots = torch.randperm(requests + 3, generator=g)[:requests].to(torch.int32)
    slots[8::9] = -1
    before = pool.double()
    desc = P.selective_scan_desc_for(x, dt, A, B, C, z)
    y = P.selective_scan_step(x, dt, A, B, C, pool, desc, D=D, z=z, dt_bias=bias, slots=slots.to(DEV))
    live, at = (slots >= 0).to(DEV), slots.long().clamp(min=0).to(DEV)
    xd, zd, v = x.double(), z.double(), dt.double() + bias.double()
    s, per = torch.logaddexp(v, torch.zeros_like(v)), d // groups
    bm, cm = (m.double().repeat_interleave(per, 1) for m in (B, C))
    sa, k = s[:, :, None] * A.double(), (18 + 2 * v.abs())[:, :, None] * U32
    past, put = torch.exp(sa) * before[at], (s * xd)[:, :, None] * bm
    h, H = past + put, past.abs() + put.abs()
    E = past.abs() * (sa.abs() * k + 6 * U32) + put.abs() * (k + 3 * U32) + U32 * H
    want = before.clone()
    want[at[live]] = h[live]
    off = torch.zeros_like(want)
    off[at[live]] = E[live]
    within(pool, want.cpu(), off.cpu(), "state")
    gate, skip = zd * torch.sigmoid(zd), D.double() * xd
    ref = ((h * cm).sum(2) + skip) * gate
    big = (cm.abs() * H).sum(2) + skip.abs()
    bound = ((cm.abs() * E).sum(2) + (n + 4) * U32 * big) * gate.abs() + (12 + 2 * zd.abs()) * U32 * gate.abs() * big
    bound = bound + out_round(dtype) * (ref.abs() + bound)
    within(y[live], ref[live].cpu(), bound[live].cpu(), "y")
    assert (y[~live] == 0).all()
