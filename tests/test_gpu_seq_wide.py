"""The sequence operators where sizes change the kernel or the arithmetic of
addresses: scans of so many channels and rows that a lane holds a pair of
channels, rows and states behind 2^31 elements, and NaN that must stay in its
own sequence, channel and group."""
import pytest
import torch

import paper_2306_14320_amd as P
from seq_cases import BF16, DEV, F32, ScanCase
from seq_reference import out_round, scan
from test_gpu_seq_scan import state_errors, within, y_bound
from test_gpu_seq_scan_bwd import NAMES, bounds, reference

pytestmark = pytest.mark.gpu

# rows x channels of 2^22 or more: odd groups whose last pair has one channel of its own
PAIRS = [
    (BF16, 16203, 16, 3, [3, 90, 91, 91, 200, 262], True, True, True, True, False),
    (F32, 17501, 5, 1, [0, 100, 240], True, True, False, True, True),
    (BF16, 16130, 20, 1, (264, 2), False, False, True, True, True),
]
PAIR_IDS = ["d%d-n%d-g%d" % c[1:4] for c in PAIRS]


@pytest.mark.timeout(300)
@pytest.mark.parametrize("case", PAIRS, ids=PAIR_IDS)
def test_scan_of_pairs(case):
    c = ScanCase(*case)
    assert c.tokens * c.d >= 1 << 22
    args, desc, kw = c.device()
    final = torch.empty(c.seqs, c.d, c.n, device=DEV)
    y = P.selective_scan(*args, desc, final_state=final, **kw)
    print("[pairs] forward done", flush=True)
    ref, ref_final = scan(*c.doubles()[:8], c.starts, c.doubles()[8], c.softplus)
    _, H, E, ends = state_errors(c)
    bound = y_bound(c, ref, H, E)
    within(y[c.lo:c.hi], ref[c.lo:c.hi], bound[c.lo:c.hi], "y")
    within(final, ref_final, torch.stack([e for _, e in ends]), "final_state")


@pytest.mark.timeout(300)
@pytest.mark.parametrize("case", PAIRS, ids=PAIR_IDS)
def test_scan_gradients_of_pairs(case):
    c = ScanCase(*case)
    args, desc, kw = c.device()
    got = P.selective_scan_backward(c.dy.to(DEV), *args, desc, d_final_state=None if c.d_final is None else c.d_final.to(DEV), **kw)
    print("[pairs] backward done", flush=True)
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


def test_states_behind_2_31_elements():
    """A pool whose last slot begins behind 2^31 floats."""
    d, n = 2048, 16
    slots = (1 << 31) // (d * n) + 2
    pool = torch.empty(slots, d, n, device=DEV)
    g = torch.Generator(device=DEV).manual_seed(1)
    state = torch.randn(1, d, n, generator=g, device=DEV)
    pool[slots - 1] = state[0]
    x, dt = (torch.randn(1, d, generator=g, device=DEV) for _ in range(2))
    B, C = (torch.randn(1, 1, n, generator=g, device=DEV) for _ in range(2))
    A = -torch.rand(d, n, generator=g, device=DEV)
    desc = P.selective_scan_desc_for(x, dt, A, B, C)
    far = P.selective_scan_step(x, dt, A, B, C, pool, desc, slots=torch.tensor([slots - 1], dtype=torch.int32, device=DEV))
    near = P.selective_scan_step(x, dt, A, B, C, state, desc)
    assert torch.equal(far, near) and torch.equal(pool[slots - 1], state[0])


def test_rows_behind_2_31_elements():
    """Rows 2^27 elements apart, the last ones behind 2^31 elements."""
    d, t, ld = 64, 19, 1 << 27
    store = torch.empty((t - 1) * ld + 2 * d, dtype=BF16, device=DEV)
    wide = store.as_strided((t, 2 * d), (ld, 1))
    wide.copy_(torch.randn(t, 2 * d, device=DEV))
    x, near = wide[:, :d], wide[:, :d].contiguous()
    w = torch.randn(d, 4, device=DEV).to(BF16)
    far, here = P.causal_conv1d_desc_for(x, w), P.causal_conv1d_desc_for(near, w)
    assert far.ld_x == ld
    assert torch.equal(P.causal_conv1d(x, w, far), P.causal_conv1d(near, w, here))
    dy = torch.randn(t, d, device=DEV).to(BF16)
    for a, b in zip(P.causal_conv1d_backward(dy, x, w, far), P.causal_conv1d_backward(dy, near, w, here)):
        assert a is b is None or torch.equal(a, b)
    z, A, B = wide[:, d:], -torch.rand(d, 16, device=DEV), torch.randn(t, 1, 16, device=DEV).to(BF16)
    zn = z.contiguous()
    far, here = P.selective_scan_desc_for(x, x, A, B, B, z), P.selective_scan_desc_for(near, near, A, B, B, zn)
    assert torch.equal(P.selective_scan(x, x, A, B, B, far, z=z), P.selective_scan(near, near, A, B, B, here, z=zn))
    for a, b in zip(P.selective_scan_backward(dy, x, x, A, B, B, far, z=z), P.selective_scan_backward(dy, near, near, A, B, B, here, z=zn)):
        assert a is b is None or torch.equal(a, b)
    norm, plain = P.rms_norm_desc_for(t, d, BF16, ld_x=ld), P.rms_norm_desc_for(t, d, BF16)
    ones = torch.ones(d, device=DEV)
    assert torch.equal(P.add_rms_norm(x, ones, norm)[0], P.add_rms_norm(near, ones, plain)[0])


@pytest.mark.parametrize("rows", [70, 2300], ids=["single", "pairs"])
def test_nan_stays_in_its_sequence(rows):
    """NaN in the middle sequence's x, dt and dy changes nothing of the others'
    rows and states."""
    d, n = 2047, 16
    starts = [0, rows // 3, rows // 3 + 5, rows]
    c = ScanCase(F32, d, n, 1, starts, True, True, True, True, True)
    (x, dt, A, B, C), desc, kw = c.device()
    dy, d_final = c.dy.to(DEV), c.d_final.to(DEV)
    taps, init = torch.randn(d, 4, device=DEV), torch.randn(3, 3, d, device=DEV)
    conv = P.causal_conv1d_desc_for(x, taps, 3)
    mid = slice(starts[1], starts[2])
    keep = torch.ones(c.tokens, dtype=torch.bool, device=DEV)
    keep[mid] = False
    keep[rows:] = False

    def outputs():
        final = torch.empty(3, d, n, device=DEV)
        y = P.selective_scan(x, dt, A, B, C, desc, final_state=final, **kw)
        g = P.selective_scan_backward(dy, x, dt, A, B, C, desc, d_final_state=d_final, **kw)
        u = P.causal_conv1d(x, taps, conv, seq_starts=kw["seq_starts"], initial_state=init)
        k = P.causal_conv1d_backward(dy, x, taps, conv, seq_starts=kw["seq_starts"], initial_state=init)
        return [v[keep] for v in (y, g.dx, g.ddt, g.dB, g.dC, g.dz, u, k.dx)] + [v[[0, 2]] for v in (final, g.d_initial_state, k.d_initial_state)]

    want = outputs()
    for v in (x, dt, dy):
        v[mid] = float("nan")
    for i, (a, b) in enumerate(zip(outputs(), want)):
        assert torch.equal(a, b), i


@pytest.mark.parametrize("rows", [40, 1500], ids=["single", "pairs"])
def test_nan_stays_in_its_channel_and_group(rows):
    """NaN in one channel, the first of the second of two odd groups: the other
    channels' gradients and the first group's dB and dC are as without it."""
    d, n = 2998, 16
    c = ScanCase(F32, d, n, 2, (rows, 1), False, True, True, True, True)
    (x, dt, A, B, C), desc, kw = c.device()
    dy, bad = c.dy.to(DEV), d // 2

    def outputs():
        y = P.selective_scan(x, dt, A, B, C, desc, **kw)
        g = P.selective_scan_backward(dy, x, dt, A, B, C, desc, **kw)
        other = [i for i in range(d) if i != bad]
        return [v[:, other] for v in (y, g.dx, g.ddt, g.dz)] + [v[other] for v in (g.dA, g.dD, g.ddt_bias)] + [g.dB[:, 0], g.dC[:, 0]]

    want = outputs()
    x[:, bad] = float("nan")
    dt[:, bad] = float("nan")
    for i, (a, b) in enumerate(zip(outputs(), want)):
        assert torch.equal(a, b), i
