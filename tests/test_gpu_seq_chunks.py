"""The scans at sequences of many chunks: states and gradients that come from
far behind, through chunks that look for themselves and through the carry
kernel."""
import pytest
import torch

import paper_2306_14320_amd as P
from seq_cases import BF16, DEV, F32, ScanCase
from seq_reference import out_round, scan
from test_gpu_seq_scan import state_errors, within, y_bound
from test_gpu_seq_scan_bwd import NAMES, bounds, reference

pytestmark = pytest.mark.gpu

CASES = [
    (F32, 64, 16, 1, (300, 2), True, True, True, False, True),
    (BF16, 50, 16, 1, (201, 3), False, True, True, True, True),
    (F32, 33, 7, 1, (700, 1), True, True, False, True, True),
    (F32, 70, 16, 2, [0, 1, 2, 2, 500, 900], True, True, True, True, True),
    (F32, 21, 24, 1, [4, 40, 480, 510, 511], False, False, True, True, True),
    (BF16, 18, 32, 1, [0, 250, 251, 600], True, True, True, True, False),
    (F32, 20, 40, 1, (102, 3), True, True, False, True, True),
    (F32, 9, 100, 1, [0, 5, 300, 301], True, False, True, True, True),
    (BF16, 24, 64, 2, (400, 1), True, True, True, True, True),
    (F32, 1, 3, 1, [0, 7, 1100, 1107, 1108, 1120], True, True, True, True, True),
]
IDS = ["%d-d%d-n%d" % (i, c[1], c[2]) for i, c in enumerate(CASES)]


@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_scan(case):
    c = ScanCase(*case)
    args, desc, kw = c.device()
    final = torch.empty(c.seqs, c.d, c.n, device=DEV)
    y = P.selective_scan(*args, desc, final_state=final, **kw)
    ref, ref_final = scan(*c.doubles()[:8], c.starts, c.doubles()[8], c.softplus)
    _, H, E, ends = state_errors(c)
    bound = y_bound(c, ref, H, E)
    within(y[c.lo:c.hi], ref[c.lo:c.hi], bound[c.lo:c.hi], "y")
    within(final, ref_final, torch.stack([e for _, e in ends]), "final_state")


@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_scan_gradients(case):
    c = ScanCase(*case)
    args, desc, kw = c.device()
    got = P.selective_scan_backward(c.dy.to(DEV), *args, desc, d_final_state=None if c.d_final is None else c.d_final.to(DEV), **kw)
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
