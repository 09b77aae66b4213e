"""Scans whose decay grows: exp(s A) over a chunk of rows passes the range of
fp32 while the states, row by row, do not.

For 24 rows from row 40 on s A is 5.7 to 6.6 a row, e^137 to e^158 over them
and at least e^91 over rows 48 to 63, which are a chunk (16 rows, one workgroup
of 64 channels, at these sizes); it is 0.001 elsewhere.  With "zero" the states
(the gradients) are exactly zero over 60 such rows; with "tiny" they come in at
1e-37 and leave at 1e22 to 1e33.

The bounds are those of test_gpu_seq_scan.py and test_gpu_seq_scan_bwd.py, which
give the step sizes 18 u for softplus.  Here a step is one rounded sum, and the
factor of a chunk of 16 rows errs by 9 u |S A| + 6 u (sums of four rows and over
the four lanes 6 u, log2 e, A log2 e and the product u each; two roots of 2 u
and a product each), which the 18 u |s A| + 6 u of each row cover.
"""
import copy

import pytest
import torch

import paper_2306_14320_amd as P
from seq_cases import DEV, F32, ScanCase
from seq_reference import U32, out_round, scan
from test_gpu_seq_scan import state_errors, within, y_bound
from test_gpu_seq_scan_bwd import NAMES, bounds, reference

pytestmark = pytest.mark.gpu
FROM = 40


def make(rows, growing, tiny):
    """64 channels, one sequence; x is zero up to behind the growing rows."""
    c = ScanCase(F32, 64, 16, 1, (rows, 1), True, True, True, False, True)
    g = torch.Generator().manual_seed(4)
    to = FROM + (24 if tiny else 60)
    c.A = 0.95 + 0.1 * torch.rand(64, 16, generator=g)
    c.dtw = torch.full((rows, 64), 0.001)
    c.dtw[FROM:to] = 6 + 0.25 * torch.rand(to - FROM, 64, generator=g)
    if growing == "steps":      # negative steps and A
        c.A, c.dtw = -c.A, -c.dtw
    c.xz = c.xz.clone()
    c.xz[:120, :64] = 0
    c.tiny = (1 + torch.rand(1, 64, 16, generator=g)) * 1e-37 if tiny else torch.zeros(1, 64, 16)
    return c


# 200 rows are 13 chunks, which add up what comes from before; 700 rows are 44, with a carry kernel
CASES = [(rows, growing, tiny) for rows in (200, 700) for growing in ("steps", "A") for tiny in (False, True)]
IDS = ["%d-%s-%s" % (r, s, "tiny" if t else "zero") for r, s, t in CASES]


@pytest.mark.parametrize("rows,growing,tiny", CASES, ids=IDS)
def test_states(rows, growing, tiny):
    c = make(rows, growing, tiny)
    c.init = c.tiny
    args, desc, kw = c.device()
    final = torch.empty(1, 64, 16, device=DEV)
    y = P.selective_scan(*args, desc, final_state=final, **kw)
    ref, ref_final = scan(*c.doubles()[:8], c.starts, c.doubles()[8], False)
    assert ref.abs().max() < 1e36 and ref_final.abs().max() < 1e36
    _, H, E, ends = state_errors(c)
    within(y, ref, y_bound(c, ref, H, E), "y")
    within(final, ref_final, torch.stack([e for _, e in ends]), "final_state")


@pytest.mark.parametrize("rows,growing,tiny", CASES, ids=IDS)
def test_gradients(rows, growing, tiny):
    """The gradient from behind comes through the growing rows; dy is zero from
    them on, the states up to behind them."""
    c = make(rows, growing, tiny)
    c.init = torch.zeros(1, 64, 16)
    c.d_final = c.tiny
    c.dy = c.dy.clone()
    c.dy[30:] = 0
    args, desc, kw = c.device()
    got = P.selective_scan_backward(c.dy.to(DEV), *args, desc, d_final_state=c.d_final.to(DEV), **kw)
    ref, positive = reference(c), copy.copy(c)
    if growing == "steps":
        positive.A, positive.dtw = -c.A, -c.dtw
    bound = bounds(positive)
    assert all((b >= 0).all() for b in bound.values())
    for name in NAMES:
        value, r = getattr(got, name), ref[name]
        assert (value is None) == (r is None), name
        if value is not None:
            assert r.abs().max() < 1e36, name
            within(value, r, bound[name] + out_round(value.dtype) * (r.abs() + bound[name]), name)
