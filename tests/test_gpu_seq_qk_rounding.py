"""The norm with the position rotation in fp32 on the GPU: errors against 64 bits
as root mean squares, in units of u = 2^-24.

A rounding is off by 0.42 u relative as a root mean square.  r: 0.65 (its sum's
error halved by the root, the root and the reciprocal); cosine and sine 0.65.
y = rotated(x r w): r, two products, a product and a sum of the rotation, the angle:
the root of 0.65^2 + 2 0.42^2 + 0.3^2 + 0.42^2 + 0.65^2 is 1.2.  dx = r (du w - n m):
du 0.85 (angle, product, sum), r 0.65, three roundings: 1.3.  dw sums terms of du n,
1.2 each and independent, and so 1.2 of the sum; a level of a sum by pairs adds
0.42 of the sum, a run of K additions as much as K / 2 levels: of some 16 levels
(lanes 4, waves 2, workgroups 3 and 7) 1.7, and 2.1 with the terms'.  Bounds are an
eighth above, a quarter for dw, of which there are as few values as channels."""

import pytest
import torch

import paper_2306_14320_amd as P
from hybrid_reference import qk
from seq_reference import U32, gradients
from test_gpu_seq_qk import EPS, F32, Case

pytestmark = pytest.mark.gpu


def _rms(v):
    return float(v.square().mean().sqrt())


@pytest.mark.parametrize("far", [False, True])
@pytest.mark.parametrize("near", [False, True])
@pytest.mark.parametrize("dim, rot", [(64, 64), (80, 40), (256, 128)])
def test_errors(dim, rot, near, far):
    c = Case(F32, 900, 6, 3, dim, rot, near, 0, far)
    y = P.qk_norm_rope(c.q, c.k, c.wq, c.wk, c.desc, **c.kw)
    g = P.qk_norm_rope_backward(c.dyq, c.dyk, c.q, c.k, c.wq, c.wk, c.desc, **c.kw)
    for x, w, dy, got, dx, dw in ((c.q, c.wq, c.dyq, y[0], g.dq, g.dwq), (c.k, c.wk, c.dyk, y[1], g.dk, g.dwk)):
        x, w, dy = (t.double().cpu() for t in (x, w, dy))
        exact = qk(x, w, c.angle, rot, near, EPS)
        ref = gradients(lambda a, b: (qk(a, b, c.angle, rot, near, EPS),), [x, w], [dy])
        assert _rms(got.double().cpu() - exact) <= 1.2 * 1.125 * U32 * _rms(exact)
        assert _rms(dx.double().cpu() - ref[0]) <= 1.3 * 1.125 * U32 * _rms(ref[0])
        assert _rms(dw.double().cpu() - ref[1]) <= 2.1 * 1.25 * U32 * _rms(ref[1])
