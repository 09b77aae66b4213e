"""The norm of more rows than one launch has workgroups for (2^26 of 64
threads): the rows on both sides of the launches' border, and the last ones, are
those of a call over them alone."""
import pytest
import torch

import paper_2306_14320_amd as P

pytestmark = pytest.mark.gpu
DEV, F32 = "cuda:0", torch.float32
ROWS, BORDER, D = (1 << 26) + 37, (1 << 26) - 1, 3


def parts(t):
    return t[BORDER - 40:BORDER + 40], t[-30:], t[:30]


def inputs(dtype):
    g = torch.Generator(device=DEV).manual_seed(8)
    x = torch.randn(ROWS, D + 1, generator=g, device=DEV).to(dtype)[:, :D]
    res = torch.randn(ROWS, D, generator=g, device=DEV)
    return x, res, 1 + 0.1 * torch.randn(D, generator=g, device=DEV)


def test_norm():
    x, res, w = inputs(torch.bfloat16)
    y, h = P.add_rms_norm(x, w, P.rms_norm_desc_for(ROWS, D, x.dtype, F32, ld_x=D + 1), residual=res)
    torch.cuda.synchronize()
    for xs, rs, ys, hs in zip(parts(x), parts(res), parts(y), parts(h)):
        y2, h2 = P.add_rms_norm(xs, w, P.rms_norm_desc_for(len(xs), D, x.dtype, F32, ld_x=D + 1), residual=rs.contiguous())
        assert torch.equal(ys, y2) and torch.equal(hs, h2)


def test_norm_in_8_bits():
    x, _, w = inputs(F32)
    q, scales, h = P.add_rms_norm_fp8(x, w, P.rms_norm_desc_for(ROWS, D, F32, ld_x=D + 1))
    torch.cuda.synchronize()
    assert h is x
    for xs, qs, ss in zip(parts(x), parts(q), parts(scales)):
        q2, s2, _ = P.add_rms_norm_fp8(xs, w, P.rms_norm_desc_for(len(xs), D, F32, ld_x=D + 1))
        assert torch.equal(qs.view(torch.uint8), q2.view(torch.uint8)) and torch.equal(ss, s2)

