"""The norm's 8-bit output where a block's scale, its largest magnitude over
448, is a subnormal number or rounds to zero.

eps = 1 and rows of subnormals give r = 1 / sqrt(1 + 0) = 1, so that y is x to
the bit, and scales and codes follow from fp32 divisions that round the same
everywhere: they are compared bit by bit with the host's."""
import numpy as np
import pytest
import torch

import paper_2306_14320_amd as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
ULP = np.float32(2.0 ** -149)
MOST = [1, 100, 223, 224, 225, 600, 671, 672, 1000, 100000, 2 ** 23 - 1, 2 ** 23, 2 ** 26, 448 * 2 ** 23, 2 ** 33]   # in units of 2^-149


def rows_of(block, d):
    """Rows whose blocks have those largest magnitudes, a small value and zero
    beside them; one block of each row is all zeros."""
    g = np.random.default_rng(1)
    x = np.zeros((len(MOST), d), np.float32)
    for i, most in enumerate(MOST):
        for at in range(0, d, block or d):
            n = min(block or d, d - at)
            x[i, at:at + n] = g.integers(-most, most + 1, n).astype(np.float32) * ULP
            x[i, at + n // 2] = -most * ULP
        if block:
            x[i, block:2 * block] = 0
    return x


@pytest.mark.parametrize("block", [0, 64])
def test_scales_that_are_subnormal(block):
    d = 256
    host = rows_of(block, d)
    top = np.abs(host).reshape(len(MOST), -1, block or d).max(2)
    scale = top / np.float32(448)
    scale = np.where(scale > 0, scale, np.float32(1))
    quotient = torch.from_numpy(host / np.repeat(scale, block or d, 1)).clamp(-448, 448)
    x = torch.from_numpy(host).to(DEV)
    desc = P.rms_norm_desc_for(len(MOST), d, torch.float32, torch.float32, 1.0, block=block)
    q, scales, _ = P.add_rms_norm_fp8(x, torch.ones(d, device=DEV), desc)
    assert torch.equal(x.cpu(), torch.from_numpy(host))
    assert np.array_equal(scales.cpu().numpy(), scale)
    assert torch.isfinite(q.cpu().float()).all(), "finite rows have codes without a value"
    assert torch.equal(q.cpu().float(), quotient.to(torch.float8_e4m3fn).float())
