"""The norm of rows with gaps between them and without a residual: h is x
itself, and the gradients take it as the forward call returned it."""
import pytest
import torch

import paper_2306_14320_amd as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("side", [False, True], ids=["current", "stream"])
def test_gradients_of_the_h_that_came_back(dtype, side):
    t, d = 9, 70
    wide = torch.randn(t, d + 5, device=DEV).to(dtype)
    x, w, dy = wide[:, 2:2 + d], 1 + 0.1 * torch.randn(d, device=DEV), torch.randn(t, d, device=DEV).to(dtype)
    stream = None
    if side:
        stream = torch.cuda.Stream()
        stream.wait_stream(torch.cuda.current_stream())
    desc = P.rms_norm_desc_for(t, d, dtype, ld_x=d + 5)
    y, h = P.add_rms_norm(x, w, desc, stream=stream)
    assert h is x
    dx, dw = P.add_rms_norm_backward(dy, h, w, desc, stream=stream)
    torch.cuda.synchronize()
    dense = P.rms_norm_desc_for(t, d, dtype)
    y2, h2 = P.add_rms_norm(x.contiguous(), w, dense)
    dx2, dw2 = P.add_rms_norm_backward(dy, h2, w, dense)
    assert torch.equal(y, y2) and torch.equal(dx, dx2) and torch.equal(dw, dw2)


def test_other_layouts_of_h_are_refused():
    w, dy = torch.ones(8, device=DEV), torch.randn(6, 8, device=DEV)
    desc = P.rms_norm_desc_for(6, 8, torch.float32)
    for h in (torch.randn(8, 6, device=DEV).t(), torch.randn(6, 9, device=DEV), torch.randn(6, 8, device=DEV).bfloat16(), torch.randn(6, 8)):
        with pytest.raises(ValueError):
            P.add_rms_norm_backward(dy, h, w, desc)
