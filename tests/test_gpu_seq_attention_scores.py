"""Window attention on the GPU where the scores are out of the ordinary: all of
a query's scores minus infinity."""
import pytest
import torch

import paper_2306_14320_amd as P
from test_gpu_seq_attention import Case

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16


@pytest.mark.parametrize("value", [-float("inf"), -1e30], ids=["infinite", "overflow"])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=str)
def test_scores_of_minus_infinity(dtype, value):
    """The softmax of scores that are all minus infinity is NaN: of a key that
    holds one, and of products beyond fp32.  Other rows keep their values."""
    c = Case(dtype, 4, 2, 64, 20, 0, [0, 90, 91, 300], None, 0)
    clean = c.run()
    rows = slice(150, 170)                     # exactly the window of row 169
    c.q[169, 0], c.q[90, 1], c.q[0, 3] = 0, 0, 0
    c.k[rows, 0], c.k[90, 0], c.k[0, 1] = 0, 0, 0
    c.q[169, 0, 0], c.q[90, 1, 0], c.q[0, 3, 0] = -value if value != -float("inf") else 1, 1e30, 1e30
    c.k[rows, 0, 0], c.k[90, 0, 0], c.k[0, 1, 0] = value, value, value
    lse = torch.zeros(c.tokens, 4, device=DEV)
    y = c.run(lse=lse)
    for t, h in ((169, 0), (90, 1), (0, 3)):
        assert torch.isnan(y[t, h]).all() and lse[t, h] == -float("inf"), (t, h)
    keep = [t for t in range(91, 300) if not 150 <= t < 189]
    assert torch.equal(y[keep], clean[keep]) and torch.equal(y[1:90, :2], clean[1:90, :2])


@pytest.mark.parametrize("window", [40, 3000], ids=["one share", "shares"])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=str)
def test_step_scores_of_minus_infinity(dtype, window):
    g = torch.Generator().manual_seed(window)
    q, k, v = (torch.randn(4, n, 64, generator=g).to(dtype).to(DEV) for n in (4, 2, 2))
    caches = [torch.randn(4, window, 2, 64, generator=g).to(dtype).to(DEV) for _ in range(2)]
    past = torch.tensor([window + 5, 30, window - 1, 0], dtype=torch.int32, device=DEV)
    slots = torch.tensor([3, 0, -1, 1], dtype=torch.int32, device=DEV)
    desc = P.window_attention_desc_for(q, k, v, window)
    assert (P.im2win_window_attention_step_workspace_bytes(desc) > 0) == (window == 3000)
    clean = P.window_attention_step(q, k, v, *[t.clone() for t in caches], past, desc, slots=slots)
    for b, h in ((0, 0), (3, 2)):              # a whole cache, and a first token alone
        q[b, h], k[b, h // 2], caches[0][slots[b], :, h // 2] = 0, 0, 0
        q[b, h, 0], k[b, h // 2, 0], caches[0][slots[b], :, h // 2, 0] = 1, -float("inf"), -float("inf")
    y = P.window_attention_step(q, k, v, *caches, past, desc, slots=slots)
    assert torch.isnan(y[0, 0]).all() and torch.isnan(y[3, 2]).all()
    assert torch.equal(y[1], clean[1]) and (y[2] == 0).all() and torch.equal(y[0, 2:], clean[0, 2:]) and torch.equal(y[3, :2], clean[3, :2])
