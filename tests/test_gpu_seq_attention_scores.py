"""Window attention on the GPU where the scores are out of the ordinary: all of
a query's scores minus infinity; scores that climb and fall by more and by less
from one block of keys to the next than the base of the exponentials is left
behind for (2^8), up to magnitudes of 100, with the bounds of the ordinary ones,
which carry the scores' size."""
import pytest
import torch

import paper_2306_14320_amd as P
import test_gpu_seq_attention as forward
import test_gpu_seq_attention_bwd as backward
from hybrid_reference import attend, ring_row
from seq_reference import U16, out_round
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


# what a key's position adds to its scores (natural units; a block has 32 keys)
PROFILES = {
    "climb": lambda p, sinks: 0.25 * (p % 400), "climb slowly": lambda p, sinks: 0.1 * (p % 400), "fall": lambda p, sinks: -0.25 * (p % 400),
    "jump": lambda p, sinks: (0.0, 60.0, -40.0, 95.0, 20.0)[p // 37 % 5], "first tokens": lambda p, sinks: 80.0 if p < sinks else 0.02 * (p % 400),
}
SHAPES = [
    (F32, 4, 2, 64, 200, 2, (420, 1), None, 0), (BF16, 3, 1, 128, 150, 4, [0, 100, 101, 420], [0, 64, 700], 0), (BF16, 2, 2, 64, 300, 3, (450, 1), None, 0),
    (F32, 2, 1, 256, 120, 1, (300, 1), None, 0), (BF16, 4, 1, 256, 130, 0, [0, 290, 330], [90, 500], 0), (BF16, 8, 2, 96, 90, 32, (300, 1), None, 0),
    (F32, 3, 1, 32, 70, 5, [0, 40, 300], [300, 2], 1), (BF16, 64, 64, 64, 200, 2, (520, 1), None, 0),
]
SHAPE_IDS = ["%s-%dq%dk%d-w%d-s%d" % ((str(c[0])[6:],) + c[1:6]) for c in SHAPES]


def _shaped(profile):
    """Case, with a channel of the queries and keys that adds the profile to the scores."""
    def build(*args):
        c = Case(*args)

        def key(p):
            return profile(p, c.sinks) / (4 * c.scale)

        c.q[:, :, 0] = 4
        for b, (lo, hi) in enumerate(zip(c.starts, c.starts[1:])):
            past = c.past_list[b]
            c.k[lo:hi, :, 0] = torch.tensor([key(past + t) for t in range(hi - lo)], device=DEV, dtype=torch.float64).to(c.dtype)[:, None]
            for p in range(past) if c.before else ():
                if p < c.sinks or p >= past - c.window:
                    c.caches[0][c.slots[b], ring_row(p, c.window, c.sinks), :, 0] = key(p)
        c.before = [t.clone() for t in getattr(c, "caches", [])]
        return c
    return build


@pytest.mark.parametrize("profile", PROFILES)
@pytest.mark.parametrize("shape", SHAPES, ids=SHAPE_IDS)
def test_far_apart(shape, profile, monkeypatch):
    monkeypatch.setattr(forward, "Case", _shaped(PROFILES[profile]))
    forward.test_forward(shape)


@pytest.mark.parametrize("profile", PROFILES)
@pytest.mark.parametrize("shape", [s for s in SHAPES if s[7] is None], ids=[i for i, s in zip(SHAPE_IDS, SHAPES) if s[7] is None])
def test_far_apart_gradients(shape, profile, monkeypatch):
    monkeypatch.setattr(backward, "Case", _shaped(PROFILES[profile]))
    backward.test_backward(shape)


@pytest.mark.parametrize("profile", PROFILES)
@pytest.mark.parametrize("dtype, h, kv, dim, window, sinks", [(F32, 4, 1, 64, 3000, 4), (BF16, 8, 2, 128, 2000, 2), (BF16, 4, 4, 256, 600, 0), (F32, 6, 2, 96, 100, 3)])
def test_far_apart_step(dtype, h, kv, dim, window, sinks, profile):
    """Shares of a request's rows, and waves of a share, whose largest scores are far apart."""
    g = torch.Generator().manual_seed(dim)
    n, scale, past = 3, dim ** -0.5, [window + 700, window - 1, 40]
    q, k, v = (torch.randn(n, m, dim, generator=g).to(dtype) for m in (h, kv, kv))
    caches = [torch.randn(n, sinks + window, kv, dim, generator=g).to(dtype) for _ in range(2)]
    q[:, :, 0] = 4
    for b, p in enumerate(past):
        k[b, :, 0] = PROFILES[profile](p, sinks) / (4 * scale)
        for r in range(sinks + window):
            caches[0][b, r, :, 0] = PROFILES[profile](r, sinks) / (4 * scale)      # rows, in the ring's order
    on = [t.to(DEV) for t in (q, k, v, *caches)]
    desc = P.window_attention_desc_for(*on[:3], window, sinks, scale=scale)
    y = P.window_attention_step(*on, torch.tensor(past, dtype=torch.int32, device=DEV), desc)
    u = U16 if dtype == BF16 else 0.0
    for b, p in enumerate(past):
        for c, new in zip(caches, (k, v)):
            c[b, ring_row(p, window, sinks)] = new[b]
        rows = min(p + 1, sinks + window)
        for head in range(h):
            kk, vv = (c[b, :rows, head // (h // kv)].double() for c in caches)
            ref, _, bound, _ = attend(q[b:b + 1, head].double(), kk, vv, rows - 1, rows, 0, scale)
            e = bound(u)
            forward._within(y[b:b + 1, head], ref, e + out_round(dtype) * (ref.abs() + e), ("y", b, head))
