"""The norm of queries and keys with the position rotation on the GPU against
the formulas in 64 bits.

Bounds (u = 2^-24, D channels of a head): mean(x^2) has D + 1 roundings, all
terms positive, so r is off by (D + 2) / 2 + 4 u relative, x r w by two more;
the rotation adds three roundings of terms |u cos| + |u' sin| and the angle's
error times |u| + |u'|.  dx = r (g - n mean(g n)): the sum has D terms of
either sign, off by (D + 8) u mean|g n|; dw sums T times the heads' terms."""
import pytest
import torch

import paper_2306_14320_amd as P
from hybrid_reference import angles, joined, pairs, qk, rotated
from seq_reference import U32, gradients, out_round

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16
EPS = 1e-6

# (dtype, tokens, query heads, key heads, head size, rotated, neighbours, spare elements between rows)
CASES = [
    (F32, 1, 1, 1, 2, 2, False, 0), (BF16, 3, 2, 1, 2, 2, True, 1), (BF16, 5, 4, 2, 64, 64, False, 0), (F32, 4, 3, 3, 80, 40, True, 3),
    (BF16, 7, 10, 5, 80, 40, False, 1), (BF16, 2, 16, 4, 128, 128, False, 128), (F32, 9, 1, 2, 96, 96, False, 0), (BF16, 3, 2, 2, 96, 64, True, 0),
    (BF16, 2, 3, 1, 256, 256, False, 2), (F32, 2, 2, 1, 512, 512, False, 0), (BF16, 3, 2, 1, 512, 256, True, 0), (F32, 3, 2, 1, 70, 34, False, 1),
    (BF16, 2, 1, 1, 510, 6, False, 1), (F32, 5, 4, 0, 32, 0, False, 0), (BF16, 5, 0, 3, 48, 16, True, 0), (BF16, 4500, 3, 1, 32, 16, False, 0),
    (F32, 1, 70, 2, 36, 36, True, 0), (BF16, 2, 2, 1, 200, 200, True, 0),
]
IDS = ["%s-%dx%d+%dx%d-r%d-%d" % ((str(c[0])[6:],) + c[1:6] + (i,)) for i, c in enumerate(CASES)]


class Case:
    def __init__(self, dtype, t, h, k, dim, rot, near, spare, far=True):
        g = torch.Generator().manual_seed(t + 31 * dim + h)

        def normal(*shape, dtype=dtype):
            return torch.randn(shape, generator=g).to(dtype).to(DEV)

        self.dtype, self.t, self.rot, self.near = dtype, t, rot, near
        rows = normal(t, (h + k) * dim + spare)
        self.q, self.k = rows[:, :h * dim].unflatten(1, (h, dim)) if h else rows[:, :0].reshape(t, 0, dim), rows[:, h * dim:(h + k) * dim].unflatten(1, (k, dim)) if k else rows[:, :0].reshape(t, 0, dim)
        self.dyq, self.dyk = normal(t, h, dim), normal(t, k, dim)
        self.wq, self.wk = 1 + 0.2 * normal(dim, dtype=F32), 1 + 0.2 * normal(dim, dtype=F32)
        self.pos = torch.randint(-5, 2 ** 31 - 1 if far else 5000, (t,), generator=g).to(torch.int32).to(DEV)
        self.pos[0] = 0
        self.freqs = (10000.0 ** (-torch.arange(0, rot, 2) / max(rot, 1))).to(DEV)
        self.desc = P.qk_norm_rope_desc_for(self.q, self.k, rot, EPS, near)
        self.angle, self.off = angles(self.pos.cpu(), self.freqs.cpu())
        self.kw = dict(positions=self.pos, freqs=self.freqs)


def _within(got, ref, bound, what):
    err = (got.double().cpu() - ref).abs()
    assert (err <= bound + 1e-30).all(), (what, float((err - bound).max()))


def _mixed(c, u, rel):
    """Error of a rotation of values that are off by rel relative."""
    a, b, rest = pairs(u.abs(), c.rot, c.near)
    cos, sin = torch.cos(c.angle).abs(), torch.sin(c.angle).abs()
    return joined((rel + 3 * U32) * (a * cos + b * sin) + c.off * (a + b), (rel + 3 * U32) * (b * cos + a * sin) + c.off * (a + b), rel * rest, c.near)


@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_forward(case):
    c = Case(*case)
    outs = []
    for x in (c.q, c.k):
        buf = torch.full((x.numel() + 256,), -9.0, dtype=c.dtype, device=DEV)
        outs.append((buf[:x.numel()].view(x.shape), buf[x.numel():]))
    P.qk_norm_rope(c.q, c.k, c.wq, c.wk, c.desc, q_out=outs[0][0], k_out=outs[1][0], **c.kw)
    torch.cuda.synchronize()
    for x, w, (y, guard) in ((c.q, c.wq, outs[0]), (c.k, c.wk, outs[1])):
        assert (guard == -9).all(), "wrote past an output"
        x, w, dim = x.double().cpu(), w.double().cpu(), case[4]
        u = x / (x.square().mean(-1, keepdim=True) + EPS).sqrt() * w
        ref = rotated(u, c.angle, c.rot, c.near)
        e = _mixed(c, u, ((dim + 2) / 2 + 8) * U32)
        _within(y, ref, e + out_round(c.dtype) * (ref.abs() + e), "y")
    # in place where the inputs are dense
    q, k = c.q.contiguous(), c.k.contiguous()
    desc = P.qk_norm_rope_desc_for(q, k, c.rot, EPS, c.near)
    q2, k2 = P.qk_norm_rope(q, k, c.wq, c.wk, desc, q_out=q, k_out=k, **c.kw)
    assert q2 is q and torch.equal(q, outs[0][0]) and torch.equal(k, outs[1][0])


@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_backward(case):
    c = Case(*case)
    args = (c.dyq, c.dyk, c.q, c.k, c.wq, c.wk, c.desc)
    got, again = P.qk_norm_rope_backward(*args, **c.kw), P.qk_norm_rope_backward(*args, **c.kw)
    assert all(torch.equal(a, b) for a, b in zip(got, again)), "two calls differ"
    dim, t = case[4], case[1]
    for x, w, dy, dx, dw in ((c.q, c.wq, c.dyq, got.dq, got.dwq), (c.k, c.wk, c.dyk, got.dk, got.dwk)):
        x, w, dy = x.double().cpu(), w.double().cpu(), dy.double().cpu()
        if not x.numel():
            assert (dw == 0).all()
            continue
        ref = gradients(lambda a, b: (qk(a, b, c.angle, c.rot, c.near, EPS),), [x, w], [dy])
        r = 1 / (x.square().mean(-1, keepdim=True) + EPS).sqrt()
        n, du = x * r, rotated(dy, c.angle, c.rot, c.near, back=True)
        edu = _mixed(c, dy, 0.0)
        g, eg = (du * w).abs(), edu * w.abs()
        k = (g * n.abs()).mean(-1, keepdim=True)
        rel = 2 * (dim + 10) * U32
        e = r * (eg + n.abs() * (eg * n.abs()).mean(-1, keepdim=True) + rel * (g + n.abs() * k))
        _within(dx, ref[0], e + out_round(c.dtype) * (ref[0].abs() + e), "dx")
        terms = (du * n).abs()
        _within(dw, ref[1], ((edu * n.abs()) + (rel + (t * x.shape[1] + 8) * U32) * terms).sum((0, 1)), "dw")
    dyq, dyk = c.dyq.clone(), c.dyk.clone()
    inplace = P.qk_norm_rope_backward(dyq, dyk, *args[2:], dq=dyq, dk=dyk, **c.kw)
    assert inplace.dq is dyq and torch.equal(dyq, got.dq) and torch.equal(dyk, got.dk)


def test_gradient_against_differences():
    """Central differences of the 64-bit form with step 1e-5 are off by about
    1e-10 of the terms' size; the fp32 gradients by under 300 roundings."""
    c = Case(F32, 6, 3, 2, 48, 32, False, 0, far=False)
    g = torch.Generator().manual_seed(8)
    got = P.qk_norm_rope_backward(c.dyq, c.dyk, c.q, c.k, c.wq, c.wk, c.desc, **c.kw)
    at = [v.double().cpu() for v in (c.q, c.k, c.wq, c.wk)]
    way = [torch.randn(v.shape, generator=g, dtype=torch.float64) for v in at]

    def value(s):
        q, k, wq, wk = (v + s * w for v, w in zip(at, way))
        return (qk(q, wq, c.angle, 32, False, EPS) * c.dyq.double().cpu()).sum() + (qk(k, wk, c.angle, 32, False, EPS) * c.dyk.double().cpu()).sum()

    terms = [a.double().cpu() * w for a, w in zip(got, way)]
    assert abs((value(1e-5) - value(-1e-5)) / 2e-5 - sum(v.sum() for v in terms)) <= 2e-5 * sum(v.abs().sum() for v in terms)


def test_zero_tokens_zeros_stream_and_graph():
    w = torch.ones(64, device=DEV)
    none = torch.empty(0, 2, 64, device=DEV)
    desc = P.qk_norm_rope_desc_for(none, none)
    f, p = torch.ones(32, device=DEV), torch.zeros(0, dtype=torch.int32, device=DEV)
    assert P.qk_norm_rope(none, none, w, w, desc, positions=p, freqs=f)[0].shape == (0, 2, 64)
    assert (P.qk_norm_rope_backward(none, none, none, none, w, w, desc, positions=p, freqs=f).dwq == 0).all()
    zero = torch.zeros(3, 2, 64, device=DEV)                    # a head of zeros: x r w is zero
    p = torch.arange(3, dtype=torch.int32, device=DEV)
    assert (P.qk_norm_rope(zero, zero, w, w, P.qk_norm_rope_desc_for(zero, zero), positions=p, freqs=f)[0] == 0).all()
    bad = torch.randn(3, 2, 64, device=DEV)
    good = P.qk_norm_rope(bad, bad, w, w, P.qk_norm_rope_desc_for(bad, bad), positions=p, freqs=f)[0]
    bad[1, 0, 5] = float("nan")                                 # stays in its head
    got = P.qk_norm_rope(bad, bad, w, w, P.qk_norm_rope_desc_for(bad, bad), positions=p, freqs=f)[0]
    assert torch.isnan(got[1, 0]).all() and torch.equal(got[1, 1], good[1, 1]) and torch.equal(got[[0, 2]], good[[0, 2]])
    c = Case(BF16, 40, 4, 2, 64, 64, False, 0)
    want = P.qk_norm_rope(c.q, c.k, c.wq, c.wk, c.desc, **c.kw)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = P.qk_norm_rope(c.q, c.k, c.wq, c.wk, c.desc, stream=side, **c.kw)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))

    def both():
        q, k = P.qk_norm_rope(c.q, c.k, c.wq, c.wk, c.desc, **c.kw)
        return (q, k) + tuple(P.qk_norm_rope_backward(q, k, c.q, c.k, c.wq, c.wk, c.desc, **c.kw))

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = both()
    for n in range(4):
        c.q.copy_(torch.randn_like(c.q))
        c.pos.add_(n)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(captured, both())), n
