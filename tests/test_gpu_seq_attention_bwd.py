"""Gradients of window attention on the GPU against those of the softmax in 64
bits; the bounds (hybrid_reference.attend_gradients) carry the errors of
scores, weights, the kept y and each operand's rounding through the sums."""
import pytest
import torch

import paper_2306_14320_amd as P
from hybrid_reference import attend, attend_gradients
from seq_reference import U16, gradients, out_round
from test_gpu_seq_attention import Case

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16

# (dtype, heads, key heads, head size, window, sinks, starts or (tokens, sequences), no cache, spare)
CASES = [
    (F32, 1, 1, 8, 1, 0, (1, 1), None, 0), (BF16, 2, 1, 16, 1, 0, (70, 1), None, 8), (BF16, 2, 1, 16, 1, 2, (70, 1), None, 0), (BF16, 4, 4, 64, 7, 0, (70, 2), None, 0),
    (F32, 6, 2, 40, 33, 2, (150, 1), None, 1), (BF16, 8, 2, 128, 100, 4, (333, 1), None, 0), (BF16, 3, 1, 80, 50, 3, (257, 1), None, 5),
    (F32, 5, 5, 96, 64, 0, (130, 1), None, 0), (BF16, 16, 1, 256, 40, 32, (90, 1), None, 0), (F32, 2, 1, 256, 30, 1, (77, 1), None, 0),
    (F32, 4, 2, 192, 65, 5, (140, 1), None, 0), (BF16, 2, 2, 184, 128, 8, (200, 1), None, 0), (BF16, 37, 1, 32, 20, 2, (40, 1), None, 0),
    (BF16, 4, 2, 64, 1000, 4, [0, 0, 1, 5, 130, 130, 131, 400], None, 0),      # empty and one-token sequences
    (F32, 3, 3, 32, 16, 3, [4, 10, 140, 141, 200, 200], None, 3),              # rows outside of the sequences
    (F32, 2, 1, 24, 40, 7, [0, 1200, 1201, 1300], None, 0),                    # first tokens seen by several pieces of queries
    (BF16, 2, 2, 96, 600, 32, (1300, 1), None, 0), (F32, 1, 1, 128, 20, 3, (1100, 2), None, 0),
    (F32, 1, 1, 8, 4, 0, (300, 300), None, 0),                                 # sequences of one token: dq and dk are zero
]
IDS = ["%s-%dq%dk%d-w%d-s%d-%d" % ((str(c[0])[6:],) + c[1:6] + (i,)) for i, c in enumerate(CASES)]


def _within(got, ref, bound, what):
    err = (got.double().cpu() - ref).abs()
    assert (err <= bound + 1e-30).all(), (what, float((err - bound).max()))


def _run(c, dy):
    lse = torch.empty(c.tokens, c.h, device=DEV)
    y = c.run(lse=lse)
    return lambda: P.window_attention_backward(dy, c.q, c.k, c.v, y, lse, c.desc, seq_starts=c.sp)


def _dy(c):
    dy = torch.randn(c.tokens, c.h, c.dim, generator=torch.Generator().manual_seed(7)).to(c.dtype)
    dy[[i for i in range(c.tokens) if i not in set(c.live)]] = float("nan")
    return dy.to(DEV)


@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_backward(case):
    c = Case(*case)
    dy = _dy(c)
    call = _run(c, dy)
    got, again = call(), call()
    assert all(torch.equal(a[c.live], b[c.live]) for a, b in zip(got, again)), "two calls differ"
    u, per = U16 if c.dtype == BF16 else 0.0, c.h // c.kv
    for b, (lo, hi) in enumerate(zip(c.starts, c.starts[1:])):
        for kh in range(c.kv if hi > lo else 0):
            k, v = c.k[lo:hi, kh].double().cpu(), c.v[lo:hi, kh].double().cpu()
            sums = [[0, 0], [0, 0]]
            for head in range(kh * per, kh * per + per):
                (dq, eq), *rest = attend_gradients(c.q[lo:hi, head].double().cpu(), k, v, dy[lo:hi, head].double().cpu(), c.window, c.sinks, c.scale, u)
                _within(got.dq[lo:hi, head], dq, eq + out_round(c.dtype) * (dq.abs() + eq), ("dq", b, head))
                for s, r in zip(sums, rest):
                    s[0], s[1] = s[0] + r[0], s[1] + r[1] * (1 + per * 2.0 ** -24)
            for name, g, (ref, e) in zip(("dk", "dv"), got[1:], sums):
                _within(g[lo:hi, kh], ref, e + out_round(c.dtype) * (ref.abs() + e), (name, b, kh))


def test_formula_is_the_gradient():
    """The reference's own formulas against automatic differentiation."""
    g = torch.Generator().manual_seed(3)
    q, k, v, dy = (torch.randn(23, 6, generator=g, dtype=torch.float64) for _ in range(4))
    want = gradients(lambda a, b, c: (attend(a, b, c, 0, 7, 2, 0.4)[0],), [q, k, v], [dy])
    for (a, _), b in zip(attend_gradients(q, k, v, dy, 7, 2, 0.4, 0.0), want):
        assert (a - b).abs().max() <= 1e-12


def test_gradient_against_differences():
    """Central differences of the 64-bit form with step 1e-5 are off by about
    1e-10 of the terms' size; the fp32 gradients by under 300 roundings."""
    c = Case(F32, 4, 2, 32, 21, 3, (90, 1), None, 0)
    dy = _dy(c)
    got = _run(c, dy)()
    g = torch.Generator().manual_seed(4)
    at = [v.double().cpu() for v in (c.q, c.k, c.v)]
    way = [torch.randn(v.shape, generator=g, dtype=torch.float64) for v in at]

    def value(s):
        q, k, v = (a + s * w for a, w in zip(at, way))
        return sum((attend(q[:, h], k[:, h // 2], v[:, h // 2], 0, 21, 3, c.scale)[0] * dy[:, h].double().cpu()).sum() for h in range(4))

    terms = [a.double().cpu() * w for a, w in zip(got, way)]
    assert abs((value(1e-5) - value(-1e-5)) / 2e-5 - sum(t.sum() for t in terms)) <= 2e-5 * sum(t.abs().sum() for t in terms)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=str)
def test_nan_stays_in_its_sequence(dtype):
    def case():
        return Case(dtype, 4, 2, 64, 20, 2, [0, 90, 91, 300, 350], None, 0)

    c = case()
    dy = _dy(c)
    clean = _run(c, dy)()
    for t, value in ((c.q, float("nan")), (c.k, float("inf")), (c.v, float("nan")), (dy, float("inf"))):
        t[120] = value
    got = _run(c, dy)()
    for rows in (slice(0, 91), slice(300, 350)):
        assert all(torch.equal(a[rows], b[rows]) for a, b in zip(got, clean))


def test_zero_tokens_stream_and_graph():
    none = torch.empty(0, 2, 16, device=DEV)
    desc = P.window_attention_desc_for(none, none, none, 4)
    assert P.window_attention_backward(none, none, none, none, none, torch.empty(0, 2, device=DEV), desc).dq.shape == (0, 2, 16)
    c = Case(BF16, 8, 2, 64, 40, 4, [0, 30, 31, 700], None, 0)
    c.q, c.k, c.v = (t[:700].contiguous() for t in (c.q, c.k, c.v))
    dy = _dy(c)[:700].contiguous()
    desc = P.window_attention_desc_for(c.q, c.k, c.v, 40, 4, 3)

    def both(stream=None):
        lse = torch.empty(700, 8, device=DEV)
        y = P.window_attention(c.q, c.k, c.v, desc, seq_starts=c.sp, lse=lse, stream=stream)
        return (y,) + tuple(P.window_attention_backward(dy, c.q, c.k, c.v, y, lse, desc, seq_starts=c.sp, stream=stream))

    want = both()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = both(side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = both()
    for n in range(4):
        c.k.copy_(torch.randn_like(c.k))
        c.sp.copy_(torch.tensor([0, 100 + n, 300, 700]))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(captured, both())), n
