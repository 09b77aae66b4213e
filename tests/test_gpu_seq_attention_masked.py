"""Infinities and NaN in window attention on the GPU: they reach what the
formula over the visible pairs alone gives them, and nothing else.  Gradients
that a masked place stood in the way of are computed again, in fp32 in another
order: both orders are off by an output's rounding, twice that for an operand of
a product in bfloat16, and 300 sums' of 2^-24, of the largest value of the row's
channels, within which the terms are."""
import pytest
import torch

import paper_2306_14320_amd as P
from seq_reference import U32, out_round
from test_gpu_seq_attention import Case

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16
INF, NAN = float("inf"), float("nan")


def _formula(c, dy, kh, lo, hi):
    """y, dq, dk and dv in 64 bits of a key head's group in the sequence [lo, hi):
    each query with the keys that it sees and no others."""
    per = c.h // c.kv
    q, dy = (t[lo:hi, kh * per:kh * per + per].double().cpu() for t in (c.q, dy))
    k, v = (t[lo:hi, kh].double().cpu() for t in (c.k, c.v))
    y, dq, dk, dv = torch.zeros_like(q), torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    j = torch.arange(hi - lo)
    for t in range(hi - lo):
        see = (j <= t) & ((j > t - c.window) | (j < c.sinks))
        w = torch.softmax((k[see] * q[t, :, None]).sum(-1) * c.scale, 1)       # heads x keys
        y[t] = (w[:, :, None] * v[see]).sum(1)
        ds = w * ((v[see] * dy[t, :, None]).sum(-1) - (dy[t] * y[t]).sum(-1, keepdim=True)) * c.scale
        dq[t] = (ds[:, :, None] * k[see]).sum(1)
        dk[see] += (ds[:, :, None] * q[t, :, None]).sum(0)
        dv[see] += (w[:, :, None] * dy[t, :, None]).sum(0)
    return y, dq, dk, dv


# (case, sequence of the change, its rows' number in it); head 1, or its key head, is changed
SMALL = (4, 2, 64, 20, 2, [0, 90, 91, 300, 350], None, 0)                      # tiles of 32 keys
WIDE = (3, 1, 256, 70, 1, [0, 150, 310], None, 0)
MANY = (128, 64, 64, 100, 3, [0, 260, 400], None, 0)                           # tiles of 128 keys, blocks that are seen as a whole
LONG = (130, 130, 32, 300, 0, [0, 10, 420], None, 0)
SHAPES = [(SMALL, 91, 300), (SMALL, 90, 91), (WIDE, 0, 150), (MANY, 0, 260), (LONG, 10, 420)]
# tensor, row in the sequence, channel (None: all), value
PLACES = [("q", 40, 5, INF), ("q", 0, None, NAN), ("k", 33, 7, -INF), ("k", 1, 3, INF), ("k", 60, None, NAN), ("v", 50, 9, -INF), ("v", 0, 2, NAN),
          ("dy", 45, 11, INF), ("dy", 100, None, NAN), ("dy", 2, 4, -INF)]


@pytest.mark.parametrize("dtype", [F32, BF16], ids=str)
@pytest.mark.parametrize("shape, lo, hi", SHAPES, ids=["small", "one token", "wide", "many", "long"])
def test_gradients_of_what_sees_it(shape, lo, hi, dtype):
    def build():
        c = Case(dtype, *shape)
        c.q, c.k, c.v = (t.contiguous() for t in (c.q, c.k, c.v))
        c.desc = P.window_attention_desc_for(c.q, c.k, c.v, c.window, c.sinks, c.seqs, c.scale)
        return c, torch.randn(c.tokens, c.h, c.dim, generator=torch.Generator().manual_seed(7)).to(dtype).to(DEV)

    def run(c, dy):
        lse = torch.empty(c.tokens, c.h, device=DEV)
        y = c.run(lse=lse)
        return (y,) + tuple(P.window_attention_backward(dy, c.q, c.k, c.v, y, lse, c.desc, seq_starts=c.sp))

    c, dy = build()
    per, head = c.h // c.kv, 1
    kh = head // per
    clean, plain = run(c, dy), _formula(c, dy, kh, lo, hi)
    for name, row, channel, value in PLACES:
        if row >= hi - lo:
            continue
        c, dy = build()
        t = dict(q=c.q, k=c.k, v=c.v, dy=dy)[name]
        t[lo + row, head if name in ("q", "dy") else kh, slice(None) if channel is None else channel] = value
        got, want = run(c, dy), _formula(c, dy, kh, lo, hi)
        for what, g, before, w, p in zip(("y", "dq", "dk", "dv"), got, clean, want, plain):
            heads = slice(kh * per, kh * per + per) if what in ("y", "dq") else slice(kh, kh + 1)
            mine = torch.zeros(g.shape, dtype=torch.bool)
            mine[lo:hi, heads] = True
            g, before, mine = g.cpu()[:c.starts[-1]], before.cpu()[:c.starts[-1]], mine[:c.starts[-1]]
            assert torch.equal(g[~mine], before[~mine]), (name, row, what, "elsewhere")
            g, before, w, p = (x.reshape(hi - lo, -1) for x in (g[lo:hi, heads], before[lo:hi, heads], w, p))
            assert torch.equal(torch.isfinite(g), torch.isfinite(w)), (name, row, value, what, int((torch.isfinite(g) != torch.isfinite(w)).sum()))
            # what does not see it: the same bits, or computed again, each within rounding of the 64-bit form
            same = w == p
            u = out_round(dtype) + 600 * U32
            size = p.abs().amax(1, keepdim=True)
            assert ((g[same].double() - before[same].double()).abs() <= 8 * u * size.expand_as(p)[same]).all(), (name, row, value, what, "places that do not see it")
            if what == "y":
                assert torch.equal(g[same], before[same]), (name, row, value, what)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=str)
def test_infinite_values_that_all_columns_see(dtype):
    """Blocks of keys that every query of a workgroup sees: an infinity among the
    values is one in the outputs, of its sign, and NaN where both signs meet."""
    c = Case(dtype, 2, 1, 64, 500, 0, [0, 900], None, 0)
    clean = c.run()
    c.v[200, 0, 3], c.v[230, 0, 3], c.v[210, 0, 7], c.v[220, 0, 7], c.v[250, 0, 40] = INF, INF, -INF, INF, NAN
    y = c.run()
    assert (y[200:730, :, 3] == INF).all() and (y[210:220, :, 7] == -INF).all() and torch.isnan(y[220:710, :, 7]).all()
    assert (y[710:720, :, 7] == INF).all() and torch.isnan(y[250:750, :, 40]).all()
    rest = [d for d in range(64) if d not in (3, 7, 40)]
    assert torch.equal(y[:900, :, rest], clean[:900, :, rest]) and torch.equal(y[:200], clean[:200]) and torch.equal(y[750:900], clean[750:900])
    # a prompt that goes on from a cache which holds them
    c = Case(dtype, 2, 1, 64, 300, 2, [0, 90], [400], 0)
    clean = c.run()
    for t, b in zip(c.caches, c.before):
        t.copy_(b)
    s = int(c.slots[0])
    c.caches[1][s, 1, 0, 5], c.caches[1][s, 2 + (390 - 2) % 300, 0, 6] = -INF, INF
    y = c.run()
    assert (y[:90, :, 5] == -INF).all() and (y[:90, :, 6] == INF).all()
    rest = [d for d in range(64) if d not in (5, 6)]
    assert torch.equal(y[:90, :, rest], clean[:90, :, rest])


@pytest.mark.parametrize("window", [90, 3000], ids=["one share", "shares"])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=str)
def test_step_infinite_values(dtype, window):
    g = torch.Generator().manual_seed(window)
    q, k, v = (torch.randn(3, n, 64, generator=g).to(dtype).to(DEV) for n in (4, 2, 2))
    caches = [torch.randn(3, window, 2, 64, generator=g).to(dtype).to(DEV) for _ in range(2)]
    past = torch.tensor([window + 5, 30, window - 1], dtype=torch.int32, device=DEV)
    desc = P.window_attention_desc_for(q, k, v, window)
    clean = P.window_attention_step(q, k, v, *[t.clone() for t in caches], past, desc)
    caches[1][0, 60, 1, 9], caches[1][1, 40, 0, 2], v[2, 0, 63], caches[1][2, 3, 0, 62], caches[1][2, 50, 0, 62] = INF, NAN, -INF, INF, -INF
    y = P.window_attention_step(q, k, v, *caches, past, desc)
    want = clean.clone()
    want[0, 2:, 9], want[2, :2, 63], want[2, :2, 62] = INF, -INF, NAN
    assert torch.equal(torch.nan_to_num(y, nan=77.0), torch.nan_to_num(want, nan=77.0))


@pytest.mark.parametrize("dtype", [F32, BF16], ids=str)
@pytest.mark.parametrize("shape, lo, hi", SHAPES[:1] + SHAPES[2:], ids=["small", "wide", "many", "long"])
def test_lowest_values_in_masked_places(shape, lo, hi, dtype):
    """The type's lowest and largest finite values: what does not see them keeps its bits."""
    def run(change):
        c = Case(dtype, *shape)
        dy = torch.randn(c.tokens, c.h, c.dim, generator=torch.Generator().manual_seed(7)).to(dtype).to(DEV)
        change(c, dy)
        lse = torch.empty(c.tokens, c.h, device=DEV)
        y = c.run(lse=lse)
        return c, (y,) + tuple(P.window_attention_backward(dy, c.q, c.k, c.v, y, lse, c.desc, seq_starts=c.sp))

    low, high = torch.finfo(dtype).min, torch.finfo(dtype).max
    c, clean = run(lambda c, dy: None)
    j = torch.arange(hi - lo)
    see = (j[None] <= j[:, None]) & ((j[None] > j[:, None] - c.window) | (j[None] < c.sinks))      # query, key
    key, query = 40, 60

    def keys(c, dy):
        c.k[lo + key], c.v[lo + key] = low, high

    _, got = run(keys)
    rows = [int(t) for t in j if not see[t, key]]                          # queries that do not see the key,
    others = [int(t) for t in j if not (see[:, t] & see[:, key]).any()]    # keys that no query sees beside it
    assert len(rows) > 20
    assert all(torch.equal(a[lo:hi][rows], b[lo:hi][rows]) for a, b in zip(got[:2], clean[:2]))
    assert all(torch.equal(a[lo:hi][others], b[lo:hi][others]) for a, b in zip(got[2:], clean[2:]))

    def queries(c, dy):
        c.q[lo + query], dy[lo + query] = high, low

    _, got = run(queries)
    rows, others = [int(t) for t in j if t != query], [int(t) for t in j if not see[query, t]]
    assert all(torch.equal(a[lo:hi][rows], b[lo:hi][rows]) for a, b in zip(got[:2], clean[:2]))
    assert len(others) > 20 and all(torch.equal(a[lo:hi][others], b[lo:hi][others]) for a, b in zip(got[2:], clean[2:]))


@pytest.mark.parametrize("dtype", [F32, BF16], ids=str)
def test_step_first_token_of_infinity(dtype):
    """A weight of exactly one."""
    q, k, v = (torch.ones(2, n, 32, device=DEV, dtype=dtype) for n in (2, 1, 1))
    v[0, 0, 3], v[1, 0, 4] = INF, -INF
    caches = [torch.full((2, 9, 1, 32), NAN, device=DEV, dtype=dtype) for _ in range(2)]
    y = P.window_attention_step(q, k, v, *caches, torch.zeros(2, dtype=torch.int32, device=DEV), P.window_attention_desc_for(q, k, v, 9))
    assert torch.equal(y, v.expand_as(y))
