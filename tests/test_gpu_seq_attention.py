"""Window attention and its single-token form on the GPU against the softmax
in 64 bits.  A score is a sum of D products, off by (D + 8) u sum |q k| scale
(u = 2^-24); the weights carry that twice, and are rounded to 2^-8 where the
values are bfloat16; the sums over n keys add n u (hybrid_reference.attend)."""
import pytest
import torch

import paper_2306_14320_amd as P
from hybrid_reference import attend, ring_row
from seq_reference import U16, equal_starts, out_round

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16

# (dtype, heads, key heads, head size, window, sinks, starts or (tokens, sequences), past or None (no cache), spare)
CASES = [
    (F32, 1, 1, 8, 1, 0, (1, 1), None, 0), (BF16, 2, 1, 16, 1, 1, (5, 1), None, 8), (BF16, 4, 4, 64, 7, 0, (70, 2), None, 0),
    (F32, 6, 2, 40, 33, 2, (150, 1), None, 1), (BF16, 8, 2, 128, 100, 4, (333, 1), None, 0), (BF16, 3, 1, 80, 50, 3, (257, 1), None, 5),
    (F32, 5, 5, 96, 64, 0, (130, 1), None, 0), (BF16, 16, 1, 256, 40, 32, (90, 1), None, 0), (F32, 2, 1, 256, 30, 1, (77, 1), None, 0),
    (F32, 4, 2, 192, 65, 5, (140, 1), None, 0), (BF16, 2, 2, 184, 128, 8, (200, 1), None, 0), (BF16, 34, 1, 32, 20, 2, (60, 1), None, 0),
    (BF16, 37, 1, 32, 20, 2, (40, 1), None, 0),                                                    # a group of a prime number of heads
    (BF16, 4, 2, 64, 1000, 4, [0, 0, 1, 5, 130, 130, 131, 400], None, 0),                          # empty and one-token sequences
    (F32, 3, 3, 32, 16, 3, [4, 10, 140, 141, 200, 200], None, 3),                                  # rows outside of the sequences
    (BF16, 4, 1, 128, 64, 4, [0, 100, 101, 101, 300], [0, 64, 9, 1000], 0),                        # prompts that go on from a cache
    (F32, 2, 2, 24, 10, 3, [0, 1, 3, 40, 41], [2, 500, 12, 13], 1), (BF16, 6, 2, 96, 33, 0, [0, 200, 201, 260], [31, 33, 1], 0),
    (F32, 8, 4, 64, 1, 2, [0, 4, 9], [0, 7], 0), (BF16, 2, 1, 72, 300, 1, [2, 90, 400], [299, 0], 2), (F32, 1, 1, 16, 5, 0, (40, 8), [3, 0, 5, 4, 6, 7, 100, 1], 0),
    (BF16, 2, 1, 16, 8, 4, (64, 4), [1 << 30, (1 << 30) - 9, 2, 3], 0),                            # far positions
    (F32, 1, 1, 8, 4, 0, (700, 700), None, 0), (BF16, 2, 1, 8, 4, 2, list(range(0, 301)), None, 0),      # many sequences of one token
]
IDS = ["%s-%dq%dk%d-w%d-s%d-%d" % ((str(c[0])[6:],) + c[1:6] + (i,)) for i, c in enumerate(CASES)]


class Case:
    def __init__(self, dtype, h, kv, dim, window, sinks, rows, past, spare, seed=0):
        g = torch.Generator().manual_seed(seed + dim + window)
        if isinstance(rows, tuple):
            self.tokens, self.seqs = rows
            self.starts, dense = equal_starts(*rows), True
        else:
            self.starts, dense = rows, False
            self.tokens, self.seqs = rows[-1] + 3, len(rows) - 1
        self.dtype, self.h, self.kv, self.dim, self.window, self.sinks, self.scale, t = dtype, h, kv, dim, window, sinks, 1.3 * dim ** -0.5, self.tokens

        def normal(*shape):
            return torch.randn(shape, generator=g, dtype=torch.float64).to(dtype)

        wide = normal(t, (h + 2 * kv) * dim + spare)
        self.live = [i for i in range(t) if self.starts[0] <= i < self.starts[-1]]
        wide[[i for i in range(t) if i not in set(self.live)]] = float("nan")
        wide = wide.to(DEV)
        self.q, self.k, self.v = (p.unflatten(1, (-1, dim)) for p in wide[:, spare:].split([h * dim, kv * dim, kv * dim], 1))
        self.sp = None if dense else torch.tensor(self.starts, dtype=torch.int32, device=DEV)
        self.desc = P.window_attention_desc_for(self.q, self.k, self.v, window, sinks, self.seqs, self.scale)
        self.past_list, self.kw = past or [0] * self.seqs, {}
        if past is not None:
            pool = self.seqs + 2
            self.slots = torch.randperm(pool, generator=g)[:self.seqs].to(torch.int32)
            self.caches = []
            for _ in range(2):
                c = normal(pool, sinks + window, kv, dim)
                for b, p in enumerate(past):        # rows that the request has not filled hold anything
                    c[self.slots[b], p:] = float("nan")
                self.caches.append(c.to(DEV))
            self.kw = dict(k_cache=self.caches[0], v_cache=self.caches[1], past=torch.tensor(past, dtype=torch.int32, device=DEV), slots=self.slots.to(DEV))
        self.before = [c.clone() for c in getattr(self, "caches", [])]

    def rows_of(self, b, which):
        """The sequence's known keys or values by position from max(0, past - window), sinks in front: values, first position."""
        lo, hi = self.starts[b:b + 2]
        new = (self.k, self.v)[which][lo:hi].double().cpu()
        past = self.past_list[b]
        if not past:
            return new, new.new_zeros(0, self.kv, self.dim), 0
        cache = self.before[which][self.slots[b]].double().cpu()
        first = max(0, past - self.window)
        old = torch.stack([cache[ring_row(p, self.window, self.sinks)] for p in range(first, past)])
        sinks = cache[:min(self.sinks, first)]
        return torch.cat((old, new)), sinks, first

    def reference(self, b, head):
        """y, lse, bound and lse's bound of a head of a sequence: positions are moved down
        behind the sinks so that forgotten ones take no room."""
        lo, hi = self.starts[b:b + 2]
        k, ks, first = self.rows_of(b, 0)
        v, vs, _ = self.rows_of(b, 1)
        n = ks.shape[0]
        kh = head // (self.h // self.kv)
        q = self.q[lo:hi, head].double().cpu()
        # with the forgotten positions left out, sinks in front of the window's first key stay in front
        gap = first - n
        return attend(q, torch.cat((ks, k))[:, kh], torch.cat((vs, v))[:, kh], self.past_list[b] - gap, self.window, self.sinks, self.scale)

    def run(self, **kw):
        return P.window_attention(self.q, self.k, self.v, self.desc, seq_starts=self.sp, **self.kw, **kw)


def _within(got, ref, bound, what):
    err = (got.double().cpu() - ref).abs()
    assert (err <= bound + 1e-30).all(), (what, float((err - bound).max()))


@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_forward(case):
    c = Case(*case)
    n = c.tokens * c.h * c.dim
    buf = torch.full((n + 512,), -5.0, dtype=c.dtype, device=DEV)
    y = buf[:n].view(c.tokens, c.h, c.dim)
    lse = torch.full((c.tokens, c.h), -5.0, device=DEV)
    c.run(y=y, lse=lse)
    torch.cuda.synchronize()
    outside = [i for i in range(c.tokens) if i not in set(c.live)]
    assert (buf[n:] == -5).all() and (y[outside] == -5).all() and (lse[outside] == -5).all(), "wrote outside of the sequences"
    u = U16 if c.dtype == BF16 else 0.0
    for b, (lo, hi) in enumerate(zip(c.starts, c.starts[1:])):
        for head in range(c.h if hi > lo else 0):
            ref, ref_lse, bound, lse_bound = c.reference(b, head)
            e = bound(u)
            _within(y[lo:hi, head], ref, e + out_round(c.dtype) * (ref.abs() + e), ("y", b, head))
            _within(lse[lo:hi, head], ref_lse, lse_bound, ("lse", b, head))
    # the caches behind the call
    for which, new in enumerate((c.k, c.v)):
        if not c.before:
            break
        want = c.before[which].clone()
        for b, (lo, hi) in enumerate(zip(c.starts, c.starts[1:])):
            end = c.past_list[b] + hi - lo
            for p in range(c.past_list[b], end):
                if p < c.sinks or p >= end - c.window:
                    want[c.slots[b], ring_row(p, c.window, c.sinks)] = new[lo + p - c.past_list[b]]
        assert torch.equal(torch.nan_to_num(c.caches[which], 77.0), torch.nan_to_num(want, 77.0)), "cache"
        c.caches[which].copy_(c.before[which])
    again = c.run()
    assert torch.equal(again[c.live], y[c.live]), "two calls differ"


@pytest.mark.parametrize("dtype", [F32, BF16], ids=str)
def test_masked_places_do_not_enter(dtype):
    """Infinities and NaN behind a query, in front of its window and in other
    sequences change nothing; a query that sees them has them."""
    c = Case(dtype, 4, 2, 64, 20, 2, [0, 90, 91, 300, 350], None, 0)
    clean = c.run()
    bad = 150                                # position 59 of its sequence
    c.k[bad], c.v[bad] = float("nan"), float("inf")
    y = c.run()
    hit = set(range(bad, bad + 20))
    keep = [i for i in range(350) if i not in hit]
    assert torch.equal(y[keep], clean[keep])
    assert torch.isnan(y[sorted(hit)]).all()
    c = Case(dtype, 4, 2, 64, 20, 2, [0, 90, 91, 300, 350], None, 0)
    c.v[bad, 1, 3], c.v[bad, 0] = float("-inf"), float("nan")
    y = c.run()
    assert torch.equal(y[keep], clean[keep])
    rows = y[sorted(hit)].float()
    assert torch.isnan(rows[:, :2]).all() and (rows[:, 2:, 3] == -float("inf")).all() and torch.isfinite(rows[:, 2:, :3]).all()
    c = Case(dtype, 4, 2, 64, 20, 2, [0, 90, 91, 300, 350], None, 0)
    c.v[92, 0] = float("inf")                # a first token: all behind it see it
    y = c.run()
    assert (y[92:300, :2].float() == float("inf")).all() and torch.equal(y[:92], clean[:92]) and torch.equal(y[300:350], clean[300:350])


def test_requests_without_a_slot():
    c = Case(BF16, 4, 2, 64, 30, 2, [0, 50, 80, 130], [5, 100, 0], 0)
    c.kw["slots"] = torch.tensor([-1, int(c.slots[1]), 99], dtype=torch.int32, device=DEV)
    lse = torch.zeros(c.tokens, 4, device=DEV)
    y = c.run(lse=lse)
    assert (y[:50] == 0).all() and (y[80:130] == 0).all() and (lse[:50] == -float("inf")).all()
    ref, _, bound, _ = c.reference(1, 3)
    e = bound(U16)
    _within(y[50:80, 3], ref, e + U16 * (ref.abs() + e), "y")
    other = [s for s in range(5) if s != int(c.slots[1])]
    assert all(torch.equal(torch.nan_to_num(a[other], 77.0), torch.nan_to_num(b[other], 77.0)) for a, b in zip(c.caches, c.before))


# (dtype, heads, key heads, head size, window, sinks, past of each request)
STEPS = [
    (F32, 1, 1, 8, 1, 0, [0, 5]), (BF16, 4, 1, 128, 100, 4, [0, 1, 3, 4, 50, 103, 104, 105, 5000]), (F32, 6, 2, 40, 33, 2, [0, 34, 35, 1 << 30]),
    (BF16, 3, 3, 256, 200, 1, [199, 200, 201, 777]), (F32, 8, 2, 192, 70, 0, [69, 70, 3]), (BF16, 34, 1, 64, 64, 32, [31, 32, 95, 96, 1000]),
    (BF16, 8, 1, 128, 3000, 4, [2999, 100000]), (F32, 2, 1, 256, 1000, 3, [999, 5]), (BF16, 16, 4, 80, 500, 4, list(range(480, 520))),
    (BF16, 5, 5, 96, 1, 3, [0, 2, 3, 9]), (F32, 64, 8, 32, 129, 0, [128] * 70), (BF16, 2, 1, 192, 40, 0, [400, 39]),
]


@pytest.mark.parametrize("case", STEPS, ids=["%s-%dq%dk%d-w%d-s%d-n%d" % ((str(c[0])[6:],) + c[1:6] + (len(c[6]),)) for c in STEPS])
def test_step(case):
    dtype, h, kv, dim, window, sinks, past = case
    n, pool = len(past), len(past) + 2
    g = torch.Generator().manual_seed(dim + window)
    wide = torch.randn(n, (h + 2 * kv) * dim + 1, generator=g).to(dtype).to(DEV)[:, 1:]
    q, k, v = (p.unflatten(1, (-1, dim)) for p in wide.split([h * dim, kv * dim, kv * dim], 1))
    slots = torch.randperm(pool, generator=g)[:n].to(torch.int32)
    slots[n // 2] = pool if n > 2 else slots[n // 2]
    caches = [torch.randn(pool, sinks + window, kv, dim, generator=g).to(dtype) for _ in range(2)]
    for c in caches:
        for b, p in enumerate(past):
            if slots[b] < pool:
                c[slots[b], p:] = float("nan")
    before = [c.clone() for c in caches]
    caches = [c.to(DEV) for c in caches]
    scale = 1.1 * dim ** -0.5
    desc = P.window_attention_desc_for(q, k, v, window, sinks, scale=scale)
    pt = torch.tensor(past, dtype=torch.int32, device=DEV)
    y = P.window_attention_step(q, k, v, *caches, pt, desc, slots=slots.to(DEV))
    u = U16 if dtype == BF16 else 0.0
    for b, p in enumerate(past):
        s = int(slots[b])
        if s >= pool:
            assert (y[b] == 0).all()
            continue
        for c, new in zip(before, (k, v)):
            c[s, ring_row(p, window, sinks)] = new[b].cpu()
        rows = min(p + 1, sinks + window)
        for head in range(h):
            kk, vv = (c[s, :rows, head // (h // kv)].double() for c in before)
            ref, _, bound, _ = attend(q[b:b + 1, head].double().cpu(), kk, vv, rows - 1, rows, 0, scale)
            e = bound(u)
            _within(y[b:b + 1, head], ref, e + out_round(dtype) * (ref.abs() + e), ("y", b, head))
    for got, want in zip(caches, before):
        assert torch.equal(torch.nan_to_num(got.cpu(), 77.0), torch.nan_to_num(want, 77.0)), "cache"
    again = [c.clone() for c in caches]
    assert torch.equal(P.window_attention_step(q, k, v, *again, pt, desc, slots=slots.to(DEV)), y), "two calls differ"


def test_steps_go_on_from_a_prompt():
    """A prompt in two parts and single tokens against one call over all rows."""
    dtype, h, kv, dim, window, sinks, n = F32, 4, 2, 64, 37, 3, 210
    g = torch.Generator().manual_seed(5)
    q, k, v = (torch.randn(n, m, dim, generator=g).to(DEV) for m in (h, kv, kv))
    whole = P.window_attention(q, k, v, P.window_attention_desc_for(q, k, v, window, sinks))
    caches = [torch.full((1, window + sinks, kv, dim), float("nan"), device=DEV) for _ in range(2)]
    got = []
    for lo, hi in ((0, 2), (2, 150)):
        part = q[lo:hi], k[lo:hi], v[lo:hi]
        past = torch.tensor([lo], dtype=torch.int32, device=DEV)
        got.append(P.window_attention(*part, P.window_attention_desc_for(*part, window, sinks), k_cache=caches[0], v_cache=caches[1], past=past))
    for t in range(150, n):
        part = q[t:t + 1], k[t:t + 1], v[t:t + 1]
        got.append(P.window_attention_step(*part, *caches, past + (t - 2), P.window_attention_desc_for(*part, window, sinks)))
    got = torch.cat(got).double().cpu()
    for head in range(h):
        ref, _, bound, _ = attend(q[:, head].double().cpu(), k[:, head // 2].double().cpu(), v[:, head // 2].double().cpu(), 0, window, sinks, dim ** -0.5)
        _within(got[:, head], ref, bound(0.0) + out_round(F32) * ref.abs(), "parts")
        _within(whole[:, head], ref, bound(0.0) + out_round(F32) * ref.abs(), "whole")


def test_zero_tokens_stream_and_graph():
    none = torch.empty(0, 2, 16, device=DEV)
    assert P.window_attention(none, none, none, P.window_attention_desc_for(none, none, none, 4)).shape == (0, 2, 16)
    c = Case(BF16, 8, 2, 64, 40, 4, [0, 30, 31, 200], [0, 50, 7], 0)
    want = c.run()
    for a, b in zip(c.caches, c.before):
        a.copy_(b)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = c.run(stream=side)
    side.synchronize()
    assert torch.equal(got[:200], want[:200])
    n, h, kv, dim, w = 3, 8, 1, 64, 3000
    q, k, v = (torch.randn(n, m, dim, device=DEV).to(BF16) for m in (h, kv, kv))
    kc, vc = (torch.randn(n, w, kv, dim, device=DEV).to(BF16) for _ in range(2))
    past = torch.tensor([0, 2998, 3005], dtype=torch.int32, device=DEV)
    desc = P.window_attention_desc_for(q, k, v, w)
    assert P.im2win_window_attention_step_workspace_bytes(desc) > 0
    P.window_attention_step(q, k, v, kc.clone(), vc.clone(), past, desc)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = P.window_attention_step(q, k, v, kc, vc, past, desc)
        past.add_(1)
    for i in range(4):
        k.copy_(torch.randn_like(k))
        k2, v2, p2 = kc.clone(), vc.clone(), past.clone()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, P.window_attention_step(q, k, v, k2, v2, p2, desc)), i
        assert torch.equal(kc, k2) and torch.equal(vc, v2) and torch.equal(past, p2 + 1)
