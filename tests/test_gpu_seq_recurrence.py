"""The gated linear recurrence, its gradients and its single-token form on the
GPU against the formulas in 64 bits.  The bounds follow the fp32 errors of each
step along the recurrence (hybrid_reference.recurrence_errors); an output adds
the rounding to its type."""
import pytest
import torch

import paper_2306_14320_amd as P
from hybrid_reference import INPUT_ERROR, decay_error, gates, recurrence, recurrence_errors
from seq_reference import equal_starts, gradients, out_round

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16

# (dtype, channels, starts or (tokens, sequences), states given, spare elements between rows)
CASES = [
    (F32, 1, (1, 1), False, 0), (BF16, 1, (5, 1), True, 1), (BF16, 2, (17, 1), False, 0), (F32, 65, (128, 1), True, 0),
    (BF16, 129, (129, 1), True, 3), (BF16, 300, (256, 4), True, 0), (F32, 70, (384, 3), False, 2),
    (BF16, 131, [0, 0, 1, 5, 130, 130, 131, 300], True, 0),      # empty and one-token sequences
    (F32, 64, [3, 10, 140, 141, 500, 500], True, 1),             # rows outside of the sequences, an empty one at the end
    (F32, 9, (4, 4), True, 0),                                   # sequences of one token
    (BF16, 6, (9000, 1), True, 0),                               # chunks of three groups
    (F32, 3, [0, 4100, 4111, 9003], False, 0),
    (F32, 5, [7, 7, 7], True, 0),                                # rows, but in no sequence
]
IDS = ["%s-d%d-%d" % (str(c[0])[6:], c[1], i) for i, c in enumerate(CASES)]


class Case:
    def __init__(self, dtype, d, rows, states, spare, seed=0, c=8.0):
        g = torch.Generator().manual_seed(seed + 100 * d)
        if isinstance(rows, tuple):
            self.tokens, self.seqs = rows
            self.starts, dense = equal_starts(*rows), True
        else:
            self.starts, dense = rows, False
            self.tokens, self.seqs = rows[-1] + 3, len(rows) - 1
        self.dtype, self.d, self.c, t = dtype, d, c, self.tokens
        outside = [k for k in range(t) if not self.starts[0] <= k < self.starts[-1]]

        def normal(*shape, dtype=dtype):
            return torch.randn(shape, generator=g, dtype=torch.float64).to(dtype)

        wide = [normal(t, d + spare) for _ in range(3)]
        dy = normal(t, d)
        for v in wide + [dy]:
            v[outside] = float("nan")
        self.lam = 2 * normal(d, dtype=F32) - 3
        self.init = normal(self.seqs, d, dtype=F32) if states else None
        self.d_final = normal(self.seqs, d, dtype=F32) if states else None
        self.x, self.r, self.i = (v.to(DEV)[:, spare:] for v in wide)
        self.dy = dy.to(DEV)
        self.sp = None if dense else torch.tensor(self.starts, dtype=torch.int32, device=DEV)
        self.desc = P.gated_recurrence_desc_for(self.x, self.r, self.i, self.seqs, c)

        def clean(v):
            v = v.double().cpu()
            v[outside] = 0
            return v

        self.cpu = [clean(v) for v in (self.x, self.r, self.i)] + [self.lam.double()]
        self.cpu_dy, self.cpu_init = clean(dy), None if self.init is None else self.init.double()
        self.live = [k for k in range(t) if self.starts[0] <= k < self.starts[-1]]

    def dev(self, v):
        return None if v is None else v.to(DEV)

    def forward(self, **kw):
        return P.gated_recurrence(self.x, self.r, self.i, self.dev(self.lam), self.desc, seq_starts=self.sp, initial_state=self.dev(self.init), **kw)

    def backward(self, **kw):
        return P.gated_recurrence_backward(self.dy, self.x, self.r, self.i, self.dev(self.lam), self.desc, seq_starts=self.sp,
                                           initial_state=self.dev(self.init), d_final_state=self.dev(self.d_final), **kw)


def _within(got, ref, bound, what):
    err = (got.double().cpu() - ref).abs()
    assert (err <= bound + 1e-30).all(), (what, float((err - bound).max()))


@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_forward(case):
    k = Case(*case)
    final = torch.full((k.seqs, k.d), float("nan"), device=DEV)
    y = torch.full((k.tokens * k.d + 512,), -7.0, dtype=k.dtype, device=DEV)
    k.forward(y=y[:k.tokens * k.d].view(k.tokens, k.d), final_state=final)
    torch.cuda.synchronize()
    rows = y[:k.tokens * k.d].view(k.tokens, k.d).cpu()
    outside = [t for t in range(k.tokens) if t not in set(k.live)]
    assert (y[k.tokens * k.d:] == -7).all() and (rows[outside] == -7).all(), "wrote outside of the sequences"
    ref, ref_final = recurrence(*k.cpu, k.c, k.starts, k.cpu_init)
    e = recurrence_errors(*k.cpu, k.c, k.starts, k.cpu_init)
    _within(rows[k.live], ref[k.live], (e["y"] + out_round(k.dtype) * (ref.abs() + e["y"]))[k.live], "y")
    _within(final, ref_final, e["final"], "final")
    again = k.forward(final_state=torch.empty_like(final))
    assert torch.equal(again[k.live], y[:k.tokens * k.d].view(k.tokens, k.d)[k.live]), "two calls differ"


@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_backward(case):
    k = Case(*case)
    kept = P.gated_recurrence_chunk_states(k.x, k.desc)
    k.forward(chunk_states=kept)
    got, again = k.backward(), k.backward(chunk_states=kept)
    for a, b in zip(got, again):
        assert (a is None and b is None) or torch.equal(a[k.live] if a.shape == k.x.shape else a, b[k.live] if b.shape == k.x.shape else b), "kept states give another result"
    dfin = None if k.d_final is None else k.d_final.double()
    ref = gradients(lambda x, r, i, lam, init: recurrence(x, r, i, lam, k.c, k.starts, init), k.cpu + [k.cpu_init], [k.cpu_dy, dfin])
    e = recurrence_errors(*k.cpu, k.c, k.starts, k.cpu_init, k.cpu_dy, dfin)
    for name, a, b in zip(("dx", "dr", "di"), got, ref):
        b = torch.zeros_like(k.cpu[0]) if b is None else b
        _within(a[k.live], b[k.live], (e[name] + out_round(k.dtype) * (b.abs() + e[name]))[k.live], name)
    _within(got.dlam, torch.zeros_like(k.cpu[3]) if ref[3] is None else ref[3], e["dlam"], "dlam")
    if k.init is not None:
        _within(got.d_initial_state, ref[4], e["d_init"], "d_init")


def test_gradient_against_differences():
    """Central differences of the 64-bit form with step 1e-5 are off by about
    1e-10 of the terms' size; the fp32 gradients by under 300 roundings."""
    k = Case(F32, 33, [0, 140, 141, 300], True, 0)
    g = torch.Generator().manual_seed(4)
    way = [torch.randn(v.shape, generator=g, dtype=torch.float64) for v in k.cpu + [k.cpu_init]]
    way[0][k.tokens - 3:] = way[1][k.tokens - 3:] = way[2][k.tokens - 3:] = 0

    def value(s):
        y, final = recurrence(*[v + s * w for v, w in zip(k.cpu, way)], k.c, k.starts, k.cpu_init + s * way[4])
        return (y * k.cpu_dy).sum() + (final * k.d_final.double()).sum()

    got = k.backward()
    terms = [torch.where(w != 0, a.double().cpu() * w, 0.0) for a, w in zip(got, way)]
    assert abs((value(1e-5) - value(-1e-5)) / 2e-5 - sum(v.sum() for v in terms)) <= 2e-5 * sum(v.abs().sum() for v in terms)


@pytest.mark.parametrize("lam,r", [(-200.0, 0.0), (-40.0, 3.0), (60.0, 5.0), (3.0, -90.0), (0.0, -200.0)], ids=str)
def test_gates_at_their_ends(lam, r):
    """Decays that are one in fp32 (the input's part then goes to zero with
    them) and decays that are zero: values and gradients stay finite and right."""
    k = Case(F32, 4, (40, 1), True, 0)
    k.lam = torch.full_like(k.lam, lam)
    k.r.fill_(r)
    k.cpu[1], k.cpu[3] = torch.full_like(k.cpu[1], r), k.lam.double()
    y = k.forward()
    ref, _ = recurrence(*k.cpu, k.c, k.starts, k.cpu_init)
    e = recurrence_errors(*k.cpu, k.c, k.starts, k.cpu_init, k.cpu_dy, k.d_final.double())
    # below 2^-126 a root's argument keeps fewer digits: its root is under 2^-63
    tiny = 2.0 ** -60
    _within(y, ref, e["y"] + out_round(F32) * ref.abs() + 40 * tiny, "y")
    got = k.backward()
    want = gradients(lambda x, rr, i, lm, init: recurrence(x, rr, i, lm, k.c, k.starts, init), k.cpu + [k.cpu_init], [k.cpu_dy, k.d_final.double()])
    for name, a, b in zip(("dx", "dr", "di", "dlam", "d_init"), got, want):
        assert torch.isfinite(a).all(), name
        b = torch.where(torch.isfinite(b), b, 0.0)      # the formula's own quotient of zeros
        _within(a, b, torch.where(torch.isfinite(e[name]), e[name], 0.0) + out_round(F32) * b.abs() + 400 * tiny, name)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=str)
def test_nan_stays_in_its_sequence(dtype):
    k = Case(dtype, 70, [0, 100, 300, 420], True, 0)
    clean_y, clean = k.forward(), k.backward()
    k.x[150] = float("nan")
    k.r[160, 3] = float("inf")
    k.i[170] = float("-inf")
    k.dy[180] = float("inf")
    final = torch.empty(3, 70, device=DEV)
    y, g = k.forward(final_state=final), k.backward()
    assert torch.isnan(y[150:300]).all() and torch.isnan(final[1]).all()
    for rows in (slice(0, 100), slice(300, 420)):
        assert torch.equal(y[rows], clean_y[rows])
        assert all(torch.equal(a[rows], b[rows]) for a, b in zip(g[:3], clean[:3]))
    assert torch.equal(y[100:150], clean_y[100:150]), "a row behind changed the rows before it"
    assert all(torch.equal(g[4][q], clean[4][q]) for q in (0, 2))


@pytest.mark.parametrize("dtype,d", [(F32, 1), (BF16, 1), (BF16, 777), (F32, 300), (BF16, 2048)], ids=str)
def test_step(dtype, d):
    n, pool = 9, 12
    g = torch.Generator().manual_seed(d)
    gates_ = torch.randn(n, 2 * d + 1, generator=g).to(dtype).to(DEV)
    x, r, i = torch.randn(n, d, generator=g).to(dtype).to(DEV), gates_[:, :d], gates_[:, d + 1:]
    lam = (torch.randn(d, generator=g) - 3).to(DEV)
    state = torch.randn(pool, d, generator=g).to(DEV)
    slots = torch.tensor([4, 11, -1, 0, 7, 12, 2, 3, 1 << 30], dtype=torch.int32, device=DEV)
    before = state.clone()
    y = P.gated_recurrence_step(x, r, i, lam, state, P.gated_recurrence_desc_for(x, r, i), slots=slots)
    log_a, a, m, sx = gates(x.double().cpu(), r.double().cpu(), i.double().cpu(), lam.double().cpu(), 8.0)
    moved = set()
    for q, s in enumerate(slots.tolist()):
        if not 0 <= s < pool:
            assert (y[q] == 0).all()
            continue
        moved.add(s)
        h0 = before[s].double().cpu()
        h = a[q] * h0 + m[q] * sx[q]
        e = decay_error(log_a[q]) * (a[q] * h0).abs() + INPUT_ERROR * (m[q] * sx[q]).abs() + 2.0 ** -24 * h.abs()
        _within(state[s], h, e, "state")
        _within(y[q], h, e + out_round(dtype) * (h.abs() + e), "y")
    assert all(torch.equal(state[s], before[s]) for s in range(pool) if s not in moved)


def test_steps_go_on_from_a_prompt():
    """A prompt in two parts and single tokens give what one call over all rows gives."""
    k = Case(F32, 96, (260, 1), False, 0)
    lam = k.dev(k.lam)
    whole = k.forward()

    def part(lo, hi, init, final):
        x, r, i = k.x[lo:hi], k.r[lo:hi], k.i[lo:hi]
        return P.gated_recurrence(x, r, i, lam, P.gated_recurrence_desc_for(x, r, i), initial_state=init, final_state=final)

    s1, s2 = torch.empty(1, 96, device=DEV), torch.empty(1, 96, device=DEV)
    got = [part(0, 131, None, s1), part(131, 257, s1, s2)]
    for t in range(257, 260):
        x, r, i = k.x[t:t + 1], k.r[t:t + 1], k.i[t:t + 1]
        got.append(P.gated_recurrence_step(x, r, i, lam, s2, P.gated_recurrence_desc_for(x, r, i)))
    e = recurrence_errors(*k.cpu, k.c, k.starts, None)["y"]
    _within(torch.cat(got), whole.double().cpu(), 2 * e + 2.0 ** -23 * whole.double().cpu().abs(), "parts")


def test_zero_tokens_stream_and_graph():
    none = torch.empty(0, 8, device=DEV)
    desc = P.gated_recurrence_desc_for(none, none, none, sequences=2)
    lam, init, final = torch.zeros(8, device=DEV), torch.randn(2, 8, device=DEV), torch.empty(2, 8, device=DEV)
    assert P.gated_recurrence(none, none, none, lam, desc, initial_state=init, final_state=final).shape == (0, 8)
    assert torch.equal(final, init)
    g = P.gated_recurrence_backward(none, none, none, none, lam, desc, initial_state=init, d_final_state=init)
    assert torch.equal(g.d_initial_state, init) and (g.dlam == 0).all()
    k = Case(BF16, 200, [0, 5, 300, 700], True, 0)
    want = k.forward()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = k.forward(stream=side)
    side.synchronize()
    assert torch.equal(got[:700], want[:700])
    lam, init, d_final = k.dev(k.lam), k.dev(k.init), k.dev(k.d_final)
    x, r, i, dy = (v[:700].contiguous() for v in (k.x, k.r, k.i, k.dy))
    desc = P.gated_recurrence_desc_for(x, r, i, k.seqs)

    def both():
        y = P.gated_recurrence(x, r, i, lam, desc, seq_starts=k.sp, initial_state=init)
        return (y,) + tuple(P.gated_recurrence_backward(dy, x, r, i, lam, desc, seq_starts=k.sp, initial_state=init, d_final_state=d_final))

    both()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = both()
    for n in range(4):
        x.copy_(torch.randn_like(x))
        k.sp.copy_(torch.tensor([0, 100 + n, 300, 700]))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(captured, both())), n
