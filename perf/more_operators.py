"""The performance cases of the operators of hybrid sequence layers: the gated
linear recurrence, the norm of queries and keys for each head with the position
rotation, and attention with a sliding window and a few first tokens that stay
visible, for training, prompts and single tokens.

Tokens are rows: a tensor of T tokens is T x D (or T x heads x head size), and
sequence b holds the rows seq_starts[b] to seq_starts[b+1].  Op names:

- "rec", "rec_train", "rec_step": with L = -c softplus(lam) sigmoid(r) and
  a = exp(L), h_t = a h_{t-1} + sqrt(1 - a^2) sigmoid(i_t) x_t; the same with
  its gradients behind it; one token of each of many requests;
- "qk", "qk_bwd": y = rotated(x / rms(x) * w) of every head's x, and gradients;
- "att", "att_train", "att_step": softmax(scale q k) v over the keys j <= t
  with j > t - W or j < S; "att" continues requests whose last W and first S
  keys and values lie in a cache and leaves the cache behind the new tokens,
  "att_train" has the gradients behind it, "att_step" is one token of each.

The cache of a request has S + W rows: position p lies in row p where p < S
and in row S + (p - S) mod W otherwise.

Where ``own`` is false, ``run`` computes them with elementary torch operations
in 32 bits; where it is true, with the framework's kernels.
"""
import math
import random

import torch

own = False

_DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-6
C = 8.0


def listed():
    return [
        # one new token of 16 requests whose states lie in a pool of slots
        dict(name="rec_step_16", op="rec_step", dtype="bf16", seqs=16, d=2048),
        # one long prompt: few rows of channels, so the time axis has to be split
        dict(name="rec_prompt_8192_bf16", op="rec", dtype="bf16", tokens=8192, seqs=1, ragged=False, d=2048, states=True),
        # prompts of many lengths, one empty and one of one token, that go on from kept states; odd sizes
        dict(name="rec_prompts_f32_odd", op="rec", dtype="f32", tokens=3001, seqs=17, ragged=True, d=777, states=True),
        # a training step's forward and backward pass over a batch of sequences
        dict(name="rec_train_bf16", op="rec_train", dtype="bf16", tokens=16384, seqs=8, ragged=False, d=4096, states=False),
        # the queries and keys of one new token of 64 requests, far into their texts
        dict(name="qk_step_64", op="qk", dtype="bf16", tokens=64, heads=16, kv=4, dim=128, rot=128, interleaved=False, far=True),
        # a batch of prompts' queries and keys
        dict(name="qk_prompts_bf16", op="qk", dtype="bf16", tokens=16384, heads=16, kv=4, dim=128, rot=128, interleaved=False, far=False),
        # gradients, odd sizes, half of each head rotated, neighbours as pairs
        dict(name="qk_bwd_f32_odd", op="qk_bwd", dtype="f32", tokens=4001, heads=10, kv=5, dim=80, rot=40, interleaved=True, far=False),
        # one new token of 128 requests with windows of 1024
        dict(name="att_step_128", op="att_step", dtype="bf16", seqs=128, heads=16, kv=4, dim=128, window=1024, sinks=4),
        # one new token of two requests with long windows: the keys have to be split
        dict(name="att_step_2_long", op="att_step", dtype="bf16", seqs=2, heads=8, kv=1, dim=128, window=4096, sinks=4),
        # prompts of many lengths, some of which go on from a cache; narrow heads and windows
        dict(name="att_prompts_bf16_odd", op="att", dtype="bf16", tokens=9001, seqs=13, ragged=True, heads=12, kv=4, dim=64, window=500, sinks=3),
        # a training step's forward and backward pass over a batch of sequences
        dict(name="att_train_bf16", op="att_train", dtype="bf16", tokens=16384, seqs=4, ragged=False, heads=16, kv=4, dim=128, window=1024, sinks=4),
        # ragged training sequences in 32 bits, a head size between powers of two, a group of three heads
        dict(name="att_train_f32_odd", op="att_train", dtype="f32", tokens=2503, seqs=5, ragged=True, heads=6, kv=2, dim=96, window=201, sinks=1),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """A case of the listed ones' ranges: 1 to 16384 tokens in up to 64
    sequences or 1 to 256 requests, 64 to 4096 channels, heads of 32 to 256 in
    up to 8 groups of up to 8, windows of 16 to 4096 tokens, up to 16 tokens
    that stay visible, and no more work than the largest listed case of the
    op's kind."""
    while True:
        op = rng.choice(["rec", "rec_train", "rec_step", "qk", "qk_bwd", "att", "att", "att_train", "att_train", "att_step", "att_step"])
        c = {"op": op, "dtype": rng.choice(["f32", "bf16", "bf16"])}
        tokens = _log_int(rng, 1, 16384)
        if op.endswith("_step"):
            c["seqs"] = _log_int(rng, 1, 256)
        elif not op.startswith("qk"):
            seqs = min(tokens, _log_int(rng, 1, 64))
            ragged = rng.random() < 0.5
            c.update(tokens=tokens if ragged else tokens // seqs * seqs, seqs=seqs, ragged=ragged)
        if op.startswith("rec"):
            d = _log_int(rng, 64, 4096)
            c["d"] = d // 64 * 64 if rng.random() < 0.5 else d
            if op != "rec_step":
                c["states"] = rng.random() < 0.5
            return c
        kv, group = rng.choice([1, 2, 3, 4, 8]), rng.choice([1, 2, 3, 4, 5, 8])
        c.update(heads=kv * group, kv=kv, dim=rng.choice([32, 64, 64, 80, 96, 128, 128, 128, 192, 256]))
        if op.startswith("qk"):
            c.update(tokens=tokens, rot=rng.choice([c["dim"], c["dim"], c["dim"] // 2]), interleaved=rng.random() < 0.3, far=rng.random() < 0.3)
            if tokens * (kv + c["heads"]) * c["dim"] <= 16384 * 20 * 128:
                return c
            continue
        c.update(window=_log_int(rng, 16, 4096), sinks=rng.choice([0, 1, 4, 16]))
        w = work(c)
        if w["flops"] * (8 if c["dtype"] == "f32" else 1) <= _largest_attention() and w["bytes"] <= 2 ** 30:
            return c


def _largest_attention():
    return work(next(c for c in listed() if c["name"] == "att_train_bf16"))["flops"]


def _lengths(c):
    """The sequences' first rows, from the case's sizes alone: equal ones, or
    cuts at random rows, one sequence empty and one of one token if they fit."""
    t, b = c["tokens"], c["seqs"]
    if not c["ragged"]:
        return [i * (t // b) for i in range(b + 1)]
    r = random.Random(1000003 * t + b)
    cuts = [r.randint(0, t) for _ in range(b - 1)]
    if b >= 4:
        cuts[1] = cuts[0]
        cuts[2] = min(t, cuts[0] + 1)
    return [0] + sorted(cuts) + [t]


def _past(c):
    """The tokens that each request has seen before the call: none, one, fewer
    than its window and many more, a third of the prompts new ones."""
    if c["op"] == "att_train":
        return [0] * c["seqs"]
    r = random.Random(7 * c["seqs"] + c["window"])
    n = [r.randint(c["window"] // 2, 4 * c["window"]) for _ in range(c["seqs"])]
    if c["seqs"] >= 4:
        n[1], n[2] = 0, 1
    if c["op"] == "att":
        n = [0 if b % 3 == 0 else v for b, v in enumerate(n)]
    return n


class _Maker:
    """Seeded tensors on the GPU."""

    def __init__(self, seed, dtype):
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(seed)
        self.dtype = dtype

    def normal(self, *shape, scale=1.0, dtype=None):
        return (torch.randn(shape, generator=self.g, device="cuda") * scale).to(dtype or self.dtype)

    def uniform(self, *shape):
        return torch.rand(shape, generator=self.g, device="cuda")

    def ints(self, lo, hi, *shape):
        return torch.randint(lo, hi, shape, generator=self.g, device="cuda", dtype=torch.int32)

    def slots(self, seqs, holes):
        """A slot of a pool for each request, in no order; where a batch is padded, every seventh place has none."""
        s = torch.randperm(seqs + 3, generator=self.g, device="cuda")[:seqs].to(torch.int32)
        if holes:
            s[6::7] = -1
        return s


def _inputs(c, seed):
    """The tensors of a case.  Views are those that a program has: both gates
    are halves of one projection's rows, queries, keys and values lie side by
    side in another's."""
    m = _Maker(seed, _DTYPE[c["dtype"]])
    op = c["op"]
    s = {"op": op}
    t = c["seqs"] if op.endswith("_step") else c["tokens"]
    if op in ("rec", "rec_train", "att", "att_train"):
        s["first"] = _lengths(c)
        s["starts"] = torch.tensor(s["first"], dtype=torch.int32, device="cuda")
        s["longest"] = max(b - a for a, b in zip(s["first"], s["first"][1:]))
        s["ragged"] = c["ragged"]
    if op.startswith("rec"):
        d = c["d"]
        gates = m.normal(t, 2 * d)
        keep = 0.9 + 0.099 * m.uniform(d)            # a where the gate is open: such layers start so
        s.update(x=m.normal(t, d), r=gates[:, :d], i=gates[:, d:], lam=torch.log(torch.expm1(-torch.log(keep) / C)))
        if op == "rec_step":
            s.update(slots=m.slots(t, True), state=m.normal(t + 3, d, dtype=torch.float32))
        elif c["states"]:
            s["init"] = m.normal(c["seqs"], d, dtype=torch.float32)
        if op == "rec_train":
            s["dy"] = m.normal(t, d)
            if c["states"]:
                s["dfinal"] = m.normal(c["seqs"], d, dtype=torch.float32)
        return s
    h, kv, dim = c["heads"], c["kv"], c["dim"]
    rows = m.normal(t, (h + 2 * kv) * dim)
    q, k, v = (p.unflatten(1, (-1, dim)) for p in rows.split([h * dim, kv * dim, kv * dim], 1))
    if op.startswith("qk"):
        rot = c["rot"]
        s.update(q=q, k=k, wq=1 + m.normal(dim, scale=0.1, dtype=torch.float32), wk=1 + m.normal(dim, scale=0.1, dtype=torch.float32),
                 rot=rot, interleaved=c["interleaved"], freqs=10000.0 ** (-torch.arange(0, rot, 2, device="cuda", dtype=torch.float32) / rot))
        s["pos"] = m.ints(100000, 2000000, t) if c["far"] else torch.arange(t, device="cuda", dtype=torch.int32) % 4096
        if op == "qk_bwd":
            s.update(dq=m.normal(t, h, dim), dk=m.normal(t, kv, dim))
        return s
    s.update(q=q.contiguous(), k=k.contiguous(), v=v, window=c["window"], sinks=c["sinks"], scale=dim ** -0.5)
    if op == "att_train":
        s["dy"] = m.normal(t, h, dim)
        return s
    s["past_list"] = _past(c)
    s["past"] = torch.tensor(s["past_list"], dtype=torch.int32, device="cuda")
    s["slots"] = m.slots(c["seqs"], op == "att_step")
    s["k_cache"] = m.normal(c["seqs"] + 3, c["sinks"] + c["window"], kv, dim)
    s["v_cache"] = m.normal(c["seqs"] + 3, c["sinks"] + c["window"], kv, dim)
    return s


def prepare(case, seed):
    """Inputs and, for the framework's calls, the descriptor that a program
    makes once for a layer and its batch."""
    s = _inputs(case, seed)
    if s["op"] in ("att", "att_step"):
        s["slot_list"] = s["slots"].tolist()
    if own:
        import paper_2306_14320_amd as P
        s["P"] = P
        op = s["op"]
        seqs = 1 if op.endswith("_step") else case.get("seqs")
        if op.startswith("rec"):
            s["desc"] = P.gated_recurrence_desc_for(s["x"], s["r"], s["i"], sequences=seqs, c=C)
        elif op.startswith("qk"):
            s["desc"] = P.qk_norm_rope_desc_for(s["q"], s["k"], rot_dim=s["rot"], eps=EPS, interleaved=s["interleaved"])
        else:
            s["desc"] = P.window_attention_desc_for(s["q"], s["k"], s["v"], window=s["window"], sinks=s["sinks"], sequences=seqs, scale=s["scale"])
    return s


def run(s):
    return (_OWN if own else _PLAIN)[s["op"]](s)


# ---------------------------------------------------------------------------
# the framework's calls
# ---------------------------------------------------------------------------

def _starts(s):
    return s["starts"] if s["ragged"] else None


def _own_rec(s):
    final = torch.empty_like(s["init"]) if "init" in s else None
    y = s["P"].gated_recurrence(s["x"], s["r"], s["i"], s["lam"], s["desc"], seq_starts=_starts(s), initial_state=s.get("init"), final_state=final)
    return y if final is None else (y, final)


def _own_rec_train(s):
    P = s["P"]
    kept = P.gated_recurrence_chunk_states(s["x"], s["desc"])
    y = P.gated_recurrence(s["x"], s["r"], s["i"], s["lam"], s["desc"], seq_starts=_starts(s), initial_state=s.get("init"), chunk_states=kept)
    g = P.gated_recurrence_backward(s["dy"], s["x"], s["r"], s["i"], s["lam"], s["desc"], seq_starts=_starts(s), initial_state=s.get("init"),
                                    d_final_state=s.get("dfinal"), chunk_states=kept)
    return (y, g.dx, g.dr, g.di, g.dlam) + ((g.d_initial_state,) if "init" in s else ())


def _own_rec_step(s):
    y = s["P"].gated_recurrence_step(s["x"], s["r"], s["i"], s["lam"], s["state"], s["desc"], slots=s["slots"])
    return y, s["state"]


def _own_qk(s):
    return s["P"].qk_norm_rope(s["q"], s["k"], s["wq"], s["wk"], s["desc"], positions=s["pos"], freqs=s["freqs"])


def _own_qk_bwd(s):
    return tuple(s["P"].qk_norm_rope_backward(s["dq"], s["dk"], s["q"], s["k"], s["wq"], s["wk"], s["desc"], positions=s["pos"], freqs=s["freqs"]))


def _own_att(s):
    y = s["P"].window_attention(s["q"], s["k"], s["v"], s["desc"], seq_starts=_starts(s), k_cache=s["k_cache"], v_cache=s["v_cache"], past=s["past"], slots=s["slots"])
    return y, s["k_cache"], s["v_cache"]


def _own_att_train(s):
    P = s["P"]
    lse = torch.empty(s["q"].shape[:2], dtype=torch.float32, device="cuda")
    y = P.window_attention(s["q"], s["k"], s["v"], s["desc"], seq_starts=_starts(s), lse=lse)
    g = P.window_attention_backward(s["dy"], s["q"], s["k"], s["v"], y, lse, s["desc"], seq_starts=_starts(s))
    return y, g.dq, g.dk, g.dv


def _own_att_step(s):
    y = s["P"].window_attention_step(s["q"], s["k"], s["v"], s["k_cache"], s["v_cache"], s["past"], s["desc"], slots=s["slots"])
    return y, s["k_cache"], s["v_cache"]


_OWN = {"rec": _own_rec, "rec_train": _own_rec_train, "rec_step": _own_rec_step, "qk": _own_qk, "qk_bwd": _own_qk_bwd,
        "att": _own_att, "att_train": _own_att_train, "att_step": _own_att_step}


# ---------------------------------------------------------------------------
# plain forms: elementary operations on whole tensors, 32 bits inside
# ---------------------------------------------------------------------------

def _softplus(v):
    return v.clamp(min=0) + torch.log1p(torch.exp(-v.abs()))


def _scanned(a, b, longest):
    """h_t = a_t h_{t-1} + b_t over the rows, by doubling: after the step s each
    row holds the product and the sum of the s rows up to it."""
    s = 1
    while s < longest:
        b = torch.cat((b[:s], a[s:] * b[:-s] + b[s:]))
        a = torch.cat((a[:s], a[s:] * a[:-s]))
        s *= 2
    return b


def _gates(s):
    x, r, i = s["x"].float(), torch.sigmoid(s["r"].float()), torch.sigmoid(s["i"].float())
    log_a = -C * _softplus(s["lam"]) * r
    return x, r, i, log_a, torch.exp(log_a), torch.sqrt(-torch.expm1(2 * log_a))


def _rec_states(s):
    x, r, i, log_a, a, root = _gates(s)
    t = x.shape[0]
    b = root * i * x
    first = torch.zeros(t + 1, dtype=torch.bool, device="cuda")
    first[s["starts"][:-1].long()] = True       # an empty sequence at the end marks the row behind the last
    first = first[:-1, None]
    at = s["starts"][:-1].long().clamp(max=t - 1)
    live = (s["starts"][1:] > s["starts"][:-1])[:, None]
    if "init" in s:
        b.index_add_(0, at, torch.where(live, a[at] * s["init"], 0.0))
    return x, r, i, log_a, a, root, _scanned(torch.where(first, 0.0, a), b, s["longest"]), first, at, live


def _plain_rec(s):
    *_, h, _, _, live = _rec_states(s)
    y = h.to(s["x"].dtype)
    if "init" not in s:
        return y
    return y, torch.where(live, h[(s["starts"][1:].long() - 1).clamp(min=0)], s["init"])


def _plain_rec_train(s):
    x, r, i, log_a, a, root, h, first, at, live = _rec_states(s)
    dtype = s["x"].dtype
    last = torch.cat((first[1:], first.new_ones(1, 1)))
    g = s["dy"].float().clone()
    if "init" in s:
        g.index_add_(0, (s["starts"][1:].long() - 1).clamp(min=0), torch.where(live, s["dfinal"], 0.0))
    after = torch.where(last, 0.0, torch.cat((a[1:], a[:1])))
    g = _scanned(after.flip(0), g.flip(0), s["longest"]).flip(0)
    before = torch.where(first, 0.0, torch.cat((h[:1], h[:-1])))
    if "init" in s:
        before.index_add_(0, at, torch.where(live, s["init"], 0.0))
    d_log = g * (a * before - a * a / root * i * x) * log_a           # of log a, times log a
    out = [h.to(dtype), (g * root * i).to(dtype), (d_log * (1 - r)).to(dtype), (g * root * x * i * (1 - i)).to(dtype),
           d_log.sum(0) * torch.sigmoid(s["lam"]) / _softplus(s["lam"])]
    if "init" in s:
        out.append(torch.where(live, g[at] * a[at], s["dfinal"]))
    return tuple(out)


def _plain_rec_step(s):
    x, _, i, _, a, root = _gates(s)
    slots, state = s["slots"].long(), s["state"]
    live = (slots >= 0)[:, None]
    h = a * state[slots.clamp(min=0)] + root * i * x
    of = torch.full((state.shape[0] + 1,), -1, device="cuda")
    of[torch.where(slots >= 0, slots, state.shape[0])] = torch.arange(slots.numel(), device="cuda")
    of = of[:-1]
    torch.where((of >= 0)[:, None], h[of.clamp(min=0)], state, out=state)
    return torch.where(live, h, 0.0).to(s["x"].dtype), state


def _angles(s):
    """cos and sin of each row's angles, T x 1 x R/2: the angles of far positions need 64 bits."""
    angle = s["pos"].double()[:, None] * s["freqs"].double()
    return torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]


def _pairs(s, x):
    """The rotated channels' pairs and the rest of a tensor of heads."""
    rot = s["rot"]
    if s["interleaved"]:
        return x[..., 0:rot:2], x[..., 1:rot:2], x[..., rot:]
    return x[..., :rot // 2], x[..., rot // 2:rot], x[..., rot:]


def _joined(s, a, b, rest):
    pair = torch.stack((a, b), -1).flatten(-2) if s["interleaved"] else torch.cat((a, b), -1)
    return torch.cat((pair, rest), -1)


def _unit(x):
    x = x.float()
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    return x * r, r


def _plain_qk(s):
    cos, sin = _angles(s)
    out = []
    for x, w in ((s["q"], s["wq"]), (s["k"], s["wk"])):
        a, b, rest = _pairs(s, _unit(x)[0] * w)
        out.append(_joined(s, a * cos - b * sin, b * cos + a * sin, rest).to(x.dtype))
    return tuple(out)


def _plain_qk_bwd(s):
    cos, sin = _angles(s)
    out = []
    for x, w, dy in ((s["q"], s["wq"], s["dq"]), (s["k"], s["wk"], s["dk"])):
        a, b, rest = _pairs(s, dy.float())
        du = _joined(s, a * cos + b * sin, b * cos - a * sin, rest)
        n, r = _unit(x)
        g = du * w
        out += [(r * (g - n * (g * n).mean(-1, keepdim=True))).to(x.dtype), (du * n).sum((0, 1))]
    return out[0], out[2], out[1], out[3]


BLOCK = 1024      # queries of a sequence that are worked on at once


def _blocks(s, n, past):
    """Blocks of the new tokens' positions and the positions of the keys that they see between them."""
    for lo in range(past, past + n, BLOCK):
        hi = min(past + n, lo + BLOCK)
        begin = max(0, lo - s["window"] + 1)
        kp = torch.arange(begin, hi, device="cuda")
        if min(s["sinks"], begin):
            kp = torch.cat((torch.arange(min(s["sinks"], begin), device="cuda"), kp))
        qp = torch.arange(lo, hi, device="cuda")[:, None]
        yield lo - past, hi - past, kp, (kp <= qp) & ((kp > qp - s["window"]) | (kp < s["sinks"]))


def _ring(s, pos):
    return torch.where(pos < s["sinks"], pos, s["sinks"] + (pos - s["sinks"]) % s["window"])


def _softmax(q, k, seen, scale):
    """Weights of queries (n x H x D) over keys (m x K x D): K x G x n x m."""
    n, h, d = q.shape
    kv = k.shape[1]
    qg = q.reshape(n, kv, h // kv, d).permute(1, 2, 0, 3).reshape(kv, -1, d)
    sc = (qg @ k.permute(1, 2, 0).contiguous()).reshape(kv, h // kv, n, -1) * scale
    sc = torch.where(seen, sc, -math.inf)
    e = torch.exp(sc - sc.amax(-1, keepdim=True))
    return qg, e / e.sum(-1, keepdim=True)


def _attend(s, q, keys, values, seen):
    n, h, d = q.shape
    _, p = _softmax(q, keys, seen, s["scale"])
    kv = keys.shape[1]
    o = p.reshape(kv, -1, keys.shape[0]) @ values.permute(1, 0, 2).contiguous()
    return o.reshape(kv, h // kv, n, d).permute(2, 0, 1, 3).reshape(n, h, d)


def _rows_at(s, cache, new, past, slot, pos):
    """Keys or values at positions: of the cache below `past`, of the new tokens from there."""
    old = cache[slot][_ring(s, pos.clamp(max=past - 1))] if past else new[:1]
    return torch.where((pos < past)[:, None, None], old, new[(pos - past).clamp(min=0)]).float()


def _plain_att(s):
    y = torch.zeros_like(s["q"])
    for b, (lo, hi) in enumerate(zip(s["first"], s["first"][1:])):
        if lo == hi:
            continue
        past, slot, k, v = s["past_list"][b], s["slot_list"][b], s["k"][lo:hi], s["v"][lo:hi]
        for i, j, pos, seen in _blocks(s, hi - lo, past):
            y[lo + i:lo + j] = _attend(s, s["q"][lo + i:lo + j].float(), _rows_at(s, s["k_cache"], k, past, slot, pos), _rows_at(s, s["v_cache"], v, past, slot, pos), seen).to(y.dtype)
        n, w, sinks = hi - lo, s["window"], s["sinks"]
        pos = torch.arange(past + max(0, n - w), past + n, device="cuda")
        if past < sinks and n > w:
            pos = torch.cat((torch.arange(past, min(sinks, past + n - w), device="cuda"), pos))
        s["k_cache"][slot, _ring(s, pos)] = k[pos - past]
        s["v_cache"][slot, _ring(s, pos)] = v[pos - past]
    return y, s["k_cache"], s["v_cache"]


def _plain_att_step(s):
    """All requests at once: each one's row is put into its cache, then the cache is read."""
    past, slots, w, sinks = s["past"].long(), s["slots"].long(), s["window"], s["sinks"]
    n, h, d = s["q"].shape
    kv = s["k"].shape[1]
    of = torch.full((s["k_cache"].shape[0] + 1,), -1, device="cuda")
    of[torch.where(slots >= 0, slots, s["k_cache"].shape[0])] = torch.arange(n, device="cuda")
    of = of[:-1]
    at, mine = _ring(s, past), (of >= 0)[:, None, None]
    pool = torch.arange(of.numel(), device="cuda")
    row = at[of.clamp(min=0)]
    for cache, new in ((s["k_cache"], s["k"]), (s["v_cache"], s["v"])):
        cache[pool, row] = torch.where(mine, new[of.clamp(min=0)], cache[pool, row])
    slot = slots.clamp(min=0)
    keys, values = s["k_cache"][slot].float(), s["v_cache"][slot].float()     # n x rows x K x D
    seen = (torch.arange(keys.shape[1], device="cuda") <= past[:, None])[:, None, None]
    q = s["q"].float().reshape(n, kv, h // kv, d)
    sc = (q @ keys.permute(0, 2, 3, 1).contiguous()) * s["scale"]
    sc = torch.where(seen, sc, -math.inf)
    e = torch.exp(sc - sc.amax(-1, keepdim=True))
    o = (e / e.sum(-1, keepdim=True)) @ values.permute(0, 2, 1, 3).contiguous()
    return torch.where((slots >= 0)[:, None, None], o.reshape(n, h, d), 0.0).to(s["q"].dtype), s["k_cache"], s["v_cache"]


def _plain_att_train(s):
    dtype = s["q"].dtype
    q, k, v, dy = (s[n].float() for n in ("q", "k", "v", "dy"))
    h, d = q.shape[1:]
    kv = k.shape[1]
    y, dq, dk, dv = (torch.zeros(z.shape, device="cuda") for z in (q, q, k, k))

    def back(rows, n):
        return rows.reshape(kv, h // kv, n, d).permute(2, 0, 1, 3).reshape(n, h, d)

    for lo, hi in zip(s["first"], s["first"][1:]):
        for i, j, pos, seen in _blocks(s, hi - lo, 0):
            n, m = j - i, pos.numel()
            at = lo + pos
            qg, p = _softmax(q[lo + i:lo + j], k[at], seen, s["scale"])
            kt, vt = k[at].permute(1, 0, 2).contiguous(), v[at].permute(1, 0, 2).contiguous()       # K x m x D
            p = p.reshape(kv, -1, m)
            dyg = dy[lo + i:lo + j].reshape(n, kv, h // kv, d).permute(1, 2, 0, 3).reshape(kv, -1, d)
            y[lo + i:lo + j] = back(p @ vt, n)
            dp = dyg @ vt.transpose(1, 2).contiguous()
            ds = p * (dp - (p * dp).sum(-1, keepdim=True)) * s["scale"]
            dq[lo + i:lo + j] = back(ds @ kt, n)
            dk[at] += (ds.transpose(1, 2).contiguous() @ qg).permute(1, 0, 2)
            dv[at] += (p.transpose(1, 2).contiguous() @ dyg).permute(1, 0, 2)
    return y.to(dtype), dq.to(dtype), dk.to(dtype), dv.to(dtype)


_PLAIN = {"rec": _plain_rec, "rec_train": _plain_rec_train, "rec_step": _plain_rec_step, "qk": _plain_qk, "qk_bwd": _plain_qk_bwd,
          "att": _plain_att, "att_train": _plain_att_train, "att_step": _plain_att_step}


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------

def _seen_pairs(n, past, window, sinks):
    """Keys that n tokens behind `past` others see, counted over the tokens."""
    return sum(min(p + 1, window) + min(sinks, max(0, p + 1 - window)) for p in range(past, past + n))


def work(case):
    """Each input read once and each output written once.  Operations: one for
    each product, sum, exponential and root of the formulas; for attention the
    products of queries, keys and values (two forward, five backward)."""
    op, e = case["op"], _DTYPE[case["dtype"]].itemsize
    step = op.endswith("_step")
    if op.startswith("rec"):
        d, seqs = case["d"], case["seqs"]
        t = seqs if step else case["tokens"]
        active = seqs - seqs // 7 if step else seqs
        state = 4 * d * (active if step else seqs if case["states"] else 0)
        if op == "rec_train":
            return {"bytes": 8 * e * t * d + 8 * d + 3 * state, "flops": 45 * t * d}
        return {"bytes": 4 * e * t * d + 4 * d + 2 * state, "flops": 16 * t * d}
    h, kv, d = case["heads"], case["kv"], case["dim"]
    if op.startswith("qk"):
        t = case["tokens"]
        heads, small = t * (h + kv) * d, 8 * d + 4 * t + 2 * case["rot"]
        return {"bytes": 3 * e * heads + small + 8 * d, "flops": 16 * heads} if op == "qk_bwd" else {"bytes": 2 * e * heads + small, "flops": 8 * heads}
    w, sinks, past = case["window"], case["sinks"], _past(case)
    row = e * kv * d                                  # keys or values of one token
    if step:
        past = [p for b, p in enumerate(past) if b % 7 != 6]
        seen = sum(_seen_pairs(1, p, w, sinks) for p in past)
        return {"bytes": 2 * e * len(past) * (h + kv) * d + 2 * row * seen, "flops": 4 * d * h * seen}
    first, t = _lengths(case), case["tokens"]
    n = [b - a for a, b in zip(first, first[1:])]
    pairs = sum(_seen_pairs(m, p, w, sinks) for m, p in zip(n, past))
    if op == "att_train":
        return {"bytes": e * t * d * (4 * h + 4 * kv), "flops": 14 * d * h * pairs}
    cached = sum(min(p, w - 1) + min(sinks, max(0, p - w + 1)) for m, p in zip(n, past) if m)
    kept = sum(min(m, w) for m in n)
    return {"bytes": e * t * d * (2 * h + 2 * kv) + 2 * row * (cached + kept), "flops": 4 * d * h * pairs}


# ---------------------------------------------------------------------------
# 64 bits, from the definitions: one token, or one head, after another
# ---------------------------------------------------------------------------

def exact(case, seed):
    s = _inputs(case, seed)
    s = {k: v.double() if torch.is_tensor(v) and v.is_floating_point() else v for k, v in s.items()}
    return _EXACT[s["op"]](s)


def _sigmoid64(v):
    return 1 / (1 + torch.exp(-v))


def _exact_rec(s):
    """Sequences side by side, one token after another."""
    train = s["op"] == "rec_train"
    first, n = s["first"][:-1], [b - a for a, b in zip(s["first"], s["first"][1:])]
    t, d = s["x"].shape
    init = s["init"] if "init" in s else torch.zeros(len(n), d, dtype=torch.float64, device="cuda")
    leaf = [v.detach().clone().requires_grad_(train) for v in (s["x"], s["r"], s["i"], s["lam"], init)]
    x, r, i, lam, h = leaf
    a = torch.exp(-C * torch.log1p(torch.exp(lam)) * _sigmoid64(r))
    b = torch.sqrt((1 - a) * (1 + a)) * _sigmoid64(i) * x
    # a row behind the last that keeps a state as it is, for sequences that have ended
    a = torch.cat((a, torch.ones(1, d, dtype=torch.float64, device="cuda")))
    b = torch.cat((b, torch.zeros(1, d, dtype=torch.float64, device="cuda")))
    at = torch.tensor([[f + j if j < m else t for f, m in zip(first, n)] for j in range(max(n))], device="cuda")
    steps = []
    for j in range(max(n)):
        h = a[at[j]] * h + b[at[j]]
        steps.append(h)
    hs = torch.stack(steps)                                                  # L x B x D
    y = torch.zeros(t + 1, d, dtype=torch.float64, device="cuda").index_copy(0, at.flatten(), torch.where((at < t)[:, :, None], hs, 0.0).flatten(0, 1))[:t]
    if not train:
        return (y, h) if "init" in s else y
    total = (y * s["dy"]).sum() + ((h * s["dfinal"]).sum() if "init" in s else 0)
    g = torch.autograd.grad(total, leaf if "init" in s else leaf[:4])
    return (y.detach(),) + tuple(g)


def _exact_rec_step(s):
    state, y = s["state"].clone(), torch.zeros_like(s["x"])
    for b, slot in enumerate(s["slots"].tolist()):
        if slot >= 0:
            a = torch.exp(-C * torch.log1p(torch.exp(s["lam"])) * _sigmoid64(s["r"][b]))
            state[slot] = a * state[slot] + torch.sqrt((1 - a) * (1 + a)) * _sigmoid64(s["i"][b]) * s["x"][b]
            y[b] = state[slot]
    return y, state


def _exact_heads(s, x, w):
    """One pair of channels after another, as complex numbers."""
    y = x / torch.sqrt(x.square().sum(-1, keepdim=True) / x.shape[-1] + EPS) * w
    half, cols = s["rot"] // 2, list(y.unbind(-1))
    for p in range(half):
        i, j = (2 * p, 2 * p + 1) if s["interleaved"] else (p, p + half)
        angle = s["pos"].double() * s["freqs"][p]
        z = torch.complex(cols[i], cols[j]) * torch.complex(torch.cos(angle), torch.sin(angle))[:, None]
        cols[i], cols[j] = z.real, z.imag
    return torch.stack(cols, -1)


def _exact_qk(s):
    return _exact_heads(s, s["q"], s["wq"]), _exact_heads(s, s["k"], s["wk"])


def _exact_qk_bwd(s):
    out = []
    for x, w, dy in ((s["q"], s["wq"], s["dq"]), (s["k"], s["wk"], s["dk"])):
        x, w = x.clone().requires_grad_(), w.clone().requires_grad_()
        out.append(torch.autograd.grad((_exact_heads(s, x, w) * dy).sum(), (x, w)))
    return out[0][0], out[1][0], out[0][1], out[1][1]


def _exact_head(s, q, k, v, past):
    """One head: queries at past.., keys and values from position 0."""
    i = torch.arange(past, past + q.shape[0], device="cuda")[:, None]
    j = torch.arange(k.shape[0], device="cuda")[None]
    hidden = (j > i) | ((i - j >= s["window"]) & (j >= s["sinks"]))
    return torch.softmax((q @ k.t() * s["scale"]).masked_fill(hidden, -math.inf), 1) @ v


def _exact_att(s):
    """Each request's whole past is laid out, with zeros where the cache has forgotten it; no query sees those."""
    kc, vc, y = s["k_cache"].clone(), s["v_cache"].clone(), torch.zeros_like(s["q"])
    w, sinks = s["window"], s["sinks"]
    single = s["op"] == "att_step"
    for b, slot in enumerate(s["slots"].tolist()):
        lo, hi = (b, b + 1) if single else s["first"][b:b + 2]
        if slot < 0 or lo == hi:
            continue
        past = s["past_list"][b]
        k, v = (torch.zeros((past,) + z.shape[1:], dtype=torch.float64, device="cuda") for z in (s["k"], s["v"]))
        known = [p for p in range(past) if p < sinks or p >= past - w]
        rows = [p if p < sinks else sinks + (p - sinks) % w for p in known]
        k[known], v[known] = kc[slot, rows], vc[slot, rows]
        k, v = torch.cat((k, s["k"][lo:hi])), torch.cat((v, s["v"][lo:hi]))
        per = s["q"].shape[1] // k.shape[1]
        for h in range(s["q"].shape[1]):
            y[lo:hi, h] = _exact_head(s, s["q"][lo:hi, h], k[:, h // per], v[:, h // per], past)
        end = past + hi - lo
        new = [p for p in range(past, end) if p < sinks or p >= end - w]
        rows = [p if p < sinks else sinks + (p - sinks) % w for p in new]
        kc[slot, rows], vc[slot, rows] = k[new], v[new]
    return y, kc, vc


def _exact_att_train(s):
    q, k, v = s["q"], s["k"], s["v"]
    per = q.shape[1] // k.shape[1]
    y, dq, dk, dv = torch.zeros_like(q), torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(k)
    for lo, hi in zip(s["first"], s["first"][1:]):
        for h in range(q.shape[1] if hi > lo else 0):
            leaf = [z.detach().clone().requires_grad_() for z in (q[lo:hi, h], k[lo:hi, h // per], v[lo:hi, h // per])]
            o = _exact_head(s, *leaf, 0)
            g = torch.autograd.grad((o * s["dy"][lo:hi, h]).sum(), leaf)
            y[lo:hi, h], dq[lo:hi, h] = o.detach(), g[0]
            dk[lo:hi, h // per] += g[1]
            dv[lo:hi, h // per] += g[2]
    return y, dq, dk, dv


_EXACT = {"rec": _exact_rec, "rec_train": _exact_rec, "rec_step": _exact_rec_step, "qk": _exact_qk, "qk_bwd": _exact_qk_bwd,
          "att": _exact_att, "att_train": _exact_att_train, "att_step": _exact_att}
