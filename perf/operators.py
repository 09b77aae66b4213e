"""The performance cases of the sequence operators: the short causal
convolution, the selective state space scan that reads its output, and the
root-mean-square norm with the residual's addition in front of both.

Tokens are rows: a tensor of T tokens is T x D, and sequence b holds the rows
seq_starts[b] to seq_starts[b+1].  Op names:

- "conv", "conv_bwd", "conv_step": y = silu(bias + sum_k w[k] x[t-W+1+k]), its
  gradients, and the form for one token of each of many sequences;
- "scan", "scan_bwd", "scan_step": h_t = exp(dt_t A) h_{t-1} + dt_t x_t B_t,
  y_t = (C_t h_t + D x_t) silu(z_t), its gradients, and the form for one token;
- "norm", "norm_fp8", "norm_bwd": h = x + residual, y = h / rms(h) * w, the
  same with y in 8 bits and a scale for each row or block, and its gradients.

Where ``own`` is false, ``run`` computes them with elementary torch operations
in 32 bits; where it is true, with the framework's kernels.
"""
import math
import random

import torch

own = False

_DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-5


def listed():
    return [
        # one new token of 16 requests whose convolution states lie in a pool of slots
        dict(name="conv_step_16", op="conv_step", dtype="bf16", seqs=16, d=2048, width=4),
        # prompts of many lengths, one empty and one of one token, that go on from kept states; odd sizes
        dict(name="conv_prompts_f32_odd", op="conv", dtype="f32", tokens=9001, seqs=23, ragged=True, d=1351, width=3, states=True),
        # a batch of training sequences, forward
        dict(name="conv_train_bf16", op="conv", dtype="bf16", tokens=16384, seqs=8, ragged=False, d=4096, width=4, states=False),
        # the same layer's gradients
        dict(name="conv_train_bwd_bf16", op="conv_bwd", dtype="bf16", tokens=16384, seqs=8, ragged=False, d=4096, width=4, states=False),
        # one new token of 128 requests
        dict(name="scan_step_128", op="scan_step", dtype="bf16", seqs=128, d=4096, n=16, groups=1),
        # one long prompt: few rows, so the time axis has to be split
        dict(name="scan_prompt_8192_bf16", op="scan", dtype="bf16", tokens=8192, seqs=1, ragged=False, d=2048, n=16, groups=1, states=True),
        # many prompts of odd sizes, states of 24 values in 3 groups of channels
        dict(name="scan_prompts_f32_odd", op="scan", dtype="f32", tokens=3001, seqs=17, ragged=True, d=777, n=24, groups=3, states=True),
        # a batch of training sequences: the gradients of the scan
        dict(name="scan_train_bwd_bf16", op="scan_bwd", dtype="bf16", tokens=16384, seqs=8, ragged=False, d=2048, n=16, groups=1, states=False),
        # ragged training sequences in 32 bits with gradients of the states
        dict(name="scan_bwd_f32_odd", op="scan_bwd", dtype="f32", tokens=1999, seqs=5, ragged=True, d=420, n=16, groups=2, states=True),
        # a served step's norm: 16 rows, the products after it read 8 bits with one scale a row
        dict(name="norm_fp8_16", op="norm_fp8", dtype="bf16", residual="f32", tokens=16, d=2048, block=0),
        # a long prompt's norm, a scale for each 128 channels
        dict(name="norm_fp8_16384", op="norm_fp8", dtype="bf16", residual="bf16", tokens=16384, d=4096, block=128),
        # a training step's gradients of the norm, residual in 32 bits, odd sizes
        dict(name="norm_bwd_bf16_odd", op="norm_bwd", dtype="bf16", residual="f32", tokens=8191, d=2049, block=0),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """A case of the listed ones' ranges: 1 to 16384 tokens in up to 64
    sequences, 64 to 4096 channels (half of them the multiples of 64 that
    models use), filters of 2 to 4 taps, states of 8 to 64 values, and no more
    elements than the largest listed case of the op's kind."""
    while True:
        op = rng.choice(["conv", "conv_bwd", "conv_step", "scan", "scan", "scan_bwd", "scan_bwd", "scan_step", "norm", "norm_fp8", "norm_bwd"])
        c = {"op": op, "dtype": rng.choice(["f32", "bf16"])}
        d = _log_int(rng, 64, 4096)
        if rng.random() < 0.5:
            d = d // 64 * 64
        tokens = _log_int(rng, 1, 16384)
        if op.endswith("_step"):
            c["seqs"] = _log_int(rng, 1, 256)
        elif not op.startswith("norm"):
            seqs = min(tokens, _log_int(rng, 1, 64))
            ragged = rng.random() < 0.5
            c.update(tokens=tokens if ragged else tokens // seqs * seqs, seqs=seqs, ragged=ragged, states=rng.random() < 0.5)
        if op.startswith("conv"):
            c.update(d=d, width=rng.choice([2, 3, 4, 4]))
        elif op.startswith("scan"):
            groups = rng.choice([1, 1, 2, 4])
            n = rng.choice([8, 16, 16, 16, 24, 32, 64])
            c.update(d=d // groups * groups, n=n, groups=groups)
            if c.get("tokens", 1) * c["d"] * n > 16384 * 2048 * 16 or c["seqs"] * c["d"] * n > 16384 * 1024:
                continue
        else:
            block = rng.choice([0, 64, 128]) if op == "norm_fp8" else 0
            c.update(tokens=tokens, d=max(block, d // block * block) if block else d, block=block, residual=rng.choice(["f32", c["dtype"]]))
        if 3072 not in c.values() and c["d"] != 1536:
            return c


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

    def slots(self, seqs):
        """A slot of a pool for each request, in no order; every seventh request is a padded place without one."""
        s = torch.randperm(seqs + 5, generator=self.g, device="cuda")[:seqs].to(torch.int32)
        s[6::7] = -1
        return s


def _inputs(c, seed):
    """The tensors of a case.  Views are those that a program has: the
    convolution's input and the gate are halves of one projection's rows, B
    and C lie behind the low-rank part of another's."""
    m = _Maker(seed, _DTYPE[c["dtype"]])
    op, d = c["op"], c["d"]
    s = {"op": op}
    if op.startswith("norm"):
        t, rd = c["tokens"], _DTYPE[c["residual"]]
        s.update(w=1 + m.normal(d, scale=0.1, dtype=torch.float32))
        if op == "norm_bwd":
            s.update(dy=m.normal(t, d), h=m.normal(t, d, scale=2.0, dtype=rd), dres=m.normal(t, d, dtype=rd))
        else:
            s.update(x=m.normal(t, d), res=m.normal(t, d, scale=2.0, dtype=rd), block=c["block"], out=m.dtype)
        return s
    t = c["seqs"] if op.endswith("_step") else c["tokens"]
    s["xz"] = m.normal(t, 2 * d)
    if op.endswith("_step"):
        s["slots"] = m.slots(c["seqs"])
    else:
        starts = _lengths(c)
        s["starts"] = torch.tensor(starts, dtype=torch.int32, device="cuda")
        s["longest"] = max(b - a for a, b in zip(starts, starts[1:]))
        s["ragged"] = c["ragged"]
    if op.startswith("conv"):
        w = c["width"]
        s.update(x=s["xz"][:, :d], w=m.normal(d, w, scale=w ** -0.5), bias=m.normal(d, scale=0.1))
        if op == "conv_step":
            s["state"] = m.normal(c["seqs"] + 5, w - 1, d)
        elif c["states"]:
            s["init"] = m.normal(c["seqs"], w - 1, d)
        if op == "conv_bwd":
            s["dy"] = m.normal(t, d)
            if c["states"]:
                s["dfinal"] = m.normal(c["seqs"], w - 1, d)
        return s
    n, g = c["n"], c["groups"]
    rank = -(-d // 16)
    low = m.normal(t, rank + 2 * g * n)
    step = torch.exp(m.uniform(d) * math.log(100) + math.log(1e-3))   # steps of 1e-3 to 1e-1, as such layers start
    s.update(x=m.normal(t, d), dt=m.normal(t, d, scale=0.5), z=s["xz"][:, d:],
             A=-(1 + torch.arange(n, device="cuda", dtype=torch.float32)) * (0.5 + m.uniform(d, 1)),
             B=low[:, rank:rank + g * n].unflatten(1, (g, n)), C=low[:, rank + g * n:].unflatten(1, (g, n)),
             D=1 + m.normal(d, scale=0.1, dtype=torch.float32), dt_bias=step + torch.log(-torch.expm1(-step)))
    if op == "scan_step":
        s["state"] = m.normal(c["seqs"] + 5, d, n, dtype=torch.float32)
    elif c["states"]:
        s["init"] = m.normal(c["seqs"], d, n, dtype=torch.float32)
    if op == "scan_bwd":
        s["dy"] = m.normal(t, d)
        if c["states"]:
            s["dfinal"] = m.normal(c["seqs"], d, n, dtype=torch.float32)
    return s


def prepare(case, seed):
    """Inputs and, for the framework's calls, the descriptor that a program
    makes once for a layer and its batch."""
    s = _inputs(case, seed)
    if own:
        import paper_2306_14320_amd as P
        s["P"] = P
        op = s["op"]
        if op.startswith("norm"):
            s["desc"] = P.rms_norm_desc_for(case["tokens"], case["d"], s["dy" if op == "norm_bwd" else "x"].dtype, s["h" if op == "norm_bwd" else "res"].dtype, EPS, block=case["block"])
        elif op.startswith("conv"):
            s["desc"] = P.causal_conv1d_desc_for(s["x"], s["w"], 1 if op == "conv_step" else case["seqs"], silu=True)
        else:
            s["desc"] = P.selective_scan_desc_for(s["x"], s["dt"], s["A"], s["B"], s["C"], s["z"], 1 if op == "scan_step" else case["seqs"], softplus=True)
    return s


def run(s):
    return (_OWN if own else _PLAIN)[s["op"]](s)


# ---------------------------------------------------------------------------
# the framework's calls
# ---------------------------------------------------------------------------

def _starts(s):
    return s["starts"] if s["ragged"] else None


def _own_conv(s):
    final = torch.empty_like(s["init"]) if "init" in s else None
    y = s["P"].causal_conv1d(s["x"], s["w"], s["desc"], bias=s["bias"], seq_starts=_starts(s), initial_state=s.get("init"), final_state=final)
    return y if final is None else (y, final)


def _own_conv_bwd(s):
    g = s["P"].causal_conv1d_backward(s["dy"], s["x"], s["w"], s["desc"], bias=s["bias"], seq_starts=_starts(s), initial_state=s.get("init"), d_final_state=s.get("dfinal"))
    return (g.dx, g.dw, g.dbias) + ((g.d_initial_state,) if "init" in s else ())


def _own_conv_step(s):
    y = s["P"].causal_conv1d_step(s["x"], s["w"], s["state"], s["desc"], bias=s["bias"], slots=s["slots"])
    return y, s["state"]


def _own_scan(s):
    final = torch.empty_like(s["init"]) if "init" in s else None
    y = s["P"].selective_scan(s["x"], s["dt"], s["A"], s["B"], s["C"], s["desc"], D=s["D"], z=s["z"], dt_bias=s["dt_bias"], seq_starts=_starts(s), initial_state=s.get("init"), final_state=final)
    return y if final is None else (y, final)


def _own_scan_bwd(s):
    g = s["P"].selective_scan_backward(s["dy"], s["x"], s["dt"], s["A"], s["B"], s["C"], s["desc"], D=s["D"], z=s["z"], dt_bias=s["dt_bias"], seq_starts=_starts(s),
                                       initial_state=s.get("init"), d_final_state=s.get("dfinal"))
    return (g.dx, g.ddt, g.dA, g.dB, g.dC, g.dD, g.dz, g.ddt_bias) + ((g.d_initial_state,) if "init" in s else ())


def _own_scan_step(s):
    y = s["P"].selective_scan_step(s["x"], s["dt"], s["A"], s["B"], s["C"], s["state"], s["desc"], D=s["D"], z=s["z"], dt_bias=s["dt_bias"], slots=s["slots"])
    return y, s["state"]


def _own_norm(s):
    return s["P"].add_rms_norm(s["x"], s["w"], s["desc"], residual=s["res"])


def _own_norm_fp8(s):
    return s["P"].add_rms_norm_fp8(s["x"], s["w"], s["desc"], residual=s["res"])


def _own_norm_bwd(s):
    return s["P"].add_rms_norm_backward(s["dy"], s["h"], s["w"], s["desc"], d_residual=s["dres"])


_OWN = {"conv": _own_conv, "conv_bwd": _own_conv_bwd, "conv_step": _own_conv_step, "scan": _own_scan, "scan_bwd": _own_scan_bwd,
        "scan_step": _own_scan_step, "norm": _own_norm, "norm_fp8": _own_norm_fp8, "norm_bwd": _own_norm_bwd}


# ---------------------------------------------------------------------------
# plain forms: elementary operations on whole tensors, 32 bits inside
# ---------------------------------------------------------------------------

def _sequence_of(starts, tokens):
    """The sequence of each row."""
    return torch.searchsorted(starts, torch.arange(tokens, device="cuda", dtype=torch.int32), right=True) - 1


def _extended(s):
    """The inputs of all sequences with each one's W-1 inputs before it (zeros
    where it has no state), and the row of each token there."""
    x, w = s["x"].float(), s["w"].shape[1]
    t, b = x.shape[0], s["starts"].numel() - 1
    row = torch.arange(t, device="cuda") + (_sequence_of(s["starts"], t) + 1) * (w - 1)
    first = s["starts"][:-1].long() + torch.arange(b, device="cuda") * (w - 1)
    ext = torch.zeros(t + b * (w - 1), x.shape[1], device="cuda")
    ext[row] = x
    if "init" in s:
        ext[first[:, None] + torch.arange(w - 1, device="cuda")] = s["init"].float()
    return ext, row, first


def _windows(s):
    ext, row, first = _extended(s)
    w = s["w"].shape[1]
    win = ext[row[:, None] + torch.arange(1 - w, 1, device="cuda")]          # T x W x D
    pre = (win * s["w"].float().t()).sum(1) + s["bias"].float()
    return ext, row, first, win, pre


def _last_rows(s):
    """Where the final state of each sequence begins in the extended inputs."""
    w = s["w"].shape[1]
    b = s["starts"].numel() - 1
    return (s["starts"][1:].long() + torch.arange(b, device="cuda") * (w - 1))[:, None] + torch.arange(w - 1, device="cuda")


def _plain_conv(s):
    ext, _, _, _, pre = _windows(s)
    y = (pre * torch.sigmoid(pre)).to(s["x"].dtype)
    return (y, ext[_last_rows(s)].to(s["x"].dtype)) if "init" in s else y


def _plain_conv_bwd(s):
    ext, row, first, win, pre = _windows(s)
    w, dtype = s["w"].shape[1], s["x"].dtype
    sig = torch.sigmoid(pre)
    g = s["dy"].float() * sig * (1 + pre * (1 - sig))
    # g of the token that ends its window W-1 rows on, zeros elsewhere: input e gets sum_k w[k] g[e-k]
    pad = torch.zeros(ext.shape[0] + w - 1, ext.shape[1], device="cuda")
    pad[row] = g
    dext = (pad[torch.arange(ext.shape[0], device="cuda")[:, None] + torch.arange(w - 1, -1, -1, device="cuda")] * s["w"].float().t()).sum(1)
    out = [None, (win * g[:, None]).sum(0).t().contiguous(), g.sum(0)]
    if "init" in s:
        dext[_last_rows(s)] += s["dfinal"].float()
        out.append(dext[first[:, None] + torch.arange(w - 1, device="cuda")].to(dtype))
    out[0] = dext[row].to(dtype)
    return tuple(out)


def _to_slots(state, slots, new):
    """The pool with each request's new state in its slot: a request without one is left out."""
    of = torch.full((state.shape[0] + 1,), -1, device="cuda")
    of[torch.where(slots >= 0, slots, state.shape[0])] = torch.arange(slots.numel(), device="cuda")
    of = of[:-1]
    return torch.where((of >= 0)[:, None, None], new[of.clamp(min=0)].to(state.dtype), state, out=state)


def _plain_conv_step(s):
    x, w, slots, state = s["x"].float(), s["w"].float(), s["slots"].long(), s["state"]
    live = (slots >= 0)[:, None]
    at = slots.clamp(min=0)
    win = torch.cat((state[at].float(), x[:, None]), 1)                     # requests x W x D
    pre = (win * w.t()).sum(1) + s["bias"].float()
    y = torch.where(live, pre * torch.sigmoid(pre), 0.0).to(s["x"].dtype)
    return y, _to_slots(state, slots, win[:, 1:])


def _softplus(v):
    return v.clamp(min=0) + torch.log1p(torch.exp(-v.abs()))


def _per_channel(m, d):
    """B or C, T x G x N, for each channel: T x D x N."""
    t, g, n = m.shape
    return m.float()[:, :, None].expand(t, g, d // g, n).reshape(t, d, n)


def _scanned(a, b, longest):
    """h_t = a_t h_{t-1} + b_t over the rows, by doubling: after the step s each
    row holds the product and the sum of the s rows up to it."""
    s = 1
    while s < longest:
        b = torch.cat((b[:s], a[s:] * b[:-s] + b[s:]))
        a = torch.cat((a[:s], a[s:] * a[:-s]))
        s *= 2
    return b


def _scan_states(s):
    x, d = s["x"].float(), s["x"].shape[1]
    raw = s["dt"].float() + s["dt_bias"]
    dt = _softplus(raw)
    a = torch.exp(dt[:, :, None] * s["A"])
    b = (dt * x)[:, :, None] * _per_channel(s["B"], d)
    t = x.shape[0]
    first = torch.zeros(t + 1, dtype=torch.bool, device="cuda")
    first[s["starts"][:-1].long()] = True       # an empty sequence at the end marks the row behind the last
    first = first[:-1, None, None]
    at = s["starts"][:-1].long().clamp(max=t - 1)
    live = (s["starts"][1:] > s["starts"][:-1])[:, None, None]
    if "init" in s:
        b.index_add_(0, at, torch.where(live, a[at] * s["init"], 0.0))
    h = _scanned(torch.where(first, 0.0, a), b, s["longest"])
    return x, raw, dt, a, h, first, at, live


def _plain_scan(s):
    x, _, _, _, h, _, _, live = _scan_states(s)
    z = s["z"].float()
    y = (h * _per_channel(s["C"], x.shape[1])).sum(2) + s["D"] * x
    y = (y * z * torch.sigmoid(z)).to(s["x"].dtype)
    if "init" not in s:
        return y
    return y, torch.where(live, h[(s["starts"][1:].long() - 1).clamp(min=0)], s["init"])


def _plain_scan_bwd(s):
    x, raw, dt, a, h, first, at, live = _scan_states(s)
    t, d = x.shape
    dtype, z = s["x"].dtype, s["z"].float()
    b, c = _per_channel(s["B"], d), _per_channel(s["C"], d)
    sig = torch.sigmoid(z)
    pre = (h * c).sum(2) + s["D"] * x
    dy = s["dy"].float()
    dz = dy * pre * sig * (1 + z * (1 - sig))
    dpre = dy * z * sig
    g = dpre[:, :, None] * c
    last = torch.cat((first[1:], first.new_ones(1, 1, 1)))
    if "init" in s:
        g.index_add_(0, (s["starts"][1:].long() - 1).clamp(min=0), torch.where(live, s["dfinal"], 0.0))
    after = torch.where(last, 0.0, torch.cat((a[1:], a[:1])))
    g = _scanned(after.flip(0), g.flip(0), s["longest"]).flip(0)
    before = torch.where(first, 0.0, torch.cat((h[:1], h[:-1])))
    if "init" in s:
        before.index_add_(0, at, torch.where(live, s["init"], 0.0))
    q = g * a * before                      # of the exponent dt A
    gb = (g * b).sum(2)                     # of dt x
    ddt = (q * s["A"]).sum(2) + gb * x
    draw_ = ddt * torch.sigmoid(raw)
    groups, n = s["B"].shape[1:]
    out = [(gb * dt + dpre * s["D"]).to(dtype), draw_.to(dtype), (q * dt[:, :, None]).sum(0),
           (g * (dt * x)[:, :, None]).reshape(t, groups, d // groups, n).sum(2).to(dtype),
           (h * dpre[:, :, None]).reshape(t, groups, d // groups, n).sum(2).to(dtype),
           (dpre * x).sum(0), dz.to(dtype), draw_.sum(0)]
    if "init" in s:
        out.append(torch.where(live, g[at] * a[at], s["dfinal"]))
    return tuple(out)


def _plain_scan_step(s):
    x, z, slots, state = s["x"].float(), s["z"].float(), s["slots"].long(), s["state"]
    d = x.shape[1]
    dt = _softplus(s["dt"].float() + s["dt_bias"])
    h = torch.exp(dt[:, :, None] * s["A"]) * state[slots.clamp(min=0)] + (dt * x)[:, :, None] * _per_channel(s["B"], d)
    y = ((h * _per_channel(s["C"], d)).sum(2) + s["D"] * x) * z * torch.sigmoid(z)
    return torch.where((slots >= 0)[:, None], y, 0.0).to(s["x"].dtype), _to_slots(state, slots, h)


def _normed(s):
    h = (s["x"].float() + s["res"].float()).to(s["res"].dtype)
    v = h.float()
    return h, v * torch.rsqrt((v * v).mean(1, keepdim=True) + EPS) * s["w"]


def _plain_norm(s):
    h, y = _normed(s)
    return y.to(s["out"]), h


def _plain_norm_fp8(s):
    h, y = _normed(s)
    t, d = y.shape
    y = y.reshape(t, -1, s["block"] or d)
    scale = y.abs().amax(2) / 448.0
    scale = torch.where(scale > 0, scale, 1.0)
    return (y / scale[:, :, None]).reshape(t, d).to(torch.float8_e4m3fn), scale, h


def _plain_norm_bwd(s):
    h, dy = s["h"].float(), s["dy"].float()
    r = torch.rsqrt((h * h).mean(1, keepdim=True) + EPS)
    gw = dy * s["w"]
    n = h * r
    dx = r * (gw - n * (gw * n).mean(1, keepdim=True)) + s["dres"].float()
    return dx.to(s["h"].dtype), (dy * n).sum(0)


_PLAIN = {"conv": _plain_conv, "conv_bwd": _plain_conv_bwd, "conv_step": _plain_conv_step, "scan": _plain_scan, "scan_bwd": _plain_scan_bwd,
          "scan_step": _plain_scan_step, "norm": _plain_norm, "norm_fp8": _plain_norm_fp8, "norm_bwd": _plain_norm_bwd}


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------

def work(case):
    """Each input read once and each output written once.  Operations: one for
    each product, sum and exponential of the formulas, counted over the states
    (the scan) or the taps (the convolution)."""
    op, d = case["op"], case["d"]
    e = _DTYPE[case["dtype"]].itemsize
    if op.startswith("norm"):
        t, r = case["tokens"], _DTYPE[case["residual"]].itemsize
        if op == "norm_bwd":
            return {"bytes": t * d * (e + 3 * r) + 8 * d, "flops": 9 * t * d}
        if op == "norm_fp8":
            return {"bytes": t * d * (e + 2 * r + 1) + 4 * d + 4 * t * (d // (case["block"] or d)), "flops": 7 * t * d}
        return {"bytes": t * d * (2 * e + 2 * r) + 4 * d, "flops": 5 * t * d}
    step = op.endswith("_step")
    seqs = case["seqs"]
    t = seqs if step else case["tokens"]
    active = seqs - seqs // 7 if step else seqs
    if op.startswith("conv"):
        w = case["width"]
        weights = e * d * (w + 1)
        state = e * (w - 1) * d * (active if step else seqs if case["states"] else 0)
        if op == "conv_bwd":
            return {"bytes": 3 * e * t * d + weights + 4 * d * (w + 1) + 3 * state, "flops": t * d * (6 * w + 8)}
        return {"bytes": 2 * e * t * d + weights + 2 * state, "flops": t * d * (2 * w + 5)}
    n, g = case["n"], case["groups"]
    weights = 4 * d * (n + 2)
    state = 4 * d * n * (active if step else seqs if case["states"] else 0)
    if op == "scan_bwd":
        return {"bytes": e * t * (7 * d + 4 * g * n) + 2 * weights + 3 * state, "flops": t * d * (18 * n + 20)}
    return {"bytes": e * t * (4 * d + 2 * g * n) + weights + 2 * state, "flops": t * d * (7 * n + 12)}


# ---------------------------------------------------------------------------
# 64 bits, from the definitions: one token after another
# ---------------------------------------------------------------------------

def exact(case, seed):
    s = _inputs(case, seed)
    op = s["op"]
    s = {k: v.double() if torch.is_tensor(v) and v.is_floating_point() else v for k, v in s.items()}
    return _EXACT[op](s)


class _Padded:
    """Sequences side by side, each from its first token: rows of a T x ... tensor as L x B x ... and back."""

    def __init__(self, starts):
        st = starts.tolist()
        self.first, self.len = st[:-1], [b - a for a, b in zip(st, st[1:])]
        self.n, self.longest = len(self.len), max(self.len)
        pos = torch.arange(self.longest, device="cuda")[:, None]
        lens = torch.tensor(self.len, device="cuda")
        self.live = pos < lens                                               # L x B
        self.at = (pos + torch.tensor(self.first, device="cuda")) * self.live

    def put(self, rows):
        live = self.live.reshape(self.live.shape + (1,) * (rows.dim() - 1))
        return torch.where(live, rows[self.at], torch.zeros((), dtype=rows.dtype, device="cuda"))

    def back(self, padded, tokens):
        out = torch.zeros((tokens,) + padded.shape[2:], dtype=padded.dtype, device="cuda")
        out[self.at[self.live]] = padded[self.live]
        return out


def _exact_conv(s):
    p = _Padded(s["starts"])
    w, t = s["w"], s["x"].shape[0]
    taps = w.shape[1]
    init = s.get("init")
    history = init.transpose(0, 1) if init is not None else torch.zeros(taps - 1, p.n, w.shape[0], dtype=torch.float64, device="cuda")
    x = s["x"].detach()
    leaf = [v.detach().clone().requires_grad_(s["op"] == "conv_bwd") for v in (x, w, s["bias"], history)]
    line = torch.cat((leaf[3], p.put(leaf[0])))                              # (W-1+L) x B x D
    pre = sum(line[k:k + p.longest] * leaf[1][:, k] for k in range(taps)) + leaf[2]
    y = p.back(pre / (1 + torch.exp(-pre)), t)
    final = torch.stack([line[n:n + taps - 1, b] for b, n in enumerate(p.len)])
    if s["op"] == "conv":
        return (y, final) if init is not None else y
    total = (y * s["dy"]).sum() + ((final * s["dfinal"]).sum() if init is not None else 0)
    g = torch.autograd.grad(total, leaf if init is not None else leaf[:3])
    return (g[0], g[1], g[2]) + ((g[3].transpose(0, 1).contiguous(),) if init is not None else ())


def _exact_conv_step(s):
    state, y = s["state"].clone(), torch.zeros_like(s["x"])
    for b, slot in enumerate(s["slots"].tolist()):
        if slot >= 0:
            win = torch.cat((state[slot], s["x"][b:b + 1]))
            pre = (win * s["w"].t()).sum(0) + s["bias"]
            y[b] = pre / (1 + torch.exp(-pre))
            state[slot] = win[1:]
    return y, state


def _recurrence(s):
    """The states after each token of the padded sequences, one token after another."""
    p = _Padded(s["starts"])
    d, groups = s["x"].shape[1], s["B"].shape[1]
    x, dt = p.put(s["x"]), p.put(torch.logaddexp(s["dt"] + s["dt_bias"], torch.zeros((), dtype=torch.float64, device="cuda")))
    bm, cm = p.put(s["B"]), p.put(s["C"])
    of = torch.arange(d, device="cuda") // (d // groups)
    h = s["init"] if "init" in s else torch.zeros(p.n, d, s["A"].shape[1], dtype=torch.float64, device="cuda")
    return p, x, dt, bm, cm, of, h


def _exact_scan(s):
    p, x, dt, bm, cm, of, h = _recurrence(s)
    ys = torch.empty_like(x)
    for i in range(p.longest):
        new = torch.exp(dt[i, :, :, None] * s["A"]) * h + (dt[i] * x[i])[:, :, None] * bm[i][:, of]
        h = torch.where(p.live[i][:, None, None], new, h)
        torch.sum(h * cm[i][:, of], 2, out=ys[i])
    y = (p.back(ys, s["x"].shape[0]) + s["D"] * s["x"]) * s["z"] / (1 + torch.exp(-s["z"]))
    return (y, h) if "init" in s else y


def _exact_scan_bwd(s):
    p, x, dt, bm, cm, of, h0 = _recurrence(s)
    a_, t = s["A"], s["x"].shape[0]
    groups, n = s["B"].shape[1:]
    d = x.shape[2]
    hs = torch.empty((p.longest + 1,) + h0.shape, dtype=torch.float64, device="cuda")
    hs[0] = h0
    pre = torch.empty_like(x)
    for i in range(p.longest):
        new = torch.exp(dt[i, :, :, None] * a_) * hs[i] + (dt[i] * x[i])[:, :, None] * bm[i][:, of]
        hs[i + 1] = torch.where(p.live[i][:, None, None], new, hs[i])
        pre[i] = (hs[i + 1] * cm[i][:, of]).sum(2)
    sig = 1 / (1 + torch.exp(-s["z"]))
    dz = s["dy"] * (p.back(pre, t) + s["D"] * s["x"]) * (sig + s["z"] * sig * (1 - sig))
    do = s["dy"] * s["z"] * sig
    dop = p.put(do)
    lam = s["dfinal"].clone() if "init" in s else torch.zeros_like(h0)       # of the state after token i
    dx, ddt, da = torch.empty_like(x), torch.empty_like(x), torch.zeros_like(a_)
    db, dc = torch.empty_like(bm), torch.empty_like(cm)
    for i in range(p.longest - 1, -1, -1):
        live = p.live[i][:, None, None]
        lam = torch.where(live, lam + dop[i][:, :, None] * cm[i][:, of], lam)
        decay = torch.exp(dt[i, :, :, None] * a_)
        into = torch.where(live, lam, 0.0)
        grad_decay = into * hs[i] * decay
        grad_in = (into * bm[i][:, of]).sum(2)
        dx[i], ddt[i] = grad_in * dt[i], (grad_decay * a_).sum(2) + grad_in * x[i]
        da += (grad_decay * dt[i][:, :, None]).sum(0)
        db[i] = (into * (dt[i] * x[i])[:, :, None]).reshape(p.n, groups, -1, n).sum(2)
        dc[i] = (hs[i + 1] * dop[i][:, :, None]).reshape(p.n, groups, -1, n).sum(2)
        lam = torch.where(live, lam * decay, lam)
    draw_ = p.back(ddt, t) / (1 + torch.exp(-(s["dt"] + s["dt_bias"])))
    out = (p.back(dx, t) + do * s["D"], draw_, da, p.back(db, t), p.back(dc, t), (do * s["x"]).sum(0), dz, draw_.sum(0))
    return out + ((lam,) if "init" in s else ())


def _exact_scan_step(s):
    state, y = s["state"].clone(), torch.zeros_like(s["x"])
    groups = s["B"].shape[1]
    of = torch.arange(y.shape[1], device="cuda") // (y.shape[1] // groups)
    for b, slot in enumerate(s["slots"].tolist()):
        if slot >= 0:
            dt = torch.logaddexp(s["dt"][b] + s["dt_bias"], torch.zeros((), dtype=torch.float64, device="cuda"))[:, None]
            state[slot] = torch.exp(dt * s["A"]) * state[slot] + dt * s["x"][b][:, None] * s["B"][b][of]
            y[b] = ((state[slot] * s["C"][b][of]).sum(1) + s["D"] * s["x"][b]) * s["z"][b] / (1 + torch.exp(-s["z"][b]))
    return y, state


def _exact_norm(s):
    h = s["x"] + s["res"]
    return h / (h.square().sum(1, keepdim=True) / h.shape[1] + EPS).sqrt() * s["w"], h


def _exact_norm_fp8(s):
    y, h = _exact_norm(s)
    scale = y.reshape(y.shape[0], -1, s["block"] or y.shape[1]).abs().amax(2) / 448
    return y / scale.repeat_interleave(y.shape[1] // scale.shape[1], 1), scale, h


def _exact_norm_bwd(s):
    h, w = s["h"].clone().requires_grad_(), s["w"].clone().requires_grad_()
    y = h / (h.square().sum(1, keepdim=True) / h.shape[1] + EPS).sqrt() * w
    return torch.autograd.grad((y * s["dy"]).sum() + (h * s["dres"]).sum(), (h, w))


_EXACT = {"conv": _exact_conv, "conv_bwd": _exact_conv, "conv_step": _exact_conv_step, "scan": _exact_scan, "scan_bwd": _exact_scan_bwd,
          "scan_step": _exact_scan_step, "norm": _exact_norm, "norm_fp8": _exact_norm_fp8, "norm_bwd": _exact_norm_bwd}
