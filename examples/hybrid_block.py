"""Two layers of a hybrid stack on the framework's sequence operators: a gated
linear recurrence, and attention with a sliding window.

A layer adds its output to the residual h (width D) of a token t:

    recurrence                                   attention
    y, h = norm(x + h)      add_rms_norm         y, h    = norm(x + h)
    u    = conv(y W_in)     causal_conv1d        q, k, v = y W_qkv, per head
    r, i = u W_gates                             q, k    = rotated(normed(q, k))   qk_norm_rope
    s    = gated scan of u  gated_recurrence     s       = attention over the last tokens
    x    = s W_out                                         and the first few       window_attention
                                                 x       = s W_out

``Recurrence`` and ``Attention`` each have ``prompt`` (packed prompts that go on
from the requests' states or caches), ``token`` (one token of each request) and
``train`` (forward and gradients).  Run as a script it serves prompts and single
tokens on random weights, says how far they are from one call over all rows,
and trains both layers for some steps.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2306_14320_amd as P  # noqa: E402


def _weights(seed, device):
    g = torch.Generator(device="cpu").manual_seed(seed)

    def normal(*shape, dtype):
        return (torch.randn(shape, generator=g) * shape[0] ** -0.5).to(dtype).to(device)

    return normal


class _Layer:
    def normed(self, x, h):
        return P.add_rms_norm(x, self.norm_w, P.rms_norm_desc_for(x.shape[0], self.width, self.dtype, h.dtype), residual=h)


class Recurrence(_Layer):
    taps = 4

    def __init__(self, width, dtype=torch.bfloat16, device="cuda", seed=0):
        normal = _weights(seed, device)
        self.width, self.dtype = width, dtype
        self.norm_w = torch.ones(width, device=device)
        self.w_in, self.w_gates, self.w_out = normal(width, width, dtype=dtype), normal(width, 2 * width, dtype=dtype), normal(width, width, dtype=dtype)
        self.conv_w = normal(self.taps, width, dtype=dtype).t().contiguous()
        self.conv_b = torch.zeros(width, dtype=dtype, device=device)
        keep = torch.linspace(0.9, 0.999, width, device=device)          # a of an open gate
        self.lam = torch.log(torch.expm1(-torch.log(keep) / 8))

    def pools(self, slots):
        """Empty states for that many requests: the convolution's and the recurrence's."""
        dev = self.norm_w.device
        return torch.zeros(slots, self.taps - 1, self.width, dtype=self.dtype, device=dev), torch.zeros(slots, self.width, device=dev)

    def _gates(self, u):
        return (u @ self.w_gates).chunk(2, 1)

    def prompt(self, x, h, starts, past, slots, pools):
        """Packed prompts (starts: int32, requests + 1 values) that go on from their slots' states."""
        y, h = self.normed(x, h)
        u0, b, at = y @ self.w_in, starts.numel() - 1, slots.long()
        conv, rec = pools[0][at], pools[1][at]
        conv_end, rec_end = torch.empty_like(conv), torch.empty_like(rec)
        u = P.causal_conv1d(u0, self.conv_w, P.causal_conv1d_desc_for(u0, self.conv_w, b, silu=False), bias=self.conv_b, seq_starts=starts,
                            initial_state=conv, final_state=conv_end)
        r, i = self._gates(u)
        s = P.gated_recurrence(u, r, i, self.lam, P.gated_recurrence_desc_for(u, r, i, b), seq_starts=starts, initial_state=rec, final_state=rec_end)
        pools[0][at], pools[1][at] = conv_end, rec_end
        return s @ self.w_out, h

    def token(self, x, h, past, slots, pools):
        y, h = self.normed(x, h)
        u0 = y @ self.w_in
        u = P.causal_conv1d_step(u0, self.conv_w, pools[0], P.causal_conv1d_desc_for(u0, self.conv_w, silu=False), bias=self.conv_b, slots=slots)
        r, i = self._gates(u)
        s = P.gated_recurrence_step(u, r, i, self.lam, pools[1], P.gated_recurrence_desc_for(u, r, i), slots=slots)
        return s @ self.w_out, h

    def train(self, x, h, sequences):
        """The output, the new residual, and a function from their gradients
        to the gradients of x (and h: the same) and of the weights."""
        norm = P.rms_norm_desc_for(x.shape[0], self.width, self.dtype, h.dtype)
        y, h = P.add_rms_norm(x, self.norm_w, norm, residual=h)
        u0 = y @ self.w_in
        conv = P.causal_conv1d_desc_for(u0, self.conv_w, sequences, silu=False)
        u = P.causal_conv1d(u0, self.conv_w, conv, bias=self.conv_b)
        r, i = self._gates(u)
        desc = P.gated_recurrence_desc_for(u, r, i, sequences)
        kept = P.gated_recurrence_chunk_states(u, desc)
        s = P.gated_recurrence(u, r, i, self.lam, desc, chunk_states=kept)

        def back(d_out, d_h):
            g = P.gated_recurrence_backward(d_out @ self.w_out.t(), u, r, i, self.lam, desc, chunk_states=kept)
            d_gates = torch.cat((g.dr, g.di), 1)
            c = P.causal_conv1d_backward(g.dx + d_gates @ self.w_gates.t(), u0, self.conv_w, conv, bias=self.conv_b)
            dx, d_norm = P.add_rms_norm_backward(c.dx @ self.w_in.t(), h, self.norm_w, norm, d_residual=d_h)
            return dx, [(self.w_out, s.t() @ d_out), (self.w_gates, u.t() @ d_gates), (self.w_in, y.t() @ c.dx), (self.conv_w, c.dw), (self.conv_b, c.dbias),
                        (self.lam, g.dlam), (self.norm_w, d_norm)]

        return s @ self.w_out, h, back


class Attention(_Layer):
    def __init__(self, width, heads=8, kv_heads=2, window=256, sinks=4, dtype=torch.bfloat16, device="cuda", seed=1):
        normal = _weights(seed, device)
        self.width, self.heads, self.kv, self.window, self.sinks, self.dtype = width, heads, kv_heads, window, sinks, dtype
        self.dim = width // heads
        self.norm_w = torch.ones(width, device=device)
        self.w_qkv, self.w_out = normal(width, (heads + 2 * kv_heads) * self.dim, dtype=dtype), normal(width, width, dtype=dtype)
        self.wq, self.wk = torch.ones(self.dim, device=device), torch.ones(self.dim, device=device)
        self.freqs = 10000.0 ** (-torch.arange(0, self.dim, 2, device=device, dtype=torch.float32) / self.dim)

    def pools(self, slots):
        """Empty caches for that many requests: keys and values of the first tokens and of a window."""
        shape = slots, self.sinks + self.window, self.kv, self.dim
        return torch.empty(shape, dtype=self.dtype, device=self.wq.device), torch.empty(shape, dtype=self.dtype, device=self.wq.device)

    def _qkv(self, y, positions):
        h, kv, dim = self.heads, self.kv, self.dim
        q, k, v = (p.unflatten(1, (-1, dim)) for p in (y @ self.w_qkv).split([h * dim, kv * dim, kv * dim], 1))
        desc = P.qk_norm_rope_desc_for(q, k)
        q2, k2 = P.qk_norm_rope(q, k, self.wq, self.wk, desc, positions=positions, freqs=self.freqs)
        return q, k, v, q2, k2, desc

    def _desc(self, q, k, v, sequences=1):
        return P.window_attention_desc_for(q, k, v, self.window, self.sinks, sequences)

    def prompt(self, x, h, starts, past, slots, pools):
        """Packed prompts of requests that have had `past` tokens (int32)."""
        y, h = self.normed(x, h)
        n, t = starts.numel() - 1, x.shape[0]
        rows = torch.arange(t, dtype=torch.int32, device=x.device)
        of = torch.searchsorted(starts, rows, right=True) - 1
        _, _, v, q, k, _ = self._qkv(y, rows - starts[of] + past[of])
        s = P.window_attention(q, k, v, self._desc(q, k, v, n), seq_starts=starts, k_cache=pools[0], v_cache=pools[1], past=past, slots=slots)
        return s.flatten(1) @ self.w_out, h

    def token(self, x, h, past, slots, pools):
        y, h = self.normed(x, h)
        _, _, v, q, k, _ = self._qkv(y, past)
        s = P.window_attention_step(q, k, v, pools[0], pools[1], past, self._desc(q, k, v), slots=slots)
        return s.flatten(1) @ self.w_out, h

    def train(self, x, h, sequences):
        norm = P.rms_norm_desc_for(x.shape[0], self.width, self.dtype, h.dtype)
        y, h = P.add_rms_norm(x, self.norm_w, norm, residual=h)
        t = x.shape[0]
        positions = torch.arange(t, dtype=torch.int32, device=x.device) % (t // sequences)
        q0, k0, v, q, k, qk = self._qkv(y, positions)
        desc = self._desc(q, k, v, sequences)
        lse = torch.empty(t, self.heads, device=x.device)
        s = P.window_attention(q, k, v, desc, lse=lse)

        def back(d_out, d_h):
            g = P.window_attention_backward((d_out @ self.w_out.t()).unflatten(1, (self.heads, self.dim)), q, k, v, s, lse, desc)
            n = P.qk_norm_rope_backward(g.dq, g.dk, q0, k0, self.wq, self.wk, qk, positions=positions, freqs=self.freqs)
            d_qkv = torch.cat((n.dq.flatten(1), n.dk.flatten(1), g.dv.flatten(1)), 1)
            dx, d_norm = P.add_rms_norm_backward(d_qkv @ self.w_qkv.t(), h, self.norm_w, norm, d_residual=d_h)
            return dx, [(self.w_out, s.flatten(1).t() @ d_out), (self.w_qkv, y.t() @ d_qkv), (self.wq, n.dwq), (self.wk, n.dwk), (self.norm_w, d_norm)]

        return s.flatten(1) @ self.w_out, h, back


def prompt(layers, x, h, starts, past, slots, pools):
    for layer, pool in zip(layers, pools):
        x, h = layer.prompt(x, h, starts, past, slots, pool)
    return x, h


def token(layers, x, h, past, slots, pools):
    for layer, pool in zip(layers, pools):
        x, h = layer.token(x, h, past, slots, pool)
    return x, h


def gradients(layers, x, h, target, sequences):
    """The mean square of output - target over equal sequences, and the
    gradients of x, h (the same) and every layer's weights."""
    backs = []
    for layer in layers:
        x, h, back = layer.train(x, h, sequences)
        backs.append(back)
    off = x.float() + h.float() - target
    loss, d_h = off.square().mean(), off * (2 / off.numel())
    d_x, d_h = d_h.to(layers[0].dtype), d_h.to(h.dtype)
    grads = []
    for back in reversed(backs):
        d_h, g = back(d_x, d_h)
        d_x = d_h.to(layers[0].dtype)
        grads = g + grads
    return loss, d_h, grads


def descend(grads, rate):
    for w, d in grads:
        w.add_(d.to(w.dtype), alpha=-rate)


def serve(layers, lengths, split, tokens, seed=1):
    """Prompts of the given lengths in two parts, cut at `split` of each, then
    `tokens` single tokens; the single tokens' outputs, and those of one prompt
    call over all rows."""
    width, dtype = layers[0].width, layers[0].dtype
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = len(lengths)
    rows = [torch.randn(m + tokens, 2, width, generator=g, device="cuda") for m in lengths]   # x and h of each request

    def packed(parts):
        both = torch.cat(parts)
        starts = torch.tensor([0] + [len(p) for p in parts], device="cuda").cumsum(0).to(torch.int32)
        return both[:, 0].to(dtype).contiguous(), both[:, 1].contiguous(), starts

    slots = torch.randperm(n + 3, generator=g, device="cuda")[:n].to(torch.int32)
    pools = [layer.pools(n + 3) for layer in layers]
    past = torch.zeros(n, dtype=torch.int32, device="cuda")
    for parts in ([r[:int(split * m)] for r, m in zip(rows, lengths)], [r[int(split * m):m] for r, m in zip(rows, lengths)]):
        x, h, starts = packed(parts)
        prompt(layers, x, h, starts, past, slots, pools)
        past = past + (starts[1:] - starts[:-1])
    out = []
    for i in range(tokens):
        now = torch.stack([r[m + i] for r, m in zip(rows, lengths)])
        out.append(sum(token(layers, now[:, 0].to(dtype).contiguous(), now[:, 1].contiguous(), past, slots, pools)))
        past = past + 1
    x, h, starts = packed(rows)
    whole = sum(prompt(layers, x, h, starts, torch.zeros_like(past), slots, [layer.pools(n + 3) for layer in layers]))
    want = torch.stack([whole[starts[b] + m:starts[b] + m + tokens] for b, m in enumerate(lengths)], 1)
    return torch.stack(out), want


def main():
    layers = [Recurrence(1024), Attention(1024)]
    got, want = serve(layers, [700, 2, 33, 256], 0.4, 8)
    print("single tokens against one prompt call: relative difference %.2g" % ((got.float() - want.float()).norm() / want.float().norm()))
    g = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn(4 * 512, 1024, generator=g, device="cuda").to(layers[0].dtype)
    h = torch.randn(4 * 512, 1024, generator=g, device="cuda")
    target = torch.roll(h, 1, 0)
    losses = []
    for _ in range(8):
        loss, _, grads = gradients(layers, x, h, target, 4)
        descend(grads, 0.5)
        losses.append(float(loss))
    print("loss " + " ".join("%.4f" % v for v in losses))


if __name__ == "__main__":
    main()
