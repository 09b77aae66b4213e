"""A state space mixer block on the framework's sequence operators.

The block of a token t with residual h and input x, both of width D:

    y, h  = norm(x + h)                      add_rms_norm (serving: 8 bits)
    u, z  = y W_in                           two halves of 2D channels each
    u     = silu(conv(u))                    causal_conv1d, four taps
    r,B,C = u W_x;  dt = r W_dt
    s     = scan(u, dt, A, B, C, D) silu(z)  selective_scan
    x     = s W_out                          the next block's input

``Block.prompt`` runs packed prompts and leaves each request's states in pools,
``Block.token`` moves every request on by one token from those states, and
``Block.train`` is one step of training with the operators' gradients.  Run as
a script it does all three on random weights and says how far single tokens
are from the prompt call over the same rows.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2306_14320_amd as P  # noqa: E402


class Block:
    def __init__(self, width, states=16, taps=4, dtype=torch.bfloat16, device="cuda", seed=0):
        g = torch.Generator(device="cpu").manual_seed(seed)
        inner, rank = 2 * width, max(1, width // 16)
        self.width, self.inner, self.rank, self.states, self.taps, self.dtype = width, inner, rank, states, taps, dtype

        def normal(*shape, scale):
            return (torch.randn(shape, generator=g) * scale).to(device)

        self.norm_w = torch.ones(width, device=device)
        self.w_in = normal(width, 2 * inner, scale=width ** -0.5).to(dtype)
        self.conv_w = normal(inner, taps, scale=taps ** -0.5).to(dtype)
        self.conv_b = torch.zeros(inner, dtype=dtype, device=device)
        self.w_x = normal(inner, rank + 2 * states, scale=inner ** -0.5).to(dtype)
        self.w_dt = normal(rank, inner, scale=rank ** -0.5).to(dtype)
        step = torch.exp(torch.rand(inner, generator=g) * 4.6 - 6.9)
        self.dt_bias = (step + torch.log(-torch.expm1(-step))).to(device)
        self.A = -torch.arange(1, states + 1, dtype=torch.float32, device=device).repeat(inner, 1)
        self.D = torch.ones(inner, device=device)
        self.w_out = normal(inner, width, scale=inner ** -0.5).to(dtype)

    def pools(self, slots):
        """Empty states for that many requests: the convolution's and the scan's."""
        dev = self.norm_w.device
        return (torch.zeros(slots, self.taps - 1, self.inner, dtype=self.dtype, device=dev),
                torch.zeros(slots, self.inner, self.states, device=dev))

    def _projections(self, u):
        low = u @ self.w_x
        n = self.states
        return low[:, :self.rank] @ self.w_dt, low[:, self.rank:self.rank + n].unflatten(1, (1, n)), low[:, self.rank + n:].unflatten(1, (1, n)), low

    def _normed(self, x, h):
        """The serving norm: 8 bits and a scale a row, as a product in 8 bits reads them."""
        desc = P.rms_norm_desc_for(x.shape[0], self.width, self.dtype, h.dtype)
        q, scales, h = P.add_rms_norm_fp8(x, self.norm_w, desc, residual=h)
        return (q.float() * scales).to(self.dtype), h

    def prompt(self, x, h, starts, slots, pools):
        """Packed prompts (starts: int32, requests + 1 values) of new requests;
        their final states go to their slots of the pools."""
        y, h = self._normed(x, h)
        u, z = (y @ self.w_in).chunk(2, 1)
        requests = starts.numel() - 1
        conv_final = torch.empty(requests, self.taps - 1, self.inner, dtype=self.dtype, device=x.device)
        desc = P.causal_conv1d_desc_for(u, self.conv_w, requests)
        u = P.causal_conv1d(u, self.conv_w, desc, bias=self.conv_b, seq_starts=starts, final_state=conv_final)
        dt, B, C, _ = self._projections(u)
        scan_final = torch.empty(requests, self.inner, self.states, device=x.device)
        desc = P.selective_scan_desc_for(u, dt, self.A, B, C, z, requests)
        s = P.selective_scan(u, dt, self.A, B, C, desc, D=self.D, z=z, dt_bias=self.dt_bias, seq_starts=starts, final_state=scan_final)
        pools[0][slots.long()], pools[1][slots.long()] = conv_final, scan_final
        return s @ self.w_out, h

    def token(self, x, h, slots, pools):
        """One token of each request."""
        y, h = self._normed(x, h)
        u, z = (y @ self.w_in).chunk(2, 1)
        u = P.causal_conv1d_step(u, self.conv_w, pools[0], P.causal_conv1d_desc_for(u, self.conv_w), bias=self.conv_b, slots=slots)
        dt, B, C, _ = self._projections(u)
        desc = P.selective_scan_desc_for(u, dt, self.A, B, C, z)
        s = P.selective_scan_step(u, dt, self.A, B, C, pools[1], desc, D=self.D, z=z, dt_bias=self.dt_bias, slots=slots)
        return s @ self.w_out, h

    def train(self, x, h, target, sequences, rate):
        """One step of gradient descent on the mean square of output - target
        over equal sequences; returns the loss before it."""
        t = x.shape[0]
        norm = P.rms_norm_desc_for(t, self.width, self.dtype, h.dtype)
        y, h = P.add_rms_norm(x, self.norm_w, norm, residual=h)
        u0, z = (y @ self.w_in).chunk(2, 1)
        conv = P.causal_conv1d_desc_for(u0, self.conv_w, sequences)
        u = P.causal_conv1d(u0, self.conv_w, conv, bias=self.conv_b)
        dt, B, C, low = self._projections(u)
        scan = P.selective_scan_desc_for(u, dt, self.A, B, C, z, sequences)
        s = P.selective_scan(u, dt, self.A, B, C, scan, D=self.D, z=z, dt_bias=self.dt_bias)
        off = (s @ self.w_out).float() - target
        loss = off.square().mean()

        d_out = (off * (2 / off.numel())).to(self.dtype)
        g = P.selective_scan_backward(d_out @ self.w_out.t(), u, dt, self.A, B, C, scan, D=self.D, z=z, dt_bias=self.dt_bias)
        d_low = torch.cat((g.ddt @ self.w_dt.t(), g.dB.flatten(1), g.dC.flatten(1)), 1)
        du = g.dx + d_low @ self.w_x.t()
        c = P.causal_conv1d_backward(du, u0, self.conv_w, conv, bias=self.conv_b)
        d_in = torch.cat((c.dx, g.dz), 1)
        _, d_norm = P.add_rms_norm_backward(d_in @ self.w_in.t(), h, self.norm_w, norm)
        for w, d in ((self.w_out, s.t() @ d_out), (self.w_x, u.t() @ d_low), (self.w_dt, low[:, :self.rank].t() @ g.ddt),
                     (self.w_in, y.t() @ d_in), (self.conv_w, c.dw), (self.conv_b, c.dbias), (self.A, g.dA), (self.D, g.dD),
                     (self.dt_bias, g.ddt_bias), (self.norm_w, d_norm)):
            w.add_(d.to(w.dtype), alpha=-rate)
        return loss


def serve(block, lengths, tokens, seed=1):
    """Prompts of the given lengths and then `tokens` single tokens each; the
    outputs of the single tokens, and those of one prompt call over all rows."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    requests = len(lengths)
    rows = [torch.randn(n + tokens, 2, block.width, generator=g, device="cuda") for n in lengths]   # x and h of each request

    def packed(parts):
        both = torch.cat(parts)
        starts = torch.tensor([0] + [len(p) for p in parts], device="cuda").cumsum(0).to(torch.int32)
        return both[:, 0].to(block.dtype).contiguous(), both[:, 1].contiguous(), starts

    slots = torch.randperm(requests + 3, generator=g, device="cuda")[:requests].to(torch.int32)
    pools = block.pools(requests + 3)
    x, h, starts = packed([r[:n] for r, n in zip(rows, lengths)])
    block.prompt(x, h, starts, slots, pools)
    out = []
    for i in range(tokens):
        now = torch.stack([r[n + i] for r, n in zip(rows, lengths)])
        out.append(block.token(now[:, 0].to(block.dtype).contiguous(), now[:, 1].contiguous(), slots, pools)[0])
    x, h, starts = packed(rows)
    whole, _ = block.prompt(x, h, starts, slots, block.pools(requests + 3))
    want = torch.stack([whole[starts[b] + n:starts[b] + n + tokens] for b, n in enumerate(lengths)], 1)
    return torch.stack(out), want


def main():
    block = Block(1024)
    got, want = serve(block, [700, 1, 33, 256], 8)
    print("single tokens against one prompt call: relative difference %.2g" % ((got.float() - want.float()).norm() / want.float().norm()))
    g = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn(4 * 512, 1024, generator=g, device="cuda").to(block.dtype)
    h = torch.randn(4 * 512, 1024, generator=g, device="cuda")
    target = torch.roll(x.float(), 1, 0)
    losses = [float(block.train(x, h, target, 4, 0.5)) for _ in range(8)]
    print("loss " + " ".join("%.4f" % v for v in losses))


if __name__ == "__main__":
    main()
