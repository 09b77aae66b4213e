"""Inputs of the selective scan's tests: sizes and sequences where the kernels
can go wrong, with NaN in the rows that no sequence holds."""
import torch

import paper_2306_14320_amd as P
from seq_reference import equal_starts

DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16

# (dtype, channels, states, groups, starts or (tokens, sequences), states given, gate, D, softplus with bias, aligned)
SCAN = [
    (F32, 1, 1, 1, (1, 1), False, False, False, False, True),
    (F32, 6, 4, 1, (5, 1), True, True, True, True, True),
    (BF16, 130, 16, 1, (70, 2), False, True, True, True, True),
    (F32, 257, 16, 1, (33, 1), True, True, True, True, False),           # an odd number of channels
    (BF16, 96, 16, 3, [0, 0, 1, 5, 37, 37, 38, 101], True, True, True, True, True),    # empty and one-token sequences
    (F32, 60, 24, 4, [3, 10, 70, 71, 75], True, True, False, True, True),              # rows in front that no sequence holds
    (BF16, 42, 8, 2, [0, 200], True, False, True, True, False),
    (F32, 40, 32, 1, (150, 3), False, True, True, False, True),
    (F32, 20, 50, 2, [0, 9, 64, 140], True, True, True, True, True),
    (BF16, 24, 128, 1, (90, 1), True, True, True, True, True),
    (F32, 8, 3, 2, (4, 4), True, True, True, True, True),                # sequences of one token
    (BF16, 16, 16, 1, (600, 1), True, True, True, True, True),           # many chunks of one sequence
    (F32, 34, 12, 1, [0, 130, 131, 500, 500, 700], True, True, True, True, True),
]
SCAN_IDS = ["%s-d%d-n%d-g%d-%d" % (str(c[0])[6:], c[1], c[2], c[3], i) for i, c in enumerate(SCAN)]


class ScanCase:
    def __init__(self, dtype, d, n, groups, rows, states, gate, skip, soft, aligned, seed=0):
        g = torch.Generator().manual_seed(2000 + seed + d)
        if isinstance(rows, tuple):
            self.tokens, self.seqs = rows
            self.starts, self.dense = equal_starts(*rows), True
        else:
            self.starts, self.dense = rows, False
            self.tokens, self.seqs = rows[-1] + 3, len(rows) - 1
        self.dtype, self.d, self.n, self.groups, self.softplus = dtype, d, n, groups, soft
        t = self.tokens

        def normal(*shape, scale=1.0, dtype=dtype):
            return (torch.randn(shape, generator=g, dtype=torch.float64) * scale).to(dtype)

        pad = 0 if aligned else 1
        self.lo, self.hi = self.starts[0], self.starts[-1]
        self.outside = [i for i in range(t) if not self.lo <= i < self.hi]
        self.xz = normal(t, 2 * d + pad)
        self.low = normal(t, 3 + pad + 2 * groups * n)
        dt = normal(t, d + pad, scale=0.7)
        if not soft:
            dt = dt.abs() * 0.2
        self.dtw = dt
        self.dy = normal(t, d)
        for rows_ in (self.xz, self.low, self.dtw, self.dy):
            rows_[self.outside] = float("nan")
        self.has_z = gate
        self.A = -(0.2 + 3 * torch.rand(d, n, generator=g))
        self.D = normal(d, dtype=F32) if skip else None
        self.dt_bias = normal(d, dtype=F32) - 1 if soft else None
        self.init = normal(self.seqs, d, n, dtype=F32) if states else None
        self.d_final = normal(self.seqs, d, n, dtype=F32) if states else None

    def _views(self, xz, low, dtw):
        gn, d = self.groups * self.n, self.d
        off = low.shape[1] - 2 * gn
        return (xz[:, :d], dtw[:, :d], low[:, off:off + gn].unflatten(1, (self.groups, self.n)),
                low[:, off + gn:].unflatten(1, (self.groups, self.n)), xz[:, d:2 * d] if self.has_z else None)

    def device(self):
        """Positional inputs (x, dt, A, B, C), the descriptor and the keywords of a call."""
        x, dt, B, C, z = self._views(self.xz.to(DEV), self.low.to(DEV), self.dtw.to(DEV))
        dev = lambda v: None if v is None else v.to(DEV)   # noqa: E731
        desc = P.selective_scan_desc_for(x, dt, self.A, B, C, z, self.seqs, softplus=self.softplus)
        kw = dict(D=dev(self.D), z=z, dt_bias=dev(self.dt_bias), initial_state=dev(self.init),
                  seq_starts=None if self.dense else torch.tensor(self.starts, dtype=torch.int32, device=DEV))
        return (x, dt, self.A.to(DEV), B, C), desc, kw

    def clean(self, v):
        v = v.clone()
        v[self.outside] = 0
        return v.double()

    def doubles(self):
        """(x, dt, A, B, C, D, z, dt_bias, init) in 64 bits, rows outside zero."""
        x, dt, B, C, z = self._views(self.xz, self.low, self.dtw)
        dbl = lambda v: None if v is None else v.double()   # noqa: E731
        return (self.clean(x), self.clean(dt), self.A.double(), self.clean(B), self.clean(C), dbl(self.D),
                None if z is None else self.clean(z), dbl(self.dt_bias), dbl(self.init))
