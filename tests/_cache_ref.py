"""Batches for the paged-cache tests, and the operators in 64 bits on the CPU.

Everything a kernel may not read is NaN: cache rows behind a sequence's tokens, pages of no
sequence, token columns behind the last sequence.

Tolerances. u = 2^-24 is half a float32 step, uo half a step of the output type. A score is a
sum of d products in float32 in an unknown order, scaled: it is off by at most
  e = scale (d + 16) u max_t sum_c |q_c k_tc|     (the 16 covers scale, log2(e), the subtraction
                                                    of the running max and the exponential)
so a probability is off by 2 e + 2^-20 of itself (2^-20: the exponential unit's own error, twice),
and by 2^-8 more where it is rounded to bfloat16. Sums over N keys are off by N u of the sum of
absolute values. With A = sum_t p_t |v_t| (p normalised)
  |O - ref|   <= A (2^-8 [bf16] + 4 e + 2 (N + 64) u + 2^-18) + uo |O|
  |lse - ref| <= 2 e + (N + 64) u + 2^-19 + 4 u |lse|
  |w - ref|   <= sum_r p_r (2 e_r + 4 u (|lse_r| + 1) + 2^-20) + (R + 64) u sum_r p_r
"""

from __future__ import annotations

import math

import torch

U = 2.0 ** -24
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: U}


class Batch:
    """Sequences with new[b] new tokens and kv[b] cached ones (the new included)."""

    def __init__(self, seed, dtype, Hq, H, d, page, new, kv, tail=0, spare=2, bad=(), width=None,
                 std=1.0, device="cpu"):
        g = torch.Generator().manual_seed(seed)
        self.dtype, self.Hq, self.H, self.d, self.page = dtype, Hq, H, d, page
        self.new, self.kv, self.B, self.bad = list(new), list(kv), len(new), set(bad)
        self.T = sum(new) + tail
        need = [-(-k // page) for k in kv]
        self.width = width or max(1, max(need))
        self.pages = sum(need) + spare
        ids = torch.randperm(self.pages, generator=g).tolist()
        # Entries that no token needs hold numbers of no page, of either sign.
        table = torch.tensor([[-1, self.pages + 7, -2 ** 31, 2 ** 31 - 1][w % 4]
                              for w in range(self.B * self.width)], dtype=torch.int64)
        table = table.view(self.B, self.width)
        at = 0
        for b in range(self.B):
            for w in range(need[b]):
                if (b, w) not in self.bad:
                    table[b, w] = ids[at]
                at += 1
        self.table = table.to(torch.int32)
        off = [0]
        for n in new:
            off.append(off[-1] + n)
        self.new_off = torch.tensor(off, dtype=torch.int32)
        self.kv_len = torch.tensor(kv, dtype=torch.int32)
        shape = (self.pages, H, page, d)
        self.K = torch.full(shape, float("nan"), dtype=dtype)
        self.V = torch.full(shape, float("nan"), dtype=dtype)
        self.weights = torch.full(shape[:3], float("nan"))
        for b, t, p, r in self.places():
            if p is not None:
                self.K[p, :, r] = torch.randn(H, d, generator=g).to(dtype)
                self.V[p, :, r] = torch.randn(H, d, generator=g).to(dtype)
                self.weights[p, :, r] = torch.rand(H, generator=g)
        self.Q = (torch.randn(Hq, self.T, d, generator=g) * std).to(dtype)
        self.Q[:, off[-1]:] = float("nan")
        self.g = g

    def place(self, b, t):
        """(page, row) of cached token t, page None where the table has none."""
        w = t // self.page
        p = int(self.table[b, w]) if w < self.width else -1
        return (p if 0 <= p < self.pages else None), t % self.page

    def places(self):
        for b in range(self.B):
            for t in range(self.kv[b]):
                p, r = self.place(b, t)
                yield b, t, p, r

    def seq(self, x, b):
        """(rows [H, kv, ...] of a paged tensor in 64 bits, which of them exist)."""
        at = [self.place(b, t) for t in range(self.kv[b])]
        live = torch.tensor([p is not None for p, _ in at], dtype=torch.bool)
        rows = [x[p, :, r].double() if p is not None else torch.zeros_like(x[0, :, 0]).double()
                for p, r in at]
        return (torch.stack(rows, 1) if rows else x.new_zeros((self.H, 0) + x.shape[3:]).double(),
                live)

    def to(self, device, layout="head"):
        """The call's tensors on the device. layout: "head" [H, T, d], "token" (a view of [T, H, d]),
        "packed" (columns of a wider projection)."""
        return dict(K_cache=self.K.to(device), V_cache=self.V.to(device),
                    page_table=self.table.to(device), new_off=self.new_off.to(device),
                    kv_len=self.kv_len.to(device)), laid_out(self.Q, layout, device)


def laid_out(x, layout, device):
    if layout == "head":
        return x.to(device)
    h, n, d = x.shape
    if layout == "token":
        return x.transpose(0, 1).contiguous().to(device).transpose(0, 1)
    wide = torch.full((n, h + 3, d + 16), float("nan"), dtype=x.dtype)
    wide[:, 2:2 + h, 16:] = x.transpose(0, 1)
    return wide.to(device)[:, 2:2 + h, 16:].transpose(0, 1)


def scores(bt, b, scale, causal):
    """Per query head: scores [n, kv] with -inf where unseen, and e (see above) [n]."""
    k, live = bt.seq(bt.K, b)
    n, m, o = bt.new[b], bt.kv[b], int(bt.new_off[b])
    q = bt.Q[:, o:o + n].double()
    t = torch.arange(m)
    last = torch.full((n,), m) if not causal else m - n + torch.arange(n)
    seen = (t[None] <= last[:, None]) & live[None]
    out = []
    for h in range(bt.Hq):
        kk = k[h // (bt.Hq // bt.H)]
        x = (q[h] @ kk.T * scale).masked_fill(~seen, -math.inf)
        mag = (q[h].abs() @ kk.abs().T).masked_fill(~seen, 0.0)
        top = mag.amax(1) if m else torch.zeros(n, dtype=torch.float64)
        out.append((x, scale * (bt.d + 16) * U * top))
    return out


def attention(bt, scale=None, causal=True, out_dtype=None):
    """(O, lse, tolerance of O, tolerance of lse), NaN in the columns of no sequence."""
    scale = 1.0 / math.sqrt(bt.d) if scale is None else scale
    uo = HALF[out_dtype or bt.dtype]
    O = torch.full((bt.Hq, bt.T, bt.d), float("nan"), dtype=torch.float64)
    L = torch.full((bt.Hq, bt.T), float("nan"), dtype=torch.float64)
    tO, tL = O.clone(), L.clone()
    for b in range(bt.B):
        n, N, o = bt.new[b], bt.kv[b], int(bt.new_off[b])
        v, _ = bt.seq(bt.V, b)
        for h, (x, e) in enumerate(scores(bt, b, scale, causal)):
            vv = v[h // (bt.Hq // bt.H)]
            lse = torch.logsumexp(x, 1) if N else torch.full((n,), -math.inf, dtype=torch.float64)
            p = torch.exp(x - torch.where(lse == -math.inf, 0.0, lse)[:, None])
            O[h, o:o + n], L[h, o:o + n] = p @ vv, lse
            A = p @ vv.abs()
            r = (2.0 ** -8 if bt.dtype == torch.bfloat16 else 0.0)
            tO[h, o:o + n] = (A * (r + 4 * e + 2 * (N + 64) * U + 2.0 ** -18)[:, None]
                              + uo * O[h, o:o + n].abs())
            tL[h, o:o + n] = 2 * e + (N + 64) * U + 2.0 ** -19 + 4 * U * lse.abs().clamp(max=1e30)
    return O, L, tO, tL


def weights(bt, lse, scale=None, causal=True):
    """Per sequence (w [H, kv], tolerance); lse float32 [Hq, T] as the kernel gets it."""
    scale = 1.0 / math.sqrt(bt.d) if scale is None else scale
    G = bt.Hq // bt.H
    out = []
    for b in range(bt.B):
        n, m, o = bt.new[b], bt.kv[b], int(bt.new_off[b])
        w = torch.zeros(bt.H, m, dtype=torch.float64)
        tol = torch.zeros(bt.H, m, dtype=torch.float64)
        for h, (x, e) in enumerate(scores(bt, b, scale, causal)):
            l = lse[h, o:o + n].double()
            dead = l == -math.inf
            p = torch.exp(x - torch.where(dead, 0.0, l)[:, None])
            p[dead] = 0.0
            w[h // G] += p.sum(0)
            tol[h // G] += (p * (2 * e + 4 * U * (l.abs().clamp(max=1e30) + 1)
                                 + 2.0 ** -20)[:, None]).sum(0)
        out.append((w, tol + (n * G + 64) * U * w))
    return out


def rotate(x, pos, inv_freq, rot, layout, axis_pairs, factor=1.0, inverse=False):
    """(y, tolerance before rounding) of x [heads, tokens, d]: |x1|, |x2| times twelve half steps
    (reduced angle pi, sine and cosine 4, factor 1, products and sum 3)."""
    y, tol = x.double().clone(), torch.zeros(x.shape, dtype=torch.float64)
    P, p = rot // 2, 0
    for axis, count in enumerate(axis_pairs):
        for _ in range(count):
            i, j = (p, p + P) if layout == "half" else (2 * p, 2 * p + 1)
            a = pos[axis].double() * float(inv_freq[p])
            c, s = torch.cos(a) * factor, torch.sin(a) * factor * (-1.0 if inverse else 1.0)
            x1, x2 = x[..., i].double(), x[..., j].double()
            y[..., i], y[..., j] = x1 * c - x2 * s, x1 * s + x2 * c
            t = 12 * U * abs(factor) * (x1.abs() + x2.abs())
            tol[..., i], tol[..., j] = t, t
            p += 1
    half = HALF[x.dtype]
    return y, torch.where(tol > 0, tol + half * (y.abs() + tol), tol)


def close(got, want, tol, what=""):
    got, want = got.detach().cpu().double(), want.double()
    same = (got == want) | (torch.isnan(got) & torch.isnan(want))
    bad = ~(same | ((got - want).abs() <= tol))
    assert not bad.any(), (f"{what}: {int(bad.sum())} of {bad.numel()} off, first at "
                           f"{bad.nonzero()[0].tolist()}: {got[bad][0]} for {want[bad][0]}, "
                           f"tolerance {tol.expand_as(bad)[bad][0]}")
