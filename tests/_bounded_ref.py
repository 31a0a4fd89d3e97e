"""The bounded cache's operators in 64 bits on the CPU.

Tolerances are those of _cache_ref. Over a cache of 4-bit values each product of a score, and of an
output, is a sum over up to three bfloat16 terms of one factor, so that sums have up to three times
as many float32 additions; what three terms leave of a float32 is below 2^-26 of it, two of a
probability 2^-17.

An exponential or a product below the smallest normal float32, 2^-126, may become 0: each of the N
products of an output is then off by up to 2^-126 (1 + |v|). Values of 4 bits are often 0, and such
a product can be all that a channel has.
"""

import math

import torch

from tests import _cache_ref as R

U = R.U


def seen_by_window(bt, b, window, sinks, causal=True):
    """[n, kv]: which cached tokens each new token of sequence b sees."""
    n, m = bt.new[b], bt.kv[b]
    p, t = m - n + torch.arange(n)[:, None], torch.arange(m)[None]
    seen = (t <= p) if causal else torch.ones(n, m, dtype=torch.bool)
    return seen if window is None else seen & ((t > p - window) | (t < sinks))


def attention(bt, window=None, sinks=0, scale=None, out_dtype=None, causal=True, terms=1):
    """As R.attention, with a window: (O, lse, tolerance of O, tolerance of lse)."""
    scale = 1.0 / math.sqrt(bt.d) if scale is None else scale
    uo = R.HALF[out_dtype or bt.dtype]
    r = 2.0 ** -8 if bt.dtype == torch.bfloat16 else 0.0
    O = torch.full((bt.Hq, bt.T, bt.d), float("nan"), dtype=torch.float64)
    L = torch.full((bt.Hq, bt.T), float("nan"), dtype=torch.float64)
    tO, tL = O.clone(), L.clone()
    for b in range(bt.B):
        n, N, o = bt.new[b], bt.kv[b], int(bt.new_off[b])
        v, _ = bt.seq(bt.V, b)
        seen = seen_by_window(bt, b, window, sinks, causal)
        for h, (x, e) in enumerate(R.scores(bt, b, scale, causal)):
            x, e = x.masked_fill(~seen, -math.inf), terms * e
            vv = v[h // (bt.Hq // bt.H)]
            lse = torch.logsumexp(x, 1) if N else torch.full((n,), -math.inf, dtype=torch.float64)
            p = torch.exp(x - torch.where(lse == -math.inf, 0.0, lse)[:, None])
            O[h, o:o + n], L[h, o:o + n] = p @ vv, lse
            A = p @ vv.abs()
            tO[h, o:o + n] = (A * (r + 4 * e + 2 * (terms * N + 64) * U + 2.0 ** -18)[:, None]
                              + uo * O[h, o:o + n].abs()
                              + 2.0 ** -126 * (N + vv.abs().sum(0)))
            tL[h, o:o + n] = 2 * e + (N + 64) * U + 2.0 ** -19 + 4 * U * lse.abs().clamp(max=1e30)
    return O, L, tO, tL


def unseen_pages(bt, window, sinks):
    """(b, page index) of the pages that no new token of their sequence sees."""
    out = set()
    for b in range(bt.B):
        seen = seen_by_window(bt, b, window, sinks).any(0)
        for w in range(-(-bt.kv[b] // bt.page)):
            if not seen[w * bt.page:(w + 1) * bt.page].any():
                out.add((b, w))
    return out


GRID = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)


def quantise(x):
    """(codes [..., d / 2], scales [..., d / 32]) uint8 of x [..., d] float64, by distances."""
    shape = x.shape
    x = x.double().reshape(-1, 32)
    bad = ~torch.isfinite(x).all(1)
    x = torch.where(bad[:, None], 0.0, x)
    top = x.abs().amax(1)
    e = torch.where(top > 0, torch.frexp(top)[1] - 3, -125).clamp(-125, 125)
    # (exact: a power of two; above 8 a distance's rounding could make 6 as near as 0)
    m = (x.abs() * torch.exp2(-e.double())[:, None]).clamp(max=8.0)
    order = torch.tensor([0, 2, 4, 6, 1, 3, 5, 7])  # the even codes first
    code = order[(m[..., None] - GRID[order]).abs().argmin(-1)]
    code = code + 8 * torch.signbit(x).long()
    code[bad] = 0
    scale = torch.where(bad, 255, e + 127)
    code = code.reshape(shape)
    return ((code[..., 0::2] | (code[..., 1::2] << 4)).to(torch.uint8),
            scale.reshape(shape[:-1] + (shape[-1] // 32,)).to(torch.uint8))


def values(codes, scales):
    """What codes [..., d / 2] with scales [..., d / 32] stand for, float64."""
    c = torch.stack((codes & 15, codes >> 4), -1).flatten(-2).long()
    x = GRID[c & 7] * torch.where(c > 7, -1.0, 1.0)
    unit = torch.exp2(scales.double() - 127).masked_fill(scales == 255, float("nan"))
    return (x.reshape(x.shape[:-1] + (-1, 32)) * unit[..., None]).flatten(-2)


class Batch4(R.Batch):
    """A batch whose K and V are what a 4-bit cache holds. Rows of no token have the scale of NaN."""

    def __init__(self, *args, **kw):
        super().__init__(*args, **kw)
        self.four = []
        for x in (self.K, self.V):
            codes, scales = quantise(x)
            junk = torch.randint(0, 256, codes.shape, generator=self.g, dtype=torch.uint8)
            codes = torch.where(torch.isnan(x[..., :1]), junk, codes)
            x.copy_(values(codes, scales))
            self.four += [codes, scales.transpose(-1, -2).contiguous()]

    def to4(self, device, layout="head"):
        """(Cache4, table, offsets and lengths, Q)."""
        import paper_2609_32197_amd as sp
        return (sp.Cache4(*(x.to(device) for x in self.four)),
                dict(page_table=self.table.to(device), new_off=self.new_off.to(device),
                     kv_len=self.kv_len.to(device)), R.laid_out(self.Q, layout, device))
