"""The bounded cache's operators in 64 bits on the CPU: attention with a window."""

import math

import torch

from tests import _cache_ref as R

U = R.U


def seen_by_window(bt, b, window, sinks):
    """[n, kv]: which cached tokens each new token of sequence b sees."""
    n, m = bt.new[b], bt.kv[b]
    p, t = m - n + torch.arange(n)[:, None], torch.arange(m)[None]
    return (t <= p) & ((t > p - window) | (t < sinks))


def attention(bt, window, sinks, scale=None, out_dtype=None, rounded=None):
    """As R.attention with a window: (O, lse, tolerance of O, tolerance of lse). rounded: what a
    probability is off by (2^-8 where it enters a product as one bfloat16)."""
    scale = 1.0 / math.sqrt(bt.d) if scale is None else scale
    uo = R.HALF[out_dtype or bt.dtype]
    r = rounded if rounded is not None else 2.0 ** -8 if bt.dtype == torch.bfloat16 else 0.0
    O = torch.full((bt.Hq, bt.T, bt.d), float("nan"), dtype=torch.float64)
    L = torch.full((bt.Hq, bt.T), float("nan"), dtype=torch.float64)
    tO, tL = O.clone(), L.clone()
    for b in range(bt.B):
        n, N, o = bt.new[b], bt.kv[b], int(bt.new_off[b])
        v, _ = bt.seq(bt.V, b)
        seen = seen_by_window(bt, b, window, sinks)
        for h, (x, e) in enumerate(R.scores(bt, b, scale, True)):
            x = x.masked_fill(~seen, -math.inf)
            vv = v[h // (bt.Hq // bt.H)]
            lse = torch.logsumexp(x, 1) if N else torch.full((n,), -math.inf, dtype=torch.float64)
            p = torch.exp(x - torch.where(lse == -math.inf, 0.0, lse)[:, None])
            O[h, o:o + n], L[h, o:o + n] = p @ vv, lse
            A = p @ vv.abs()
            tO[h, o:o + n] = (A * (r + 4 * e + 2 * (N + 64) * U + 2.0 ** -18)[:, None]
                              + uo * O[h, o:o + n].abs())
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
