"""Attention of few rows over a bf16 cache: probabilities keep 16 bits, so float32 outputs are as good as
a float32 softmax's, but for 2^-16 of the sum of absolute values, and bf16 outputs are those rounded."""

import pytest
import torch

import paper_2609_32197_amd as sp
from tests import _cache_ref as R
from tests.test_gpu_paged_attn import BF, F, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("Hq,H,d,page,new,kv,bad", [
    (4, 1, 128, 16, (1, 1, 1, 1), (15, 16, 17, 33), ()),
    (8, 2, 128, 64, (1, 0, 1), (3000, 50, 0), ()),
    (14, 2, 80, 16, (2, 2), (1234, 31), ()),
    (16, 2, 128, 16, (2, 1), (100, 260), ((0, 2), (1, 0))),
    (8, 1, 64, 128, (4, 3), (2100, 70), ()),
    (3, 3, 8, 256, (30, 1), (30, 600), ()),
])
@pytest.mark.parametrize("workspace", [False, True])
def test_few_rows(gpu, Hq, H, d, page, new, kv, bad, workspace):
    bt = R.Batch(81, BF, Hq, H, d, page, new, kv, tail=1, bad=bad)
    wO, _, _, _ = R.attention(bt, out_dtype=F)
    tol = torch.full_like(wO, float("nan"))
    for b in range(bt.B):
        n, N, o = bt.new[b], bt.kv[b], int(bt.new_off[b])
        v, _ = bt.seq(bt.V, b)
        for h, (x, e) in enumerate(R.scores(bt, b, d ** -0.5, True)):
            lse = torch.logsumexp(x, 1) if N else torch.full((n,), -float("inf"), dtype=x.dtype)
            p = torch.exp(x - torch.where(lse == -float("inf"), 0.0, lse)[:, None])
            A = p @ v[h // (Hq // H)].abs()
            # The float32 tolerance of _cache_ref, and 2^-16 for the two halves of a probability.
            tol[h, o:o + n] = A * (2.0 ** -16 + 4 * e + 2 * (N + 64) * R.U + 2.0 ** -18)[:, None]
    O, _ = run(bt, "token", workspace, out=F)
    R.close(O, wO, tol + R.U * wO.abs(), "O, float32")
    O, _ = run(bt, "token", workspace)
    R.close(O, wO, tol + R.HALF[BF] * (wO.abs() + tol), "O")
