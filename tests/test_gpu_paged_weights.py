"""Attention weight per cached token against 64 bits."""

import math

import pytest
import torch

import paper_2609_32197_amd as sp
from tests import _cache_ref as R
from tests.test_gpu_paged_attn import CASES, BF, F

pytestmark = pytest.mark.gpu


def expect(bt, w, lse, start, **kw):
    """w [pages, H, page] after the call, from `start` (None: overwritten)."""
    want = bt.weights.double()
    tol = torch.zeros_like(want)
    for b, (x, t) in enumerate(R.weights(bt, lse, **kw)):
        for s in range(bt.kv[b]):
            p, r = bt.place(b, s)
            if p is not None:
                base = start[p, :, r].double() if start is not None else 0.0
                want[p, :, r] = x[:, s] + base
                tol[p, :, r] = t[:, s] + (R.U * want[p, :, r].abs() if start is not None else 0.0)
    R.close(w, want, tol, "weights")


@pytest.mark.parametrize("dtype,Hq,H,d,page,new,kv,bad", CASES)
@pytest.mark.parametrize("causal", [True, False])
def test_weights(gpu, dtype, Hq, H, d, page, new, kv, bad, causal):
    bt = R.Batch(41, dtype, Hq, H, d, page, new, kv, tail=2, bad=bad)
    lse = R.attention(bt, causal=causal)[1].float()
    for order, acc, hint in (("head", True, True), ("token", False, True), ("packed", True, False)):
        t, q = bt.to("cuda", order)
        del t["V_cache"]
        hints = dict(max_new=max(new), max_kv=max(kv)) if hint else {}
        w = bt.weights.cuda()
        r = sp.sparsp_paged_weights(q, lse.cuda(), weights=w, causal=causal, accumulate=acc, **t,
                                    **hints)
        assert r is w
        expect(bt, w, lse, bt.weights if acc else None, causal=causal)


def test_weights_sum_to_the_rows(gpu):
    """A row's weights sum to one: the total is the number of rows that see a token."""
    bt = R.Batch(42, BF, 6, 2, 128, 32, (70, 1, 4), (1000, 333, 2))
    t, q = bt.to("cuda")
    _, lse = sp.sparsp_paged_attn(q, **t)
    del t["V_cache"]
    w = torch.zeros(bt.pages, 2, 32, device="cuda")
    sp.sparsp_paged_weights(q, lse, weights=w, **t)
    rows = 6 * (70 + 1 + 2)  # two of the last sequence's four tokens lie before its first
    # Each row's sum is off by the exponentials' and lse's relative error, below 2^-16 here.
    assert abs(float(w.double().sum()) - rows) < rows * 2.0 ** -16


def test_rows_of_minus_infinity_add_nothing(gpu):
    bt = R.Batch(43, F, 2, 2, 64, 16, (3,), (40,))
    t, q = bt.to("cuda")
    del t["V_cache"]
    lse = R.attention(bt)[1].float()
    lse[0, 1] = -math.inf
    w = bt.weights.cuda()
    sp.sparsp_paged_weights(q, lse.cuda(), weights=w, accumulate=False, **t)
    expect(bt, w, lse, None)


def test_hints_below_the_truth(gpu):
    bt = R.Batch(44, BF, 4, 2, 64, 16, (33, 2), (900, 100))
    t, q = bt.to("cuda")
    del t["V_cache"]
    lse = R.attention(bt)[1].float()
    for hint in (dict(max_new=1, max_kv=1), dict(max_kv=100000), {}):
        w = bt.weights.cuda()
        sp.sparsp_paged_weights(q, lse.cuda(), weights=w, **t, **hint)
        expect(bt, w, lse, bt.weights)


def test_no_new_tokens_writes_zero(gpu):
    bt = R.Batch(45, BF, 2, 1, 64, 16, (0, 0), (20, 0))
    t, q = bt.to("cuda")
    del t["V_cache"]
    w = bt.weights.cuda()
    sp.sparsp_paged_weights(q, torch.empty(2, 0, device="cuda"), weights=w, **t)
    R.close(w, bt.weights.double(), torch.zeros(1))
    sp.sparsp_paged_weights(q, torch.empty(2, 0, device="cuda"), weights=w, accumulate=False, **t)
    expect(bt, w, torch.empty(2, 0), None)


@pytest.mark.parametrize("dtype,Hq,H,d,page,new,kv,bad",
                         [c for c in CASES if sum(c[5]) * c[1] // c[2] > 32] +
                         [(F, 4, 1, 8, 16, (600, 1, 0), (700, 30, 9), ((0, 3),)),
                          (BF, 4, 1, 8, 16, (600, 1, 0), (700, 30, 9), ((0, 3),))])
@pytest.mark.parametrize("causal", [True, False])
def test_weights_of_a_wide_table(gpu, dtype, Hq, H, d, page, new, kv, bad, causal):
    """Room for long sequences makes a launch of many workgroups, however short they are."""
    bt = R.Batch(46, dtype, Hq, H, d, page, new, kv, tail=2, bad=bad, width=40000 // page)
    lse = R.attention(bt, causal=causal)[1].float()
    t, q = bt.to("cuda", "token")
    del t["V_cache"]
    w = bt.weights.cuda()
    sp.sparsp_paged_weights(q, lse.cuda(), weights=w, causal=causal, **t)
    expect(bt, w, lse, bt.weights, causal=causal)
    # The same with the true lengths known, which few workgroups cover.
    w = bt.weights.cuda()
    sp.sparsp_paged_weights(q, lse.cuda(), weights=w, causal=causal, accumulate=False, max_kv=max(kv),
                            max_new=max(new), **t)
    expect(bt, w, lse, None, causal=causal)
