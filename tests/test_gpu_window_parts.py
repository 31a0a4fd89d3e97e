"""Attention with a window over bf16 rows, many row tiles: the last round of workgroups in parts."""

import pytest
import torch

import paper_2609_32197_amd as sp
from tests import _bounded_ref as B
from tests import _cache_ref as R

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32

CASES = [
    # d, Hq, H, page, new, kv, window, sinks, row tiles of the last round, parts of each
    (128, 64, 8, 64, (700, 500), (1300, 2900), 2500, 40, 24 * 8, 2),
    (128, 128, 8, 128, (520,), (3500,), 2048, 4, 1 * 8, 2),
    (128, 64, 8, 64, (1030,), (6000,), 5000, 130, 1 * 8, 5),
    (96, 64, 8, 32, (1030,), (3100,), 2500, 7, 1 * 8, 2),
    (64, 96, 8, 16, (900, 500), (3000, 2200), 2500, 40, 74 * 8, 2),
]


@pytest.mark.parametrize("d,Hq,H,page,new,kv,window,sinks,tiles,parts", CASES)
def test_last_round_in_parts(gpu, d, Hq, H, page, new, kv, window, sinks, tiles, parts):
    """With every workspace and a max_new below the truth, against 64 bits for some heads, against whole
    tiles for all, and the same twice. Pages that no row sees have no entry."""
    seen = dict(window=window, sinks=sinks)
    one = R.Batch(61, BF, 1, H, d, page, new, kv)
    bt = R.Batch(61, BF, Hq, H, d, page, new, kv, tail=3, bad=B.unseen_pages(one, window, sinks))
    t, q = bt.to("cuda")
    hints = dict(max_new=max(new), max_kv=max(kv))
    full = sp.sparsp_paged_attn_workspace_bytes(t["K_cache"], t["page_table"], bt.T, Hq, **hints, **seen)
    # The partial rows of those tiles and nothing else: the launch has such a round.
    assert full == tiles * 128 * parts * (d + 2) * 4

    def run(nbytes, **kw):
        ws = torch.full((nbytes + 256,), 255, dtype=torch.uint8, device="cuda")
        O = torch.full((Hq, bt.T, d), float("nan"), device="cuda")
        lse = torch.full((Hq, bt.T), float("nan"), device="cuda")
        sp.sparsp_paged_attn(q, **t, **{**hints, **kw}, O=O, lse=lse, workspace=ws[:nbytes],
                             out_dtype=sp.F32, **seen)
        assert (ws[nbytes:] == 255).all()
        return O, lse, (ws[:nbytes] != 255).any()

    live, G = sum(new), Hq // H
    some = [0, G - 1, Hq - 1]
    sub = R.Batch(61, BF, 1, H, d, page, new, kv, tail=3, bad=bt.bad)
    want = []
    for h in some:
        k = h // G
        sub.Hq, sub.H, sub.Q = 1, 1, bt.Q[h:h + 1]
        sub.K, sub.V = bt.K[:, k:k + 1], bt.V[:, k:k + 1]
        want.append(B.attention(sub, window, sinks, out_dtype=F))
    whole, wholeL, _ = run(0)
    # What either of two calls may be off by, of all heads: R's tolerances with A below max |v| and
    # |q|.|k| below the largest lengths' product.
    top, far = float(torch.nan_to_num(bt.V).abs().max()), float(wholeL[:, :live].abs().max())
    length = [float(torch.nan_to_num(x).float().norm(dim=-1).max()) for x in (bt.Q, bt.K)]
    e, N = d ** -0.5 * (d + 16) * R.U * length[0] * length[1], max(kv)
    tO = top * (2.0 ** -8 + 4 * e + 2 * (N + 64) * R.U + 2.0 ** -18 + R.U)
    tL = 2 * e + (N + 64) * R.U + 2.0 ** -19 + 4 * R.U * far
    for nbytes, used in ((0, False), (full - 16, None), (full, True), (2 * full, True)):
        O, L, wrote = run(nbytes)
        if used is not None:
            assert bool(wrote) == used
        again = run(nbytes)
        few = run(nbytes, max_new=max(new) - 200)
        assert torch.equal(O[:, :live], again[0][:, :live]) and torch.equal(L[:, :live], again[1][:, :live])
        for got, lse in ((O, L), (few[0], few[1])):
            # Columns of no sequence stay as they were.
            assert torch.isnan(got[:, live:]).all() and torch.isnan(lse[:, live:]).all()
            for h, (wO, wL, uO, uL) in zip(some, want):
                R.close(got[h:h + 1], wO, uO, f"O of head {h} with {nbytes}")
                R.close(lse[h:h + 1], wL, uL, f"lse of head {h} with {nbytes}")
            assert (got[:, :live] - whole[:, :live]).abs().max() <= 2 * tO
            assert (lse[:, :live] - wholeL[:, :live]).abs().max() <= 2 * tL


@pytest.mark.parametrize("d,Hq,H,page,new,kv,window,sinks,tiles,parts", CASES[:1] + CASES[4:])
def test_in_a_graph(gpu, d, Hq, H, page, new, kv, window, sinks, tiles, parts):
    """Captured with its join, replayed with other lengths, against the same call outside."""
    bt = R.Batch(62, BF, Hq, H, d, page, new, kv)
    t, q = bt.to("cuda")
    ws = torch.empty(tiles * 128 * parts * (d + 2) * 4, dtype=torch.uint8, device="cuda")
    kw = dict(max_new=max(new), max_kv=max(kv), window=window, sinks=sinks, workspace=ws)
    sp.sparsp_paged_attn(q, **t, **kw)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        O, lse = sp.sparsp_paged_attn(q, **t, **kw)
    for less in (0, 5, 700):
        t["kv_len"].copy_(torch.tensor([k - less for k in kv], dtype=torch.int32))
        want = sp.sparsp_paged_attn(q, **t, **kw)
        O.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(O, want[0]) and torch.equal(lse, want[1])
