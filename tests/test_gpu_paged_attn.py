"""Attention of new tokens over the paged cache against 64 bits."""

import math

import pytest
import torch

import paper_2609_32197_amd as sp
from tests import _cache_ref as R

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32


def run(bt, order="head", workspace=True, out=None, hint=True, **kw):
    t, q = bt.to("cuda", order)
    hints = dict(max_new=max(bt.new), max_kv=max(bt.kv)) if hint else {}
    ws = None
    if workspace:
        n = sp.sparsp_paged_attn_workspace_bytes(t["K_cache"], t["page_table"], bt.T, bt.Hq, **hints)
        ws = torch.full((n // 4 + 4,), float("nan"), device="cuda")
    odt = out or bt.dtype
    O = torch.full((bt.Hq, bt.T, bt.d), float("nan"), dtype=odt, device="cuda")
    lse = torch.full((bt.Hq, bt.T), float("nan"), device="cuda")
    r = sp.sparsp_paged_attn(q, **t, **hints, O=O, lse=lse, workspace=ws,
                             out_dtype=sp.BF16 if odt == BF else sp.F32, **kw)
    assert r[0] is O and r[1] is lse
    return O, lse


def check(bt, O, lse, **kw):
    wO, wL, tO, tL = R.attention(bt, out_dtype=O.dtype, **kw)
    R.close(lse, wL, tL, "lse")
    R.close(O, wO, tO, "O")


CASES = [
    # dtype, Hq, H, d, page, new, kv, bad pages
    (BF, 1, 1, 64, 16, (1,), (1,), ()),
    (BF, 4, 1, 128, 16, (1, 1, 1, 1), (15, 16, 17, 33), ()),
    (BF, 8, 2, 128, 64, (1, 0, 1), (700, 50, 0), ()),
    (BF, 6, 2, 64, 32, (5, 1, 9), (3, 200, 9), ()),              # rows that see nothing
    (BF, 14, 2, 80, 16, (3, 2), (1234, 31), ()),
    (BF, 3, 3, 96, 128, (40, 17, 0, 64), (40, 300, 7, 127), ()),
    (BF, 16, 2, 128, 16, (2, 1), (100, 260), ((0, 2), (1, 0))),  # pages that do not exist
    (BF, 2, 2, 8, 256, (70, 33), (70, 600), ()),
    (BF, 8, 8, 128, 64, (130, 257), (1000, 257), ()),
    (BF, 12, 4, 64, 16, (300, 1, 77), (517, 900, 77), ((0, 5),)),
    (BF, 5, 1, 128, 32, (1, 2, 3), (33, 34, 35), ((0, 0), (0, 1))),  # no page at all
    (F, 2, 1, 64, 16, (1, 1), (1, 40), ()),
    (F, 6, 2, 100, 32, (5, 0, 33), (4, 9, 333), ()),
    (F, 8, 1, 128, 64, (2, 1), (1500, 65), ((0, 3),)),
    (F, 4, 4, 4, 16, (20, 3), (50, 3), ()),
    (F, 3, 3, 96, 16, (150,), (700,), ()),
]


@pytest.mark.parametrize("dtype,Hq,H,d,page,new,kv,bad", CASES)
@pytest.mark.parametrize("causal", [True, False])
def test_attention(gpu, dtype, Hq, H, d, page, new, kv, bad, causal):
    bt = R.Batch(21, dtype, Hq, H, d, page, new, kv, tail=2, bad=bad)
    for order, ws, hint in (("head", True, True), ("token", False, True), ("packed", True, False)):
        check(bt, *run(bt, order, ws, causal=causal, hint=hint), causal=causal)


@pytest.mark.parametrize("new,kv", [((1, 1), (5000, 700)), ((3, 2), (1, 6011)), ((40,), (4100,))])
@pytest.mark.parametrize("dtype", [BF, F])
def test_split_keys(gpu, dtype, new, kv):
    """Long caches in parts: with every workspace from none to enough, and float32 output."""
    bt = R.Batch(22, dtype, 8, 2, 128, 64, new, kv, tail=1)
    check(bt, *run(bt, out=F), causal=True)
    t, q = bt.to("cuda")
    full = sp.sparsp_paged_attn_workspace_bytes(t["K_cache"], t["page_table"], bt.T, 8, max(new),
                                                max(kv))
    assert full > 0
    for nbytes in (0, 15, full // 3, full - 1, full, 2 * full):
        ws = torch.full((nbytes + 256,), 255, dtype=torch.uint8, device="cuda")
        O, lse = sp.sparsp_paged_attn(q, **t, max_new=max(new), max_kv=max(kv),
                                      workspace=ws[:nbytes])
        n = sum(new)
        wO, wL, tO, tL = R.attention(bt)
        R.close(O[:, :n], wO[:, :n], tO[:, :n], f"O with {nbytes}")
        R.close(lse[:, :n], wL[:, :n], tL[:, :n], f"lse with {nbytes}")
        assert (ws[nbytes:] == 255).all()


@pytest.mark.parametrize("d,page,bad", [(64, 16, ()), (128, 256, ((0, 3), (0, 64), (0, 80)))])
def test_long_cache_without_workspace(gpu, d, page, bad):
    """More keys than one list of page numbers holds, and a last tile of one key."""
    bt = R.Batch(33, BF, 1, 1, d, page, (50,), (2 * 16384 + 1,), bad=bad)
    check(bt, *run(bt, workspace=False), causal=True)


def test_hints_only_size_the_launch(gpu):
    """Hints below the truth, above it, and none: right every time."""
    bt = R.Batch(23, BF, 4, 2, 64, 16, (90, 1, 35), (2100, 600, 40))
    t, q = bt.to("cuda")
    wO, wL, tO, tL = R.attention(bt)
    ws = torch.empty(1 << 22, dtype=torch.uint8, device="cuda")
    for hint in (dict(max_new=1, max_kv=1), dict(max_new=7, max_kv=10000), dict(max_kv=513),
                 dict(max_new=100000), {}):
        O, lse = sp.sparsp_paged_attn(q, **t, **hint, workspace=ws)
        R.close(lse, wL, tL, f"lse with {hint}")
        R.close(O, wO, tO, f"O with {hint}")


@pytest.mark.parametrize("dtype", [BF, F])
def test_large_and_tiny_scores(gpu, dtype):
    """Scores in the hundreds (a probability of one), and a scale that flattens them."""
    bt = R.Batch(24, dtype, 4, 2, 64, 16, (6, 40), (300, 45), std=60.0)
    check(bt, *run(bt), causal=True)
    check(bt, *run(bt, softmax_scale=1e-4), scale=1e-4)


def test_lengths_beyond_the_table(gpu):
    """A kv_len past the table's width is cut to it."""
    bt = R.Batch(25, BF, 2, 2, 64, 16, (1, 1), (64, 48), width=4)
    t, q = bt.to("cuda")
    t["kv_len"] = torch.tensor([2 ** 31 - 1, 48], dtype=torch.int32, device="cuda")
    O, lse = sp.sparsp_paged_attn(q, **t)
    wO, wL, tO, tL = R.attention(bt)
    R.close(lse, wL, tL)
    R.close(O, wO, tO)


def test_strided_output_and_no_lse(gpu):
    bt = R.Batch(26, BF, 6, 3, 128, 32, (4, 9), (100, 60))
    t, q = bt.to("cuda", "token")
    wide = torch.full((bt.T, 8, 144), 7.0, dtype=BF, device="cuda")
    O = wide[:, 1:7, :128].transpose(0, 1)
    r, lse = sp.sparsp_paged_attn(q, **t, O=O, want_lse=False)
    assert lse is None
    wO, _, tO, _ = R.attention(bt)
    R.close(O, wO, tO)
    assert (wide[:, 0] == 7).all() and (wide[:, 7] == 7).all() and (wide[:, :, 128:] == 7).all()


def test_same_call_twice_is_the_same(gpu):
    bt = R.Batch(27, BF, 8, 1, 128, 64, (3, 1), (4000, 2500))
    a, b = run(bt), run(bt)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_merges_with_another_cache(gpu):
    """Two caches attended apart and joined by sparsp_lse_merge: the attention over both."""
    H, T, d, block = 2, 64, 64, 64
    bt = R.Batch(28, F, H, H, d, 16, (T,), (200,))
    k, _ = bt.seq(bt.K, 0)
    v, _ = bt.seq(bt.V, 0)
    parts = []
    for lo, hi in ((0, 90), (90, 200)):
        pt = R.Batch(29, F, H, H, d, 16, (T,), (hi - lo,))
        pt.Q = bt.Q
        for s in range(hi - lo):
            p, r = pt.place(0, s)
            pt.K[p, :, r], pt.V[p, :, r] = k[:, lo + s].float(), v[:, lo + s].float()
        parts.append(run(pt, causal=False))
    geom = sp.Geometry(H, T, d, block, 0, 1, sp.F32)
    (O, lse), (O2, lse2) = parts
    sp.sparsp_lse_merge(geom, (0, H), O, lse, O2, lse2)
    wO, wL, tO, tL = R.attention(bt, causal=False)
    R.close(O, wO, 2 * tO)
    R.close(lse, wL, 2 * tL)


def test_agrees_with_block_attention(gpu):
    """A cache of a whole sequence, every block kept: sparsp_block_sparse_attn's result."""
    H, L, d, block = 2, 512, 128, 128
    g = torch.Generator().manual_seed(30)
    q, k, v = (torch.randn(H, L, d, generator=g).to(BF).cuda() for _ in range(3))
    geom = sp.Geometry(H, L, d, block, 0, 4, sp.BF16)
    _, _, sc = sp.sparsp_block_scores(geom, q, k)
    mask, sel = sp.sparsp_topk_mask(geom, sc, 4)
    o = sp.sparsp_demand_union_gather(geom, mask, k, v)
    O1, l1 = sp.sparsp_block_sparse_attn(geom, q, sel, o["slot_of"], o["K_packed"], o["V_packed"],
                                         out_dtype=sp.F32)
    Kc = torch.zeros(8, H, 64, d, dtype=BF, device="cuda")
    Vc = torch.zeros_like(Kc)
    table = torch.arange(8, dtype=torch.int32, device="cuda").flip(0).view(1, 8).contiguous()
    off = torch.tensor([0, L], dtype=torch.int32, device="cuda")
    kv = torch.tensor([L], dtype=torch.int32, device="cuda")
    sp.sparsp_paged_append(k, v, Kc, Vc, table, off, kv)
    O2, l2 = sp.sparsp_paged_attn(q, Kc, Vc, table, off, kv, causal=False, out_dtype=sp.F32)
    # Each is within 2^-8 A of the exact output, A < 4 for a mean of unit normals.
    assert (O1 - O2).abs().max() < 2 * 2.0 ** -8 * 4
    assert (l1 - l2).abs().max() < 1e-4


def test_offsets_past_32_bits(gpu):
    """A page whose K starts past 2^31 elements (and 2^32 bytes) of the cache."""
    H, d, page = 4, 128, 256
    pages = 2 ** 31 // (H * page * d) + 3
    Kc = torch.zeros(pages, H, page, d, dtype=BF, device="cuda")
    Vc = torch.zeros_like(Kc)
    bt = R.Batch(31, BF, 8, H, d, page, (2, 1), (300, 20), spare=0)
    table = (bt.table.long() + pages - bt.pages).to(torch.int32)
    table[bt.table < 0] = -1
    table[bt.table >= bt.pages] = -1
    Kc[pages - bt.pages:] = bt.K.cuda()
    Vc[pages - bt.pages:] = bt.V.cuda()
    O, lse = sp.sparsp_paged_attn(bt.Q.cuda(), Kc, Vc, table.cuda(), bt.new_off.cuda(),
                                  bt.kv_len.cuda())
    wO, wL, tO, tL = R.attention(bt)
    R.close(lse, wL, tL)
    R.close(O, wO, tO)
    w = torch.zeros(pages, H, page, device="cuda")
    sp.sparsp_paged_weights(bt.Q.cuda(), lse, Kc, table.cuda(), bt.new_off.cuda(),
                            bt.kv_len.cuda(), w)
    for b, (want, tol) in enumerate(R.weights(bt, lse.cpu())):
        for s in range(bt.kv[b]):
            p, r = bt.place(b, s)
            R.close(w[p + pages - bt.pages, :, r], want[:, s], tol[:, s])


def test_another_stream(gpu):
    bt = R.Batch(32, BF, 8, 2, 64, 16, (1, 3), (800, 90))
    t, q = bt.to("cuda")
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    O = torch.empty(8, bt.T, 64, dtype=BF, device="cuda")
    lse = torch.empty(8, bt.T, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    sp.sparsp_paged_attn(q, **t, O=O, lse=lse, workspace=ws, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    wO, wL, tO, tL = R.attention(bt)
    R.close(lse, wL, tL)
    R.close(O, wO, tO)


def test_more_row_tiles_than_a_grid_holds(gpu):
    """2^26 rows of one key head are 2^21 tiles of 32 rows."""
    n, kv, d = 1 << 25, 40, 4
    g = torch.Generator(device="cuda").manual_seed(31)
    Q = torch.randn((2, n, d), generator=g, device="cuda")
    K, V = (torch.randn((3, 1, 16, d), generator=g, device="cuda") for _ in range(2))
    i32 = dict(dtype=torch.int32, device="cuda")
    O, lse = sp.sparsp_paged_attn(Q, K, V, torch.tensor([[2, 0, 1]], **i32),
                                  torch.tensor([0, n], **i32), torch.tensor([kv], **i32),
                                  causal=False)
    k, v = (x.cpu()[[2, 0, 1], 0].reshape(48, d)[:kv].double() for x in (K, V))
    at = torch.cat([torch.arange(0, n, 9973, device="cuda"), torch.arange(n - 40, n, device="cuda")])
    q = Q[:, at].cpu().double()
    s = 0.5 * (q[:, :, None, :] * k).sum(-1)
    p = torch.softmax(s, -1)
    e = 0.5 * (d + 16) * R.U * (q.abs()[:, :, None, :] * k.abs()).sum(-1).amax(-1)
    tL = 2 * e + (kv + 64) * R.U + 2.0 ** -19 + 4 * R.U * torch.logsumexp(s, -1).abs()
    R.close(lse[:, at], torch.logsumexp(s, -1), tL, "lse")
    w = (p[..., None] * v).sum(-2)
    A = (p[..., None] * v.abs()).sum(-2)
    tO = A * (4 * e[..., None] + 2 * (kv + 64) * R.U + 2.0 ** -18) + R.U * w.abs()
    R.close(O[:, at], w, tO, "O")
    assert torch.isfinite(O).all()


@pytest.mark.parametrize("dtype,Hq,H,d", [(BF, 4, 2, 128), (BF, 3, 1, 80), (BF, 6, 1, 64), (F, 4, 1, 64)])
@pytest.mark.parametrize("causal", [True, False])
def test_long_prompts_among_many_single_tokens(gpu, dtype, Hq, H, d, causal):
    """More than 64 sequences, of which two have many tokens and some none."""
    new = (1, 0, 1, 5, 300) + (1,) * 60 + (0, 0, 417, 2, 1, 0)
    kv = tuple(n if b % 7 == 1 else n + 40 * (b % 5) + 900 * (b % 23 == 4) for b, n in enumerate(new))
    bt = R.Batch(33, dtype, Hq, H, d, 16, new, kv, tail=3, bad=((4, 2),))
    for ws, hint in ((True, True), (False, True), (True, False)):
        check(bt, *run(bt, "token", ws, causal=causal, hint=hint), causal=causal)
