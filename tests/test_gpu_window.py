"""Attention with a sliding window and first tokens that stay visible, against 64 bits."""

import pytest
import torch

import paper_2609_32197_amd as sp
from tests import _bounded_ref as B
from tests import _cache_ref as R

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32


def run(bt, window, sinks, order="head", workspace=True, out=None, hint=True, **kw):
    t, q = bt.to("cuda", order)
    hints = dict(max_new=max(bt.new), max_kv=max(bt.kv)) if hint else {}
    ws = None
    if workspace:
        n = sp.sparsp_paged_attn_workspace_bytes(t["K_cache"], t["page_table"], bt.T, bt.Hq, **hints,
                                                 window=window, sinks=sinks)
        ws = torch.full((n // 4 + 4,), float("nan"), device="cuda")
    odt = out or bt.dtype
    O = torch.full((bt.Hq, bt.T, bt.d), float("nan"), dtype=odt, device="cuda")
    lse = torch.full((bt.Hq, bt.T), float("nan"), device="cuda")
    r = sp.sparsp_paged_attn(q, **t, **hints, O=O, lse=lse, workspace=ws, window=window, sinks=sinks,
                             out_dtype=sp.BF16 if odt == BF else sp.F32, **kw)
    assert r[0] is O and r[1] is lse
    return O, lse


def check(bt, window, sinks, O, lse, **kw):
    wO, wL, tO, tL = B.attention(bt, window, sinks, out_dtype=O.dtype, **kw)
    R.close(lse, wL, tL, "lse")
    R.close(O, wO, tO, "O")


CASES = [
    # dtype, Hq, H, d, page, new, kv, bad pages
    (BF, 1, 1, 64, 16, (1,), (1,), ()),
    (BF, 4, 1, 128, 16, (1, 1, 1, 1), (15, 16, 17, 330), ()),
    (BF, 8, 2, 128, 64, (1, 0, 1), (700, 50, 0), ()),
    (BF, 6, 2, 64, 32, (5, 1, 9), (3, 200, 9), ()),              # rows that see nothing
    (BF, 14, 2, 80, 16, (3, 2), (1234, 31), ()),
    (BF, 3, 3, 96, 128, (40, 17, 0, 64), (40, 300, 7, 127), ()),
    (BF, 16, 2, 128, 16, (2, 1), (100, 260), ((0, 2), (1, 0), (1, 15))),  # no such pages
    (BF, 2, 2, 8, 256, (70, 33), (70, 1600), ()),
    (BF, 8, 8, 128, 64, (130, 257), (1000, 257), ()),
    (BF, 12, 4, 64, 16, (300, 1, 77), (517, 900, 77), ((0, 5), (0, 30))),
    (BF, 5, 1, 128, 32, (1, 2, 3), (33, 34, 35), ((0, 0), (0, 1))),  # no page at all
    (F, 2, 1, 64, 16, (1, 1), (1, 400), ()),
    (F, 6, 2, 100, 32, (5, 0, 33), (4, 9, 333), ()),
    (F, 8, 1, 128, 64, (2, 1), (1500, 65), ((0, 3), (0, 22))),
    (F, 3, 3, 96, 16, (150,), (700,), ()),
]


@pytest.mark.parametrize("dtype,Hq,H,d,page,new,kv,bad", CASES)
@pytest.mark.parametrize("window,sinks", [(1, 0), (7, 4), (33, 0), (64, 65), (300, 1),
                                          (2 ** 31 - 1, 2 ** 31 - 1)])
def test_window(gpu, dtype, Hq, H, d, page, new, kv, bad, window, sinks):
    bt = R.Batch(41, dtype, Hq, H, d, page, new, kv, tail=2, bad=bad)
    for order, ws, hint in (("head", True, True), ("token", False, True), ("packed", True, False)):
        check(bt, window, sinks, *run(bt, window, sinks, order, ws, hint=hint))


@pytest.mark.parametrize("dtype,Hq,new,kv", [(BF, 8, (1, 3), (4000, 2500)), (BF, 8, (200, 40), (1500, 900)),
                                             (F, 4, (2, 30), (1900, 2100))])
@pytest.mark.parametrize("window,sinks", [(100, 5), (777, 130)])
@pytest.mark.parametrize("page", [16, 128])
def test_pages_out_of_the_window_are_not_read(gpu, dtype, Hq, new, kv, window, sinks, page):
    """Their entries name no page, and the cache holds NaN wherever no token of the window lies."""
    whole = R.Batch(42, dtype, Hq, 2, 64, page, new, kv)
    gone = B.unseen_pages(whole, window, sinks)
    assert gone
    bt = R.Batch(42, dtype, Hq, 2, 64, page, new, kv, bad=gone)
    check(bt, window, sinks, *run(bt, window, sinks))
    # Entries that name a page of NaN.
    nan = next(p for p in range(bt.pages) if torch.isnan(bt.K[p]).all())
    for b, w in gone:
        bt.table[b, w] = nan
    O, lse = run(bt, window, sinks)
    for b, w in gone:
        bt.table[b, w] = -1
    check(bt, window, sinks, O, lse)


@pytest.mark.parametrize("dtype,new", [(BF, (1, 2)), (BF, (400, 3)), (F, (1, 40))])
def test_parts(gpu, dtype, new):
    """Long windows in parts, with every workspace from none to enough, float32 output."""
    window, sinks, kv = 3000, 70, (9000, 3100)
    bt = R.Batch(43, dtype, 8, 2, 128, 64, new, kv)
    t, q = bt.to("cuda")
    kw = dict(window=window, sinks=sinks)
    full = sp.sparsp_paged_attn_workspace_bytes(t["K_cache"], t["page_table"], bt.T, 8, max(new),
                                                max(kv), **kw)
    assert full > 0
    wO, wL, tO, tL = B.attention(bt, window, sinks, out_dtype=F)
    for nbytes in (0, full // 3, full - 1, full, 2 * full):
        ws = torch.full((nbytes + 256,), 255, dtype=torch.uint8, device="cuda")
        O, lse = sp.sparsp_paged_attn(q, **t, max_new=max(new), max_kv=max(kv), out_dtype=sp.F32,
                                      workspace=ws[:nbytes], **kw) if dtype is F else \
            sp.sparsp_paged_attn(q, **t, max_new=max(new), max_kv=max(kv), workspace=ws[:nbytes],
                                 O=torch.empty(8, bt.T, 128, device="cuda"), out_dtype=sp.F32, **kw)
        R.close(O, wO, tO, f"O with {nbytes}")
        R.close(lse, wL, tL, f"lse with {nbytes}")
        assert (ws[nbytes:] == 255).all()


@pytest.mark.parametrize("window,sinks", [(20000, 3), (5, 20000)])
@pytest.mark.parametrize("new", [1, 50])
def test_more_keys_than_a_list_of_pages(gpu, window, sinks, new):
    bt = R.Batch(44, BF, 1, 1, 64, 16, (new,), (50001,))
    check(bt, window, sinks, *run(bt, window, sinks, workspace=False))


def test_window_of_one_is_the_token(gpu):
    """A token that sees itself alone gets its own value, whatever its score."""
    bt = R.Batch(45, BF, 4, 4, 64, 32, (70, 1), (70, 40), std=50.0)
    O, _ = run(bt, 1, 0)
    for b in range(2):
        v, _ = bt.seq(bt.V, b)
        o, n = int(bt.new_off[b]), bt.new[b]
        assert torch.equal(O[:, o:o + n].cpu().double(), v[:, bt.kv[b] - n:])


def test_wide_window_is_the_whole(gpu):
    for dtype, new in ((BF, (1, 3)), (BF, (90, 40)), (F, (5, 1))):
        bt = R.Batch(46, dtype, 8, 2, 64, 16, new, (400, 300))
        t, q = bt.to("cuda")
        wO, wL, tO, tL = R.attention(bt)
        for window, sinks in ((400, 0), (1 << 30, 7), (1, 400)):
            O, lse = sp.sparsp_paged_attn(q, **t, window=window, sinks=sinks)
            R.close(O, wO, tO)
            R.close(lse, wL, tL)


def test_large_scores(gpu):
    """Scores past 2^24: the largest visible one is what the others are relative to."""
    for dtype, new in ((BF, (1, 2)), (BF, (150,))):
        bt = R.Batch(47, dtype, 4, 2, 64, 16, new, (700,) * len(new), std=3e6)
        bt.V.abs_()
        O, lse = run(bt, 90, 20)
        wO, wL, _, tL = B.attention(bt, 90, 20)
        R.close(lse, wL, tL, "lse")
        assert torch.isfinite(O).all()


def test_same_call_twice_in_a_graph_and_on_a_stream(gpu):
    bt = R.Batch(48, BF, 8, 2, 128, 64, (3, 1), (4000, 2500))
    want = run(bt, 1500, 64)
    again = run(bt, 1500, 64)
    assert torch.equal(want[0], again[0]) and torch.equal(want[1], again[1])
    t, q = bt.to("cuda")
    ws = torch.empty(1 << 22, dtype=torch.uint8, device="cuda")
    kw = dict(window=1500, sinks=64, max_new=3, max_kv=4000, workspace=ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    O, lse = sp.sparsp_paged_attn(q, **t, **kw, stream=side)
    side.synchronize()
    assert torch.equal(O, want[0]) and torch.equal(lse, want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        gO, gl = sp.sparsp_paged_attn(q, **t, **kw)
    for _ in range(3):
        gO.zero_()
        sp.sparsp_paged_attn(q, **t, **kw)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(gO, want[0]) and torch.equal(gl, want[1])
        # A replay reads the lengths as they are then.
        t["kv_len"][1] = 1200
        graph.replay()
        torch.cuda.synchronize()
        bt.kv[1] = 1200
        wO, wL, tO, tL = B.attention(bt, 1500, 64)
        R.close(gO, wO, tO)
        t["kv_len"][1] = bt.kv[1] = 2500


def test_refused(gpu):
    bt = R.Batch(49, BF, 2, 2, 64, 16, (1,), (40,))
    t, q = bt.to("cuda")
    for kw in (dict(window=0), dict(window=-3), dict(window=5, sinks=-1)):
        with pytest.raises(sp.SparspError):
            sp.sparsp_paged_attn(q, **t, **kw)
    for kw in (dict(sinks=4), dict(window=5, causal=False), dict(window=1 << 31),
               dict(window=5, sinks=1 << 40)):
        with pytest.raises(ValueError):
            sp.sparsp_paged_attn(q, **t, **kw)
