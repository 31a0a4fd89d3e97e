"""A cache held in 4 bits: what is written into it, read back, and its attention, against 64 bits."""

import pytest
import torch

import paper_2609_32197_amd as sp
from tests import _bounded_ref as B
from tests import _cache_ref as R

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32


# ---------------------------------------------------------------------------
# writing and reading
# ---------------------------------------------------------------------------


def lengths(new, kv):
    off = [0]
    for n in new:
        off.append(off[-1] + n)
    return (torch.tensor(off, dtype=torch.int32, device="cuda"),
            torch.tensor(kv, dtype=torch.int32, device="cuda"))


def write(x, page=16):
    """Codes [tokens, d / 2] and scales [tokens, d / 32] that V = x [tokens, d] gets, and it read back."""
    n, d = x.shape
    need = -(-n // page)
    cache = sp.Cache4.zeros(need, 1, page, d)
    table = torch.arange(need, dtype=torch.int32, device="cuda").view(1, -1)
    off, kv = lengths([n], [n])
    v = x.cuda()[None].contiguous()
    sp.sparsp_paged_append4(torch.zeros_like(v), v, cache, table, off, kv)
    k, back = sp.sparsp_paged_read4(cache, table, off, kv, n, dtype=x.dtype)
    assert (k == 0).all()
    codes = cache.V.view(need * page, d // 2)[:n].cpu()
    scales = cache.V_scales.transpose(-1, -2).reshape(need * page, d // 32)[:n].cpu()
    return codes, scales, back[0].cpu()


def same(x):
    codes, scales, back = write(x)
    want = B.quantise(x)
    assert torch.equal(scales, want[1])
    assert torch.equal(codes, want[0])
    v = B.values(*want)
    assert torch.equal(torch.nan_to_num(back.double(), nan=-7.0), torch.nan_to_num(v, nan=-7.0))


@pytest.mark.parametrize("dtype", [BF, F])
def test_codes_of_every_border(gpu, dtype):
    """Every border of the grid, one step of the type to either side, and the values themselves, with
    the largest of the 32 from just above a power of two to just below the next, both signs."""
    edge = torch.tensor([0.0, 0.25, 0.5, 0.75, 1.0, 1.25, 1.5, 1.75, 2.0, 2.5, 3.0, 3.5, 4.0, 5.0, 6.0])
    if dtype is BF:  # (as integers, a step is one)
        bits = edge.to(BF).view(torch.int16)
        edge = torch.cat([(bits + s).clamp(min=0).view(BF).float() for s in (-1, 0, 1)])
    else:
        bits = edge.view(torch.int32)
        edge = torch.cat([(bits + s).clamp(min=0).view(F) for s in (-1, 0, 1)])
    rows = []
    for top in (4.0, 4.03125, 5.0, 6.0, 7.0, 7.96875):
        for sign in (1.0, -1.0):
            for part in edge.split(31):
                row = torch.zeros(32)
                row[0], row[1:1 + len(part)] = -sign * top, sign * part
                rows.append(row)
    x = torch.stack(rows)
    # Every power of two that a float32 scale can have and a few at its ends.
    for power in (0, -3, 100, 124, -121, -124, -127, -128, -129, -130):
        same((x.double() * 2.0 ** power).to(dtype))


@pytest.mark.parametrize("dtype", [BF, F])
def test_codes_of_special_rows(gpu, dtype):
    x = torch.randn(40, 64, generator=torch.Generator().manual_seed(3))
    x[0] = 0.0
    x[1] = -0.0
    x[2, 5] = float("inf")
    x[3, 40] = float("nan")
    x[4, 3] = -float("inf")
    x[5] = torch.finfo(dtype).max
    x[6] = torch.finfo(dtype).tiny
    x[7] = 2.0 ** -140
    x[8, :32] = 2.0 ** 127
    x[9, 32:] *= 2.0 ** 60
    same(x.to(dtype))


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("d,page", [(32, 16), (64, 256), (96, 64), (128, 32)])
def test_codes_of_random_rows(gpu, dtype, d, page):
    x = torch.randn(3001, d, generator=torch.Generator().manual_seed(4)) * torch.logspace(-20, 20, 3001)[:, None]
    codes, scales, back = write(x.to(dtype), page)
    want = B.quantise(x.to(dtype))
    assert torch.equal(codes, want[0]) and torch.equal(scales, want[1])
    assert torch.equal(back.double(), B.values(*want))


APPENDS = [
    # dtype, Hq, H, d, page, new, kv, rot, layout, axes, bad pages
    (BF, 4, 2, 128, 64, (1, 1, 1), (1, 64, 130), 128, "half", 1, ()),
    (BF, 3, 1, 64, 16, (5, 0, 21), (5, 9, 40), 64, "interleaved", 1, ((2, 1),)),
    (BF, 8, 8, 96, 32, (7, 3), (100, 2), 48, "half", 1, ()),       # places before the first token
    (BF, 2, 2, 32, 256, (300,), (500,), 8, "half", 1, ()),         # pairs four apart
    (BF, 2, 2, 128, 16, (33, 2), (33, 90), 20, "half", 1, ()),     # and ten
    (BF, 2, 1, 64, 16, (17,), (40,), 6, "half", 1, ()),            # and three
    (BF, 5, 5, 128, 128, (40, 17), (40, 300), 126, "interleaved", 3, ()),
    (BF, 40, 8, 128, 64, (1100,), (1100,), 128, "half", 3, ()),
    (BF, 2, 2, 64, 16, (2100,), (2100,), 64, "interleaved", 1, ()),  # several tokens a workgroup
    (F, 4, 2, 64, 16, (1, 30), (77, 30), 64, "half", 1, ()),
    (F, 3, 3, 128, 64, (9, 2), (9, 200), 32, "interleaved", 1, ((1, 3),)),
    (F, 2, 1, 96, 32, (50,), (64,), 96, "half", 3, ()),
]


@pytest.mark.parametrize("dtype,Hq,H,d,page,new,kv,rot,layout,axes,bad", APPENDS)
@pytest.mark.parametrize("order", ["head", "token", "packed"])
def test_append(gpu, dtype, Hq, H, d, page, new, kv, rot, layout, axes, bad, order):
    bt = B.Batch4(51, dtype, Hq, H, d, page, new, kv, tail=2, bad=bad)
    cache, t, q = bt.to4("cuda", order)
    before = [x.clone() for x in cache.tensors]
    n = bt.T
    K = torch.randn(H, n, d, generator=bt.g).to(dtype)
    V = torch.randn(H, n, d, generator=bt.g).to(dtype)
    pairs = rot // 2
    axis = (pairs,) if axes == 1 else (pairs - 2 * (pairs // 3), pairs // 3, pairs // 3)
    wide = torch.int64 if order == "token" else torch.int32
    pos = torch.randint(-50, 200000, (axes, n), generator=bt.g).to(wide)
    pos[:, 0] = 0
    f = torch.pow(10000.0, -2.0 * torch.arange(pairs, dtype=torch.float64) / rot).float()
    rotary = sp.Rotary(rot, layout, axis, 1.25)
    out = sp.sparsp_paged_append4(R.laid_out(K, order, "cuda"), R.laid_out(V, order, "cuda"), cache,
                                  **t, rotary=rotary, positions=pos.cuda(), inv_freq=f.cuda(), Q=q)
    live = int(bt.new_off[-1])
    y, tol = R.rotate(bt.Q[:, :live], pos[:, :live], f, rot, layout, axis, 1.25)
    R.close(out[:, :live], y, tol, "Q")
    # K in 64 bits, not rounded to its type.
    k64, _ = R.rotate(K[:, :live].double().to(F).to(dtype), pos[:, :live], f, rot, layout, axis, 1.25)
    want = [x.cpu().clone() for x in before]
    for b in range(bt.B):
        for i in range(new[b]):
            slot, col = kv[b] - new[b] + i, int(bt.new_off[b]) + i
            if slot < 0 or bt.place(b, slot)[0] is None:
                continue
            p, r = bt.place(b, slot)
            for x, (codes, scales) in ((k64, want[:2]), (V.double(), want[2:])):
                c, s = B.quantise(x[:, col])
                codes[p, :, r], scales[p, :, :, r] = c, s
    for name, got, w in zip(("K", "K scales", "V", "V scales"), cache.tensors, want):
        assert torch.equal(got.cpu(), w), name
    # In place, and the same codes.
    again = sp.Cache4(*(x.clone() for x in before))
    r = sp.sparsp_paged_append4(K.cuda(), V.cuda(), again, **t, rotary=rotary, positions=pos.cuda(),
                                inv_freq=f.cuda(), Q=q, Q_out=q)
    assert r is q and torch.equal(q[:, :live], out[:, :live])
    assert all(torch.equal(a, b) for a, b in zip(again.tensors, cache.tensors))
    # Columns of no sequence keep their Q.
    assert torch.isnan(q[:, live:]).all()
    # What is read is what stands there, in either type, and 0 where there is no place.
    for dt in (BF, F):
        rk = torch.full((H, n, d), 7.0, dtype=dt, device="cuda")
        rv = R.laid_out(torch.full((H, n, d), 7.0, dtype=dt), order, "cuda")
        sp.sparsp_paged_read4(cache, **t, tokens=n, K=rk, V=rv)
        for got, codes, scales in ((rk, *want[:2]), (rv, *want[2:])):
            assert (got[:, live:] == 7).all()
            w = torch.zeros(H, live, d, dtype=torch.float64)
            for b in range(bt.B):
                for i in range(new[b]):
                    slot = kv[b] - new[b] + i
                    p, r = bt.place(b, slot) if slot >= 0 else (None, 0)
                    if p is not None:
                        w[:, int(bt.new_off[b]) + i] = B.values(codes[p, :, r], scales[p, :, :, r])
            assert torch.equal(got[:, :live].cpu().double(), w)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("factor", [2.0 ** 127, 2.0 ** -140])
def test_rotations_of_any_factor(gpu, layout, factor):
    """K beyond what float32 holds: its codes keep their signs, at the largest and smallest scale."""
    g = torch.Generator().manual_seed(6)
    K = torch.randn(2, 50, 64, generator=g) * torch.logspace(-30, 37, 50)[:, None]
    bt = B.Batch4(52, F, 2, 2, 64, 16, (50,), (50,))
    cache, t, _ = bt.to4("cuda")
    pos = torch.randint(0, 9000, (1, 50), generator=g, dtype=torch.int32)
    f = torch.pow(10000.0, -torch.arange(32, dtype=torch.float64) / 32).float()
    sp.sparsp_paged_append4(K.cuda(), K.cuda(), cache, **t, rotary=sp.Rotary(64, layout, (32,), factor),
                            positions=pos.cuda(), inv_freq=f.cuda())
    y, _ = R.rotate(K, pos, f, 64, layout, (32,), factor)
    got = [x.cpu() for x in cache.tensors]
    for i in range(50):
        p, r = bt.place(0, i)
        codes, scales = B.quantise(y[:, i])
        assert torch.equal(got[0][p, :, r], codes) and torch.equal(got[1][p, :, :, r], scales), i


def test_read_of_a_whole_cache(gpu):
    """new_off as the running sums of kv_len: every cached token, in order."""
    bt = B.Batch4(52, BF, 2, 2, 64, 16, (1, 1, 1), (37, 5, 64))
    cache, t, _ = bt.to4("cuda")
    off, kv = lengths(bt.kv, bt.kv)
    k, v = sp.sparsp_paged_read4(cache, t["page_table"], off, kv, sum(bt.kv))
    at = 0
    for b in range(3):
        for got, x in ((k, bt.K), (v, bt.V)):
            assert torch.equal(got[:, at:at + bt.kv[b]].cpu().double(), bt.seq(x, b)[0])
        at += bt.kv[b]


# ---------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------


def run(bt, order="head", workspace=True, out=None, hint=True, **kw):
    cache, t, q = bt.to4("cuda", order)
    hints = dict(max_new=max(bt.new), max_kv=max(bt.kv)) if hint else {}
    ws = None
    if workspace:
        w = {k: kw[k] for k in ("window", "sinks") if k in kw}
        n = sp.sparsp_paged_attn4_workspace_bytes(cache, t["page_table"], bt.T, bt.Hq, **hints, **w,
                                                  dtype=bt.dtype)
        ws = torch.full((n // 4 + 4,), float("nan"), device="cuda")
    odt = out or bt.dtype
    O = torch.full((bt.Hq, bt.T, bt.d), float("nan"), dtype=odt, device="cuda")
    lse = torch.full((bt.Hq, bt.T), float("nan"), device="cuda")
    r = sp.sparsp_paged_attn4(q, cache, **t, **hints, O=O, lse=lse, workspace=ws,
                              out_dtype=sp.BF16 if odt == BF else sp.F32, **kw)
    assert r[0] is O and r[1] is lse
    return O, lse


def check(bt, O, lse, **kw):
    wO, wL, tO, tL = B.attention(bt, out_dtype=O.dtype, terms=3, **kw)
    R.close(lse, wL, tL, "lse")
    R.close(O, wO, tO, "O")


CASES = [
    # dtype, Hq, H, d, page, new, kv, bad pages
    (BF, 1, 1, 64, 16, (1,), (1,), ()),
    (BF, 4, 1, 128, 16, (1, 1, 1, 1), (15, 16, 17, 330), ()),
    (BF, 8, 2, 128, 64, (1, 0, 1), (700, 50, 0), ()),
    (BF, 6, 2, 64, 32, (5, 1, 9), (3, 200, 9), ()),              # rows that see nothing
    (BF, 14, 2, 96, 16, (2, 1), (1234, 31), ()),
    (BF, 3, 3, 96, 128, (40, 17, 0, 64), (40, 300, 7, 127), ()),
    (BF, 16, 2, 128, 16, (2, 1), (100, 260), ((0, 2), (1, 0), (1, 15))),  # no such pages
    (BF, 2, 2, 32, 256, (70, 33), (70, 1600), ()),
    (BF, 8, 1, 32, 16, (3,), (100,), ()),
    (BF, 8, 8, 128, 64, (130, 257), (1000, 257), ()),
    (BF, 12, 4, 64, 16, (300, 1, 77), (517, 900, 77), ((0, 5), (0, 30))),
    (BF, 5, 1, 128, 32, (1, 2, 3), (33, 34, 35), ((0, 0), (0, 1))),  # no page at all
    (F, 2, 1, 64, 16, (1, 1), (1, 400), ()),
    (F, 6, 2, 96, 32, (5, 0, 33), (4, 9, 333), ()),
    (F, 8, 1, 128, 64, (2, 1), (1500, 65), ((0, 3), (0, 22))),
    (F, 3, 3, 32, 16, (150,), (700,), ()),
    (F, 16, 2, 128, 16, (1, 40), (90, 60), ()),
]


@pytest.mark.parametrize("dtype,Hq,H,d,page,new,kv,bad", CASES)
@pytest.mark.parametrize("seen", [dict(), dict(causal=False), dict(window=1), dict(window=33, sinks=5),
                                  dict(window=200, sinks=65)])
def test_attention(gpu, dtype, Hq, H, d, page, new, kv, bad, seen):
    bt = B.Batch4(53, dtype, Hq, H, d, page, new, kv, tail=2, bad=bad)
    for order, ws, hint in (("head", True, True), ("token", False, True), ("packed", True, False)):
        check(bt, *run(bt, order, ws, hint=hint, **seen), **seen)


@pytest.mark.parametrize("dtype,new", [(BF, (1, 2)), (BF, (400, 3)), (F, (1, 40))])
@pytest.mark.parametrize("seen", [dict(), dict(window=3000, sinks=70)])
def test_parts(gpu, dtype, new, seen):
    kv = (7000, 3100)
    bt = B.Batch4(54, dtype, 8, 2, 128, 64, new, kv)
    cache, t, q = bt.to4("cuda")
    full = sp.sparsp_paged_attn4_workspace_bytes(cache, t["page_table"], bt.T, 8, max(new), max(kv),
                                                 dtype=dtype, **seen)
    assert full > 0
    wO, wL, tO, tL = B.attention(bt, out_dtype=F, terms=3, **seen)
    for nbytes in (0, full // 3, full - 1, full, 2 * full):
        ws = torch.full((nbytes + 256,), 255, dtype=torch.uint8, device="cuda")
        O, lse = sp.sparsp_paged_attn4(q, cache, **t, max_new=max(new), max_kv=max(kv),
                                       workspace=ws[:nbytes], out_dtype=sp.F32, **seen)
        R.close(O, wO, tO, f"O with {nbytes}")
        R.close(lse, wL, tL, f"lse with {nbytes}")
        assert (ws[nbytes:] == 255).all()


@pytest.mark.parametrize("new", [1, 50])
def test_more_keys_than_a_list_of_pages(gpu, new):
    bt = B.Batch4(55, BF, 1, 1, 64, 16, (new,), (2 * 16384 + 1,), bad=((0, 3), (0, 1030)))
    check(bt, *run(bt, workspace=False))


def test_precision_of_few_rows(gpu):
    """Probabilities enter as two bf16: nearly every bf16 output is the exact one rounded."""
    bt = B.Batch4(56, BF, 8, 2, 128, 64, (1, 1), (900, 300))
    O, _ = run(bt)
    want = B.attention(bt)[0]
    assert (O.cpu() == want.to(BF)).double().mean() > 0.98


@pytest.mark.parametrize("dtype,new", [(BF, (6, 1)), (BF, (90, 40)), (F, (5, 1))])
def test_large_and_tiny_scores(gpu, dtype, new):
    bt = B.Batch4(57, dtype, 4, 2, 64, 16, new, (300, 45), std=60.0)
    check(bt, *run(bt))
    check(bt, *run(bt, softmax_scale=1e-4), scale=1e-4)


def test_far_pages(gpu):
    """A cache whose rows lie past 2^31 bytes."""
    H, page, d = 8, 64, 128
    pages = (1 << 31) // (H * page * d // 2) + 9
    cache = sp.Cache4.zeros(pages, H, page, d)
    table = torch.tensor([[pages - 1, pages - 3], [0, pages - 2]], dtype=torch.int32, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(5)
    off, kv = lengths([100, 70], [100, 70])
    K, V = (torch.randn(H, 170, d, generator=g, device="cuda", dtype=BF) for _ in range(2))
    sp.sparsp_paged_append4(K, V, cache, table, off, kv)
    k, v = sp.sparsp_paged_read4(cache, table, off, kv, 170)
    for x, got in ((K, k), (V, v)):
        assert torch.equal(got.cpu().double(), B.values(*B.quantise(x.cpu())))
    q = torch.randn(H, 170, d, generator=g, device="cuda", dtype=BF)
    small = sp.Cache4.zeros(4, H, page, d)
    near = torch.tensor([[0, 1], [2, 3]], dtype=torch.int32, device="cuda")
    sp.sparsp_paged_append4(K, V, small, near, off, kv)
    a = sp.sparsp_paged_attn4(q, cache, table, off, kv)
    b = sp.sparsp_paged_attn4(q, small, near, off, kv)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_a_step_in_a_graph_and_on_a_stream(gpu):
    """Append, attention and read of a step: eager, on another stream, captured and replayed."""
    bt = B.Batch4(58, BF, 8, 2, 128, 64, (1, 1, 3), (800, 63, 2000))
    cache, t, q = bt.to4("cuda")
    n = bt.T
    K, V = (torch.randn(2, n, 128, generator=bt.g).to(BF).cuda() for _ in range(2))
    pos = torch.randint(0, 5000, (n,), generator=bt.g, dtype=torch.int32).cuda()
    f = torch.pow(10000.0, -torch.arange(64, dtype=torch.float64) / 64).float().cuda()
    ws = torch.empty(1 << 22, dtype=torch.uint8, device="cuda")

    def step(c, stream=None):
        r = sp.sparsp_paged_append4(K, V, c, **t, rotary=sp.Rotary(128), positions=pos, inv_freq=f,
                                    Q=q, stream=stream)
        o, lse = sp.sparsp_paged_attn4(r, c, **t, max_new=3, max_kv=2000, workspace=ws, window=500,
                                       sinks=4, stream=stream)
        return (r, o, lse) + sp.sparsp_paged_read4(c, **t, tokens=n, stream=stream) + c.tensors

    def fresh():
        return sp.Cache4(*(x.clone() for x in cache.tensors))

    want = step(fresh())
    side, c = torch.cuda.Stream(), fresh()
    side.wait_stream(torch.cuda.current_stream())
    got = step(c, side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    c = fresh()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(c)
    for _ in range(3):
        for x, old in zip(c.tensors, cache.tensors):
            x.copy_(old)
        for x in got[:5]:
            x.zero_()
        graph.replay()
        eager = step(fresh())
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        assert all(torch.equal(a, b) for a, b in zip(eager, want))


def test_run_beside_the_cache_of_rows(gpu):
    """What a 4-bit cache holds, read back and appended to a cache of rows, attends alike."""
    H, d, page, B_ = 4, 64, 32, 3
    new, kv = (70, 20, 33), (70, 20, 33)
    off, kvl = lengths(new, kv)
    g = torch.Generator().manual_seed(6)
    n = sum(new)
    Q, K, V = (torch.randn(h, n, d, generator=g).to(BF).cuda() for h in (8, H, H))
    need = [-(-k // page) for k in kv]
    table = torch.full((B_, max(need)), -1, dtype=torch.int32)
    ids = torch.randperm(sum(need), generator=g)
    at = 0
    for b, w in enumerate(need):
        table[b, :w] = ids[at:at + w]
        at += w
    table = table.cuda()
    four = sp.Cache4.zeros(sum(need), H, page, d)
    sp.sparsp_paged_append4(K, V, four, table, off, kvl)
    k, v = sp.sparsp_paged_read4(four, table, off, kvl, n)
    Kc, Vc = (torch.zeros(sum(need), H, page, d, dtype=BF, device="cuda") for _ in range(2))
    sp.sparsp_paged_append(k, v, Kc, Vc, table, off, kvl)
    for seen in (dict(), dict(window=11, sinks=2)):
        a, la = sp.sparsp_paged_attn4(Q, four, table, off, kvl, **seen)
        b, lb = sp.sparsp_paged_attn(Q, Kc, Vc, table, off, kvl, **seen)
        # Both round probabilities to bf16 (2^-8 of sums below max |v|) and the output.
        top = float(v.abs().max())
        assert (a.double() - b.double()).abs().max() <= 4 * 2.0 ** -8 * top
        assert (la - lb).abs().max() <= 2.0 ** -17


@pytest.mark.parametrize("dtype,new", [(BF, (1, 2)), (BF, (70, 9)), (F, (1, 30))])
@pytest.mark.parametrize("size", [2.0 ** 20, 2.0 ** 24])
@pytest.mark.parametrize("seen", [dict(), dict(window=120, sinks=9)])
def test_scores_of_2_to_the_24(gpu, dtype, new, size, seen):
    """Scores size + 0, 2, 4 or 6, every one of them a float32: their differences count, whatever is
    subtracted from them on the way. (A product of each is exact, so e of the tolerance is the
    2^-22 of the largest difference, 6, that c2 and its product are off by.)"""
    kv = (300, 700)
    bt = B.Batch4(59, dtype, 4, 2, 32, 16, new, kv)
    x = torch.zeros(bt.K.shape, dtype=torch.float64)
    x[..., 0] = 1.0
    x[..., 1] = 2.0 * torch.randint(0, 4, bt.K.shape[:3], generator=bt.g)
    x[..., 2] = 6.0  # (the scale is one)
    live = ~torch.isnan(bt.K[..., 0])
    codes, scales = B.quantise(x)
    assert torch.equal(B.values(codes, scales), x)
    scales[~live] = 255
    bt.four[:2] = [codes, scales.transpose(-1, -2).contiguous()]
    bt.K.copy_(torch.where(live[..., None], x, float("nan")))
    bt.Q.zero_()
    bt.Q[..., 0], bt.Q[..., 1] = size, 1.0
    O, lse = run(bt, softmax_scale=1.0, **seen)
    wO, wL, _, _ = B.attention(bt, scale=1.0, **seen)
    A = B.attention(bt_abs(bt), scale=1.0, **seen)[0]
    N, half = max(kv), R.HALF[dtype]
    r = 2.0 ** -8 if dtype is BF else 0.0
    tol = A * (r + 4 * 6 * 2.0 ** -22 + 2 * (3 * N + 64) * B.U + 2.0 ** -18) + half * wO.abs()
    R.close(O, wO, tol, "O")
    R.close(lse, wL, 4 * B.U * wL.abs() + 2.0 ** -16, "lse")


def bt_abs(bt):
    import copy
    other = copy.copy(bt)
    other.V = bt.V.abs()
    return other



@pytest.mark.parametrize("d,Hq,new,kv", [(128, 8, (1100,), (4000,)),           # nine tiles of eight heads
                                         (96, 64, (1030,), (2100,)),           # 65 a head: one over a round
                                         (64, 96, (900, 500), (3000, 2200)),   # three a CU
                                         (128, 64, (700, 500), (1300, 2900))])
@pytest.mark.parametrize("seen", [dict(), dict(causal=False), dict(window=2500, sinks=40)])
def test_last_round_in_parts(gpu, d, Hq, new, kv, seen):
    """Row tiles of a little over a round of workgroups: with every workspace, against eight heads of
    their own, which are one round, and the same twice."""
    H = 8
    bt = B.Batch4(60, BF, Hq, H, d, 64, new, kv)
    cache, t, q = bt.to4("cuda")
    w = {k: seen[k] for k in seen if k != "causal"}
    hints = dict(max_new=max(new), max_kv=max(kv))
    full = sp.sparsp_paged_attn4_workspace_bytes(cache, t["page_table"], bt.T, Hq, **hints, **w)
    G = Hq // H
    assert full > 0
    want, lse = zip(*(sp.sparsp_paged_attn4(q[g::G].contiguous(), cache, **t, out_dtype=sp.F32, **seen)
                      for g in range(G)))
    for nbytes in (0, full // 2, full):
        ws = torch.full((nbytes + 256,), 255, dtype=torch.uint8, device="cuda")
        O, L = sp.sparsp_paged_attn4(q, cache, **t, **hints, workspace=ws[:nbytes], out_dtype=sp.F32,
                                     **seen)
        again = sp.sparsp_paged_attn4(q, cache, **t, **hints, workspace=ws[:nbytes], out_dtype=sp.F32,
                                      **seen)
        assert torch.equal(O, again[0]) and torch.equal(L, again[1])
        assert (ws[nbytes:] == 255).all()
        # A max_new below the truth sizes the launch for fewer row tiles than there are.
        few = sp.sparsp_paged_attn4(q, cache, **t, max_new=max(new) - 200, max_kv=max(kv) // 2,
                                    workspace=ws[:nbytes], out_dtype=sp.F32, **seen)
        assert (few[0] - O).abs().max() <= 2 * 2.0 ** -8 * 6
        assert (few[1] - L).abs().max() <= 2.0 ** -16
        for g in range(G):
            # Both round probabilities to bf16, by 2^-8 of sums of p |v| below max |v|.
            assert (O[g::G] - want[g]).abs().max() <= 2 * 2.0 ** -8 * 6
            assert (L[g::G] - lse[g]).abs().max() <= 2.0 ** -16
    # Some heads against 64 bits.
    some = B.Batch4(60, BF, Hq, H, d, 64, new, kv)
    assert torch.equal(some.Q, bt.Q)
    some.Hq, some.H, some.Q = 1, 1, bt.Q[G - 1:G]
    some.K, some.V = bt.K[:, :1], bt.V[:, :1]
    wO, wL, tO, tL = B.attention(some, terms=3, out_dtype=F, **seen)
    R.close(O[G - 1:G], wO, tO, "O")
    R.close(L[G - 1:G], wL, tL, "lse")
