"""Eviction: which tokens stay, and where they and everything else end up, bit for bit."""

import pytest
import torch

import paper_2609_32197_amd as sp
from tests import _cache_ref as R

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32


def choose(w, n, keep, first, recent):
    """Kept tokens of one head, w float32 [n] with NaN below everything."""
    if n <= keep:
        return list(range(n))
    free = list(range(first, n - recent))

    def order(t):
        x = float(w[t])
        return (1, 0.0, t) if x != x else (0, -x, t)

    best = sorted(free, key=order)[:keep - first - recent]
    return sorted(list(range(first)) + best + list(range(n - recent, n)))


def check(bt, keep, first, recent, out_of_place=False):
    K, V, W = bt.K.clone(), bt.V.clone(), bt.weights.clone()
    k, v, w, table = K.cuda(), V.cuda(), W.cuda(), bt.table
    dst = None
    if out_of_place:  # pages behind all others, sequence after sequence
        each = -(-keep // bt.page) + 1
        dst = (bt.pages + torch.arange(bt.B * each)).view(bt.B, each).to(torch.int32)
        more = (bt.B * each,)
        k, v, w = (torch.cat((x, torch.full(more + x.shape[1:], 5.0, dtype=x.dtype).cuda()))
                   for x in (k, v, w))
        K, V, W = k.cpu(), v.cpu(), w.cpu()
        pages = bt.pages + bt.B * each
        # (numbers of no page must stay numbers of no page in the larger cache)
        table = torch.where(bt.table >= bt.pages, 2 ** 31 - 1, bt.table.long()).to(torch.int32)
    out, kept = sp.sparsp_cache_evict(k, v, w, table.cuda(), bt.kv_len.cuda(), keep, first, recent,
                                      dst_table=None if dst is None else dst.cuda())
    assert out.cpu().tolist() == [min(x, keep) for x in bt.kv]
    want = torch.full((bt.B, bt.H, keep), -1, dtype=torch.int32)
    src = (K.clone(), V.clone(), W.clone())
    for b in range(bt.B):
        n = bt.kv[b]
        at = [bt.place(b, t) for t in range(n)]
        for h in range(bt.H):
            ws = [float("nan") if p is None else src[2][p, h, r] for p, r in at]
            stay = choose(ws, n, keep, first, recent)
            want[b, h, :len(stay)] = torch.tensor(stay, dtype=torch.int32)
            for j, t in enumerate(stay):
                if dst is None:
                    q, r = bt.place(b, j)
                else:
                    q, r = int(dst[b, j // bt.page]), j % bt.page
                p, s = at[t]
                if p is None or q is None:
                    continue
                for x, y in zip((K, V, W), src):
                    x[q, h, r] = y[p, h, s]
    assert torch.equal(kept.cpu(), want)
    for name, got, ref in (("K", k, K), ("V", v, V), ("weights", w, W)):
        i = torch.int16 if got.dtype == BF else torch.int32
        assert torch.equal(got.cpu().view(i), ref.view(i)), name


CASES = [
    # dtype, H, d, page, kv, keep, first, recent, bad pages
    (BF, 1, 64, 16, (2,), 1, 0, 0, ()),
    (BF, 2, 128, 16, (40, 3, 0, 17), 16, 2, 5, ()),
    (BF, 3, 80, 32, (100, 99, 98), 98, 0, 98, ()),          # nothing to choose
    (BF, 2, 128, 64, (1500, 700, 64), 333, 4, 100, ()),
    (BF, 1, 8, 256, (5000,), 1200, 0, 0, ()),                # several chunks in one call
    (F, 2, 100, 16, (200, 31), 31, 31, 0, ()),
    (F, 1, 128, 32, (777,), 700, 1, 1, ((0, 3), (0, 20))),   # pages that do not exist
    (F, 1, 4, 16, (90, 65), 64, 0, 3, ()),
]


@pytest.mark.parametrize("dtype,H,d,page,kv,keep,first,recent,bad", CASES)
@pytest.mark.parametrize("out_of_place", [False, True])
def test_evict(gpu, dtype, H, d, page, kv, keep, first, recent, bad, out_of_place):
    bt = R.Batch(51, dtype, H, H, d, page, (0,) * len(kv), kv, bad=bad)
    check(bt, keep, first, recent, out_of_place)


@pytest.mark.parametrize("kind", ["equal", "zeros", "few", "wild", "negative"])
def test_weights_that_tie_or_are_not_numbers(gpu, kind):
    bt = R.Batch(52, BF, 2, 2, 16, 16, (0, 0), (500, 130))
    g = torch.Generator().manual_seed(1)
    s = bt.weights.shape
    bt.weights = {
        "equal": lambda: torch.full(s, 0.25),
        "zeros": lambda: torch.where(torch.rand(s, generator=g) < 0.5, 0.0, -0.0),
        "few": lambda: torch.randint(0, 3, s, generator=g).float(),
        "wild": lambda: torch.tensor([0.0, float("inf"), float("nan"), -float("inf"), 1e-45, 3e38,
                                      -1.0])[torch.randint(0, 7, s, generator=g)],
        "negative": lambda: -torch.rand(s, generator=g),
    }[kind]()
    for keep, first, recent in ((129, 0, 0), (100, 3, 9), (60, 0, 59)):
        check(bt, keep, first, recent)


def test_one_long_cache(gpu):
    """A choice among many tokens, whose keys share their leading digits."""
    n, keep = 70001, 9999
    H, d, page = 2, 16, 64
    pages = -(-n // page)
    g = torch.Generator().manual_seed(2)
    table = torch.randperm(pages, generator=g).to(torch.int32).view(1, -1)
    w = 1.0 + torch.randint(0, 3000, (pages, H, page), generator=g).float() * 2.0 ** -23
    K = torch.randn(pages, H, page, d, generator=g).to(BF)
    k, v, ww = K.cuda(), (-K).cuda(), w.cuda()
    kv = torch.tensor([n], dtype=torch.int32, device="cuda")
    out, kept = sp.sparsp_cache_evict(k, v, ww, table.cuda(), kv, keep, 7, 50)
    t = torch.arange(n)
    p, r = table[0].long()[t // page], t % page
    j = torch.arange(keep)
    q, s = table[0].long()[j // page], j % page
    for h in range(H):
        x = w[p, h, r].clone()
        x[:7] = x[n - 50:] = float("inf")
        stay = torch.sort(torch.sort(-x, stable=True).indices[:keep]).values
        assert torch.equal(kept[0, h].cpu().long(), stay)
        assert torch.equal(k.cpu()[q, h, s], K[p, h, r][stay])
        assert torch.equal(v.cpu()[q, h, s], -K[p, h, r][stay])
        assert torch.equal(ww.cpu()[q, h, s], w[p, h, r][stay])
    assert out.item() == keep
