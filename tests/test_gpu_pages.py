"""Pages taken, given back, forked, compacted and copied, against loops over lists."""

import random

import pytest
import torch

import paper_2609_32197_amd as sp
from tests import _bounded_ref as B
from tests import _cache_ref as R

pytestmark = pytest.mark.gpu
I32 = torch.int32


def ints(x):
    return torch.tensor(x, dtype=I32, device="cuda")


class Pool:
    """Tables, counts and contents as lists, and the calls as loops."""

    def __init__(self, seed, pages, page, width, kv, share=0.0, shuffled=True, holders=0):
        r = random.Random(seed)
        self.r, self.pages, self.page, self.width, self.kv = r, pages, page, width, list(kv)
        ids = list(range(pages))
        if shuffled:
            r.shuffle(ids)
        self.refs = [0] * pages
        self.table = []
        for b, k in enumerate(kv):
            need = -(-k // page)
            same = 0
            if b and r.random() < share:
                same = min(r.randint(0, need), min(kv[b - 1], k) // page)
            row = self.table[-1][:same] if b else []
            row = row + [ids.pop() for _ in range(need - same)]
            row += [r.choice([-1, pages, -2 ** 31, 2 ** 31 - 1]) for _ in range(width - need)]
            self.table.append(row)
            for p in row[:need]:
                self.refs[p] += 1
        for _ in range(holders):  # held by something else
            self.refs[r.randrange(pages)] += 1

    def named(self, p):
        return 0 <= p < self.pages

    def take(self, refs, table, wants, avoid=()):
        free = [p for p in range(self.pages) if refs[p] <= 0 and p not in avoid]
        got = []
        for (b, j), p in zip(wants, free):
            table[b][j] = p
            refs[p] = 1
            got.append(p)
        return len(free) - len(wants), got

    def reserve(self, new):
        wants = []
        for b, (k, n) in enumerate(zip(self.kv, new)):
            if n > 0:
                for j in range(max(k - n, 0) // self.page, -(-k // self.page)):
                    if not self.named(self.table[b][j]):
                        wants.append((b, j))
        return self.take(self.refs, self.table, wants)[0]

    def release(self, kv, window=0, sinks=0):
        for b, k in enumerate(kv):
            for j in range(self.width):
                lo, hi = j * self.page, (j + 1) * self.page - 1
                if lo < k and not (window and lo >= sinks and hi <= k - window):
                    continue
                if self.named(self.table[b][j]):
                    self.refs[self.table[b][j]] -= 1
                self.table[b][j] = -1

    def fork(self, parents):
        """(table, kv, refs, left, copies [(src, dst)])."""
        refs, table, kv, wants, src = list(self.refs), [], [], [], []
        for row in self.table:
            for p in row:
                if self.named(p):
                    refs[p] -= 1
        for i, p in enumerate(parents):
            live = 0 <= p < len(self.table)
            k = self.kv[p] if live else 0
            need = -(-k // self.page)
            row = [q if self.named(q) else -1 for q in self.table[p][:need]] if live else []
            row += [-1] * (self.width - need)
            if k % self.page and row[need - 1] >= 0:
                q = row[need - 1]
                if p in parents[:i] or self.refs[q] != 1:
                    wants.append((i, need - 1))
                    src.append(q)
                    row[need - 1] = -1
            for q in row:
                if q >= 0:
                    refs[q] += 1
            table.append(row)
            kv.append(k)
        left, got = self.take(refs, table, wants, set(src))
        return table, kv, refs, left, list(zip(src, got))

    def compact(self):
        used = [p for p in range(self.pages) if self.refs[p] > 0]
        n = len(used)
        src = [p for p in used if p >= n]
        dst = [p for p in range(n) if self.refs[p] <= 0]
        to = {p: p for p in used if p < n}
        to.update(zip(src, dst))
        refs = [0] * self.pages
        for p in used:
            refs[to[p]] = self.refs[p]
        return [[to.get(p, -1) for p in row] for row in self.table], refs, n, list(zip(src, dst))


def caches(pages, page):
    """Buffers of several sizes, each page's contents its own."""
    g = torch.Generator(device="cuda").manual_seed(7)
    four = sp.Cache4(*(torch.randint(0, 256, s, generator=g, device="cuda", dtype=torch.uint8)
                       for s in ((pages, 2, page, 32), (pages, 2, 2, page)) * 2))
    rows = torch.randn(pages, 3, page, 100, generator=g, device="cuda")
    weights = torch.randn(pages, 3, page, generator=g, device="cuda")
    return four, rows, weights


def tensors(group):
    return [t for c in group for t in (c.tensors if isinstance(c, sp.Cache4) else (c,))]


def moved(before, copies):
    out = [t.clone() for t in before]
    if copies:
        src, dst = (torch.tensor(x, device="cuda") for x in zip(*copies))
        for t, old in zip(out, before):
            t[dst] = old[src]
    return out


SHAPES = [
    # pages, page, width, kv
    (1, 16, 1, (1,)),
    (40, 16, 5, (1, 16, 17, 0, 80)),
    (300, 64, 20, (700, 64, 63, 65, 1280, 1)),
    (3000, 16, 30, tuple(range(1, 400, 3))),
    (20000, 32, 9, tuple((7 * b) % 289 for b in range(1500))),   # more than one count holds
    (16384, 256, 70, (17920, 3)),
    (16385, 128, 3, tuple([129] * 1024)),
    (40000, 16, 2100, (33600, 1, 20000)),
]


@pytest.mark.parametrize("pages,page,width,kv", SHAPES)
@pytest.mark.parametrize("share,holders", [(0.0, 0), (0.5, 5)])
@pytest.mark.parametrize("most", [1, 100])
def test_reserve(gpu, pages, page, width, kv, share, holders, most):
    p = Pool(1, pages, page, width, kv, share, holders=holders)
    new = [p.r.choice([0, 1, p.r.randint(0, most)]) for _ in kv]
    if most == 100:  # a page that is gone among those of the new tokens
        p.table[0][-1] = -1
    for b in range(len(kv)):
        p.kv[b] = min(kv[b] + new[b], page * width)
    off = [0]
    for n in new:
        off.append(off[-1] + n)
    refs, table = ints(p.refs), ints(p.table)
    left = sp.sparsp_pages_reserve(refs, table, ints(off), ints(p.kv), page)
    want = p.reserve(new)
    assert int(left) == want
    assert table.tolist() == p.table and refs.tolist() == p.refs
    # Once more: everything is there.
    given = torch.full((1,), 99, dtype=I32, device="cuda")
    if want >= 0:
        assert sp.sparsp_pages_reserve(refs, table, ints(off), ints(p.kv), page, left=given) is given
        assert int(given) == want
        assert table.tolist() == p.table and refs.tolist() == p.refs


@pytest.mark.parametrize("pages", [30, 17000])
def test_reserve_runs_out(gpu, pages):
    p = Pool(2, pages, 16, 200, (0, 0, 0), holders=0)
    for q in range(pages):
        p.refs[q] = int(q % 7 != 3 or q > 200)
    p.kv = [300, 2000, 500]
    new = [300, 2000, 500]
    refs, table = ints(p.refs), ints(p.table)
    left = sp.sparsp_pages_reserve(refs, table, ints([0, 300, 2300, 2800]), ints(p.kv), 16)
    want = p.reserve(new)
    assert want < 0 and int(left) == want
    assert table.tolist() == p.table and refs.tolist() == p.refs


@pytest.mark.parametrize("pages,page,width,kv", SHAPES)
@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (100, 4), (33, 70), (2 ** 31 - 1, 5)])
def test_release(gpu, pages, page, width, kv, window, sinks):
    p = Pool(3, pages, page, width, kv, 0.4)
    shorter = [p.r.choice([0, k, k, k // 2]) for k in kv]
    refs, table = ints(p.refs), ints(p.table)
    kw = dict(window=window, sinks=sinks) if window else {}
    assert sp.sparsp_pages_release(refs, table, ints(shorter), page, **kw) is refs
    p.release(shorter, window, sinks)
    assert table.tolist() == p.table and refs.tolist() == p.refs


@pytest.mark.parametrize("pages,page,width,kv", SHAPES)
@pytest.mark.parametrize("share,holders", [(0.0, 0), (0.6, 9)])
@pytest.mark.parametrize("kind", ["same", "beams", "some", "more"])
def test_fork(gpu, pages, page, width, kv, share, holders, kind):
    p = Pool(4, pages, page, width, kv, share, holders=holders)
    B_ = len(kv)
    few = [p.r.randrange(B_) for _ in range(max(1, B_ // 8))]
    parents = {"same": list(range(B_)), "beams": [p.r.choice(few) for _ in range(B_)],
               "some": [p.r.choice([-1, B_, 2 ** 31 - 1, p.r.randrange(B_)]) for _ in range(B_ // 2 + 1)],
               "more": [p.r.randrange(B_) for _ in range(B_ + 70)]}[kind]
    # Two rows share a partly filled page: nobody's own.
    if B_ > 2 and kv[1] and kv[2] >= kv[1] and share:
        j = (kv[1] - 1) // page
        p.refs[p.table[2][j]] -= 1
        p.table[2][j] = p.table[1][j]
        p.refs[p.table[1][j]] += 1
    group = caches(min(pages, 3000), page) if pages <= 3000 else ()
    before = [t.clone() for t in tensors(group)]
    refs, table, kvl = ints(p.refs), ints(p.table), ints(p.kv)
    old = refs.clone(), table.clone(), kvl.clone()
    got = sp.sparsp_pages_fork(refs, table, kvl, ints(parents), page, group)
    t, k, r, left, copies = p.fork(parents)
    assert got[0].tolist() == t and got[1].tolist() == k
    assert int(got[3]) == left
    assert got[2].tolist() == r
    for x, y in zip(tensors(group), moved(before, copies)):
        assert torch.equal(x, y)
    assert all(torch.equal(x, y) for x, y in zip((refs, table, kvl), old))


@pytest.mark.parametrize("pages,page,width,kv", SHAPES)
@pytest.mark.parametrize("shuffled", [True, False])
def test_compact(gpu, pages, page, width, kv, shuffled):
    p = Pool(5, pages, page, width, kv, 0.3, shuffled, holders=4)
    group = caches(pages, page) if pages <= 3000 else (torch.arange(pages * 8, device="cuda").view(-1, 8),)
    before = [t.clone() for t in tensors(group)]
    refs, table = ints(p.refs), ints(p.table)
    old = refs.clone(), table.clone()
    got = sp.sparsp_pages_compact(refs, table, group)
    t, r, n, copies = p.compact()
    assert int(got[2]) == n and got[0].tolist() == t and got[1].tolist() == r
    for x, y in zip(tensors(group), moved(before, copies)):
        assert torch.equal(x, y)
    assert torch.equal(refs, old[0]) and torch.equal(table, old[1])
    # Compact already: nothing moves.
    again = sp.sparsp_pages_compact(got[1], got[0], group)
    assert torch.equal(again[0], got[0]) and torch.equal(again[1], got[1]) and int(again[2]) == n
    # Without contents.
    bare = sp.sparsp_pages_compact(refs, table)
    assert torch.equal(bare[0], got[0]) and torch.equal(bare[1], got[1])


def test_nothing_and_everything_in_use(gpu):
    for refs, n in (([0] * 50, 0), ([-3, 0] * 25, 0), ([1] * 50, 50), ([2 ** 31 - 1] * 50, 50)):
        table, counts, live = sp.sparsp_pages_compact(ints(refs), ints([[3, 49], [-1, 60]]))
        assert int(live) == n
        assert counts.tolist() == [max(x, 0) for x in refs]
        assert table.tolist() == ([[3, 49], [-1, -1]] if n else [[-1, -1], [-1, -1]])


def test_copy(gpu):
    group = caches(90, 64)
    before = [t.clone() for t in tensors(group)]
    src = [3, 5, 5, -1, 90, 7, 2 ** 31 - 1, 8, 89]
    dst = [4, 6, 88, 9, 10, 90, 11, -2 ** 31, 0]
    sp.sparsp_pages_copy(ints(src), ints(dst), group)
    pairs = [(s, d) for s, d in zip(src, dst) if 0 <= s < 90 and 0 <= d < 90]
    for x, y in zip(tensors(group), moved(before, pairs)):
        assert torch.equal(x, y)
    sp.sparsp_pages_copy(ints([]), ints([]), group)


def test_far_pages_are_copied(gpu):
    """Contents past 2^32 bytes."""
    x = torch.zeros(70000, 65536 // 4, dtype=torch.float32, device="cuda")
    x[69999] = torch.arange(65536 // 4, device="cuda")
    sp.sparsp_pages_copy(ints([69999]), ints([69990]), x)
    assert torch.equal(x[69990], x[69999]) and (x[69989] == 0).all() and (x[69991] == 0).all()


@pytest.mark.parametrize("bad", range(4))
def test_whatever_the_arrays_hold(gpu, bad):
    """Lengths, offsets and counts of any value: the calls end, and nothing outside is written."""
    g = torch.Generator(device="cuda").manual_seed(bad)

    def wild(*shape):
        x = torch.randint(-2 ** 31, 2 ** 31, shape, generator=g, device="cuda", dtype=torch.int64)
        return (x if bad % 2 else x % 61 - 5).to(I32)

    def framed(x):
        wide = torch.full((x.numel() + 2048,), 12345, dtype=I32, device="cuda")
        wide[1024:-1024] = x.flatten()
        return wide, wide[1024:-1024].view(x.shape)

    pages = (50, 40000)[bad // 2]
    rf, refs = framed(wild(pages))
    tf, table = framed(wild(33, 20))
    kv, off, parents = wild(33), wild(34), wild(70)
    group = torch.zeros(pages, 64, device="cuda")
    sp.sparsp_pages_fork(refs, table, kv, parents, 16, group)
    sp.sparsp_pages_compact(refs, table, group)
    sp.sparsp_pages_release(refs, table, kv, 16, window=20, sinks=3)
    sp.sparsp_pages_reserve(refs, table, off, kv, 16)
    torch.cuda.synchronize()
    for f in (rf, tf):
        assert (f[:1024] == 12345).all() and (f[-1024:] == 12345).all()


def test_a_turn_in_a_graph(gpu):
    """Fork, release and reserve captured, replayed with other parents, against eager and the loops."""
    p = Pool(6, 400, 16, 30, (100, 37, 250, 16, 401))
    refs, table, kv = ints(p.refs), ints(p.table), ints(p.kv)
    parents = ints([0, 0, 2, 3, 4])
    off = ints([0, 5, 10, 15, 20, 25])
    group = caches(400, 16)
    ws = torch.empty(sp.sparsp_pages_workspace_bytes(refs, table, 5), dtype=torch.uint8, device="cuda")
    first = [t.clone() for t in tensors(group)]

    def turn():
        t, k, r, left = sp.sparsp_pages_fork(refs, table, kv, parents, 16, group, workspace=ws)
        sp.sparsp_pages_release(r, t, k, 16, window=60, sinks=16)
        k = k + 5
        sp.sparsp_pages_reserve(r, t, off, k, 16, left=left, workspace=ws)
        return t, k, r, left

    turn()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = turn()
    for choice in ([0, 0, 2, 3, 4], [4, 4, 4, 4, 4], [-1, 2, 2, 1, -1]):
        parents.copy_(ints(choice))
        for t, f in zip(tensors(group), first):
            t.copy_(f)
        for x in got:
            x.fill_(-77)
        graph.replay()
        torch.cuda.synchronize()
        q = Pool(6, 400, 16, 30, (100, 37, 250, 16, 401))
        q.table, q.kv, q.refs, _, copies = q.fork(choice)
        q.release(q.kv, 60, 16)
        q.kv = [k + 5 for k in q.kv]
        left = q.reserve([5] * 5)
        assert got[0].tolist() == q.table and got[1].tolist() == q.kv
        assert got[2].tolist() == q.refs and int(got[3]) == left
        for x, y in zip(tensors(group), moved(first, copies)):
            assert torch.equal(x, y)
        eager = turn()
        assert all(torch.equal(a, b) for a, b in zip(eager, got))


def test_on_a_stream(gpu):
    p = Pool(8, 200, 16, 12, (100, 37, 150))
    refs, table, kv = ints(p.refs), ints(p.table), ints(p.kv)
    parents = ints([1, 1, 0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = sp.sparsp_pages_fork(refs, table, kv, parents, 16, stream=side)
    out = sp.sparsp_pages_compact(got[2], got[0], stream=side)
    side.synchronize()
    t, k, r, left, _ = p.fork([1, 1, 0])
    assert got[0].tolist() == t and got[2].tolist() == r and int(got[3]) == left
    p.table, p.refs = t, r
    t, r, n, _ = p.compact()
    assert out[0].tolist() == t and out[1].tolist() == r and int(out[2]) == n


def test_refused(gpu):
    refs, table, kv = ints([1] * 9), ints([[0, 1]]), ints([20])
    parents, x = ints([0]), torch.zeros(9, 8, device="cuda")
    small = torch.zeros(16, dtype=torch.uint8, device="cuda")
    for call, kind in (
            (lambda: sp.sparsp_pages_fork(refs, table, kv, parents, 24), sp.SparspError),
            (lambda: sp.sparsp_pages_fork(refs, table, kv, parents, 16, (x, x)), sp.SparspError),
            (lambda: sp.sparsp_pages_fork(refs, table, kv, parents, 16, x[:8]), ValueError),
            (lambda: sp.sparsp_pages_fork(refs, table, kv, parents, 16, x[:, :3].contiguous()),
             sp.SparspError),
            (lambda: sp.sparsp_pages_fork(refs, table, kv, parents, 16, x[:, ::2]), ValueError),
            (lambda: sp.sparsp_pages_fork(refs, table, kv, ints([]), 16), sp.SparspError),
            (lambda: sp.sparsp_pages_fork(refs, table, kv, parents, 16, refs_out=refs), sp.SparspError),
            (lambda: sp.sparsp_pages_fork(refs, table, kv, parents, 16, workspace=small), sp.SparspError),
            (lambda: sp.sparsp_pages_fork(refs, table, kv, parents.long(), 16), ValueError),
            (lambda: sp.sparsp_pages_fork(refs, table, kv, parents, 16, tuple(x.clone() for _ in range(9))),
             sp.SparspError),
            (lambda: sp.sparsp_pages_compact(refs, table, page_table_out=table), sp.SparspError),
            (lambda: sp.sparsp_pages_compact(refs, table, live=ints([1, 2])), ValueError),
            (lambda: sp.sparsp_pages_reserve(refs, table, ints([0]), kv, 16), ValueError),
            (lambda: sp.sparsp_pages_reserve(refs, table, ints([0, 1]), kv, 512), sp.SparspError),
            (lambda: sp.sparsp_pages_release(refs, table, kv, 16, window=0), ValueError),
            (lambda: sp.sparsp_pages_release(refs, table, kv, 16, sinks=4), ValueError),
            (lambda: sp.sparsp_pages_copy(ints([0, 1]), ints([2]), x), ValueError),
            (lambda: sp.sparsp_pages_copy(ints([0]), ints([2]), ()), ValueError)):
        with pytest.raises(kind):
            call()


def test_run_of_a_cache_that_stays_bounded(gpu):
    """Prompts, steps with a window, forks, ends and compactions on one pool, for a cache of rows and one
    of 4 bits with one table: at every step attention equals that over the tokens kept in lists."""
    H, Hq, d, page, width, window, sinks, pages = 2, 4, 32, 16, 12, 40, 5, 40
    g, r = torch.Generator().manual_seed(9), random.Random(9)
    K, V = (torch.full((pages, H, page, d), float("nan"), dtype=torch.bfloat16, device="cuda")
            for _ in range(2))
    four = sp.Cache4.zeros(pages, H, page, d)
    for s in (four.K_scales, four.V_scales):
        s.fill_(255)
    refs = torch.zeros(pages, dtype=I32, device="cuda")
    table = torch.full((3, width), -1, dtype=I32, device="cuda")
    kv = torch.zeros(3, dtype=I32, device="cuda")
    held = [[], [], []]  # each sequence's (k, v) rows [H, d]
    for step in range(14):
        parents = [i if r.random() < 0.6 else r.choice([-1, 0, 1, 2]) for i in range(3)]
        new = [r.choice([1, 1, 2]) if held[p] and p >= 0 else r.randint(1, 30) for p in parents]
        table, kv, refs, left = sp.sparsp_pages_fork(refs, table, kv, ints(parents), page, (K, V, four))
        held = [list(held[p]) if p >= 0 else [] for p in parents]
        sp.sparsp_pages_release(refs, table, kv, page, window=window, sinks=sinks)
        for i in range(3):
            if len(held[i]) + new[i] > page * width:
                new[i] = 0
        off = [0]
        for n in new:
            off.append(off[-1] + n)
        kv = kv + ints(new)
        left = sp.sparsp_pages_reserve(refs, table, ints(off), kv, page)
        assert int(left) >= 0 and int((refs > 0).sum()) == pages - int(left)
        n = off[-1]
        if n == 0:
            continue
        q, k, v = (torch.randn(h, n, d, generator=g).to(torch.bfloat16).cuda() for h in (Hq, H, H))
        sp.sparsp_paged_append(k, v, K, V, table, ints(off), kv)
        sp.sparsp_paged_append4(k, v, four, table, ints(off), kv)
        for i in range(3):
            held[i] += [(k[:, c].cpu(), v[:, c].cpu()) for c in range(off[i], off[i + 1])]
        if step % 4 == 3:
            table, refs, live = sp.sparsp_pages_compact(refs, table, (K, V, four))
            assert int((refs[int(live):] != 0).sum()) == 0
        a = sp.sparsp_paged_attn(q, K, V, table, ints(off), kv, window=window, sinks=sinks)
        b = sp.sparsp_paged_attn4(q, four, table, ints(off), kv, window=window, sinks=sinks)
        # The same tokens in a cache of their own.
        bt = R.Batch(10, torch.bfloat16, Hq, H, d, page, new, [len(x) for x in held])
        bt.Q = q.cpu()
        for bits, (O, lse) in ((16, a), (4, b)):
            for i in range(3):
                for t, (x, y) in enumerate(held[i]):
                    p, row = bt.place(i, t)
                    if bits == 4:
                        x, y = (B.values(*B.quantise(z)).to(torch.bfloat16) for z in (x, y))
                    bt.K[p, :, row], bt.V[p, :, row] = x, y
            wO, wL, tO, tL = B.attention(bt, window, sinks, terms=3)
            R.close(lse, wL, tL, f"lse of {bits} bits, step {step}")
            R.close(O, wO, tO, f"O of {bits} bits, step {step}")
