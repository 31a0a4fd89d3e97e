"""New tokens into the paged cache: places, rotation, and everything else left as it was."""

import pytest
import torch

import paper_2609_32197_amd as sp
from tests import _cache_ref as R

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32


def bits(t):
    return t.contiguous().view(torch.int16 if t.dtype == BF else torch.int32).cpu()


@pytest.mark.parametrize("dtype,Hq,H,d,page,new,kv,bad,order,rot,layout", [
    (BF, 4, 2, 128, 16, (1, 1, 1), (1, 16, 17), (), "token", 128, "half"),
    (BF, 6, 3, 64, 32, (0, 40, 3, 1), (5, 40, 131, 64), ((2, 3),), "packed", 32, "interleaved"),
    (BF, 1, 1, 8, 256, (5, 300), (0, 300), (), "head", 8, "half"),     # new tokens before the first
    (BF, 2, 2, 80, 64, (9, 2), (4, 70), (), "token", 20, "half"),       # four of nine have a place
    (F, 5, 5, 100, 16, (33, 0, 7), (50, 0, 7), ((0, 2),), "packed", 50, "half"),
    (F, 2, 1, 128, 128, (1,), (129,), (), "head", 0, "half"),
])
@pytest.mark.parametrize("with_weights", [False, True])
def test_append(gpu, dtype, Hq, H, d, page, new, kv, bad, order, rot, layout, with_weights):
    bt = R.Batch(7, dtype, Hq, H, d, page, new, kv, tail=3, bad=bad)
    t, q = bt.to("cuda", order)
    k = torch.randn(H, bt.T, d, generator=bt.g).to(dtype)
    v = torch.randn(H, bt.T, d, generator=bt.g).to(dtype)
    pos = torch.randint(0, 100000, (1, bt.T), generator=bt.g, dtype=torch.int32)
    qf = torch.where(torch.isnan(bt.Q), 1.0, bt.Q)
    q = R.laid_out(qf, order, "cuda")
    w = bt.weights.cuda() if with_weights else None
    kw = {}
    if rot:
        f = torch.from_numpy(sp.sparsp_rope_frequencies(rot)[0])
        q_out = torch.full((Hq, bt.T, d), 7.0, dtype=dtype, device="cuda")
        kw = dict(rotary=sp.Rotary(rot, layout), positions=pos.cuda(), inv_freq=f.cuda(), Q=q,
                  Q_out=q_out)
        kr, ktol = R.rotate(k, pos, f, rot, layout, (rot // 2,))
    else:
        kr, ktol = k.double(), torch.zeros(1)
    out = sp.sparsp_paged_append(R.laid_out(k, order, "cuda"), R.laid_out(v, order, "cuda"),
                                 weights=w, **t, **kw)
    want_k, want_v, want_w = bt.K.double(), bt.V.clone(), bt.weights.clone()
    tol = torch.zeros(want_k.shape, dtype=torch.float64)
    for b in range(bt.B):
        for i in range(new[b]):
            slot, col = kv[b] - new[b] + i, int(bt.new_off[b]) + i
            p, r = bt.place(b, slot) if slot >= 0 else (None, 0)
            if p is not None:
                want_k[p, :, r], want_v[p, :, r] = kr[:, col], v[:, col]
                tol[p, :, r] = ktol[:, col] if rot else 0.0
                want_w[p, :, r] = 0.0
    R.close(t["K_cache"], want_k, tol, "K")
    assert torch.equal(bits(t["V_cache"]), bits(want_v))
    if with_weights:
        assert torch.equal(bits(w), bits(want_w))
    if rot:
        want, qtol = R.rotate(qf, pos, f, rot, layout, (rot // 2,))
        want[:, sum(new):] = 7.0  # columns of no sequence: as they were
        assert out is q_out
        R.close(out, want, qtol, "Q")
    else:
        assert out is None


def test_many_tokens_and_sequences(gpu):
    """Runs of several tokens per workgroup, across many sequence ends."""
    g = torch.Generator().manual_seed(9)
    new = torch.randint(0, 40, (301,), generator=g).tolist()
    kv = [n + int(torch.randint(0, 50, (1,), generator=g)) for n in new]
    bt = R.Batch(8, BF, 1, 1, 16, 16, new, kv, tail=5)
    t, _ = bt.to("cuda")
    k = torch.randn(1, bt.T, 16, generator=g).to(BF)
    sp.sparsp_paged_append(k.cuda(), (2 * k).cuda(), **t)
    K, V = t["K_cache"].cpu(), t["V_cache"].cpu()
    for b in range(bt.B):
        for i in range(new[b]):
            p, r = bt.place(b, kv[b] - new[b] + i)
            col = int(bt.new_off[b]) + i
            bt.K[p, :, r], bt.V[p, :, r] = k[:, col], 2 * k[:, col]
    assert torch.equal(bits(K), bits(bt.K)) and torch.equal(bits(V), bits(bt.V))


def test_offsets_that_are_no_offsets(gpu):
    """Descending, negative and too large offsets and lengths: clamped, nothing else is touched."""
    bt = R.Batch(11, BF, 1, 1, 16, 16, (3, 2, 4), (10, 20, 30))
    t, _ = bt.to("cuda")
    t["new_off"] = torch.tensor([-5, 2, 1, 2 ** 31 - 1], dtype=torch.int32, device="cuda")
    t["kv_len"] = torch.tensor([-3, 2 ** 31 - 1, 30], dtype=torch.int32, device="cuda")
    k = torch.randn(1, bt.T, 16, generator=bt.g).to(BF)
    sp.sparsp_paged_append(k.cuda(), k.cuda(), **t)
    # Sequence 0 has tokens 0, 1 and no cached ones, sequence 1 none, sequence 2 tokens 2.. (the
    # end is raised to the start): none of the first two is written. Where later tokens go
    # is for the clamped offsets to say; what matters is that rows of sequences 0 and 1 stay.
    K = t["K_cache"].cpu()
    for b in (0, 1):
        for s in range(bt.kv[b]):
            p, r = bt.place(b, s)
            assert torch.equal(bits(K[p, :, r]), bits(bt.K[p, :, r]))
