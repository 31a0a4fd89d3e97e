"""new_off that does not ascend: outputs are any values in the columns of the sequences, and nothing
else is written; the call after it is right."""

import pytest
import torch

import paper_2609_32197_amd as sp

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32


@pytest.mark.parametrize("dtype,Hq,H,d,T,off,kv", [
    (F, 1, 1, 64, 20009, (0, 10000, 0, 20000), (500, 3, 700)),     # tiles of all sequences, too few of them
    (BF, 4, 2, 128, 6009, (7, 3000, 10, 6000), (900, 0, 4000)),
    (BF, 2, 2, 64, 29, (5, 2, 4, -2 ** 31, 26), (40, 50, 60, 70)),
    (F, 2, 1, 32, 13, (3, 4, 3, 4, 3, 4), (20,) * 5),
])
def test_descending_offsets(gpu, dtype, Hq, H, d, T, off, kv):
    page = 16
    g = torch.Generator(device="cuda").manual_seed(71)
    B, width = len(kv), -(-max(kv) // page)
    pages = B * width + 2
    K, V = (torch.randn((pages, H, page, d), generator=g, device="cuda").to(dtype) for _ in range(2))
    q = torch.randn((Hq, T, d), generator=g, device="cuda").to(dtype)
    i32 = dict(dtype=torch.int32, device="cuda")
    table = torch.randperm(B * width, generator=g, device="cuda").to(torch.int32).view(B, width)
    new_off, kv_len = torch.tensor(off, **i32), torch.tensor(kv, **i32)
    claimed = torch.zeros(T, dtype=torch.bool)
    for b in range(B):
        lo = min(max(off[b], 0), T)
        claimed[lo:min(max(off[b + 1], lo), T)] = True
    n = sp.sparsp_paged_attn_workspace_bytes(K, table, T, Hq)
    space = torch.full((n + 512,), 7, dtype=torch.uint8, device="cuda")
    O = torch.full((Hq, T, d), 5.0, dtype=dtype, device="cuda")
    lse = torch.full((Hq, T), 5.0, device="cuda")
    w = torch.full((pages, H, page), 5.0, device="cuda")
    k0, v0, w0 = K.clone(), V.clone(), w.clone()
    sp.sparsp_paged_attn(q, K, V, table, new_off, kv_len, O=O, lse=lse, workspace=space[:n])
    sp.sparsp_paged_weights(q, torch.zeros_like(lse), K, table, new_off, kv_len, w)
    assert torch.equal(K, k0) and torch.equal(V, v0) and (space[n:] == 7).all()
    free = ~claimed.cuda()
    assert int(free.sum()) > 0 and (O[:, free] == 5).all() and (lse[:, free] == 5).all()
    mine = torch.zeros(pages, page, dtype=torch.bool)
    for b in range(B):
        t = torch.arange(kv[b])
        mine[table[b].cpu().long()[t // page], t % page] = True
    other = ~mine.cuda()
    assert torch.equal(w.transpose(1, 2)[other], w0.transpose(1, 2)[other])
    # The same buffers with offsets that ascend: as with fresh ones.
    step = T // (B + 1)
    good = torch.arange(0, step * (B + 1), step, **i32)[:B + 1]
    args = (q, K, V, table, good, kv_len)
    sp.sparsp_paged_attn(*args, O=O, lse=lse, workspace=space[:n])
    want, wl = sp.sparsp_paged_attn(*args, workspace=torch.zeros_like(space)[:n])
    mine = slice(0, int(good[-1]))
    assert torch.equal(O[:, mine], want[:, mine]) and torch.equal(lse[:, mine], wl[:, mine])
