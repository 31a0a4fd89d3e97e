"""Calls on a stream that is not the current one, with outputs and workspaces of their own making."""

import pytest
import torch

import paper_2609_32197_amd as sp

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def long_cache(seed, kv, B=2, H=2, d=64, page=64):
    """A cache of more than 16,384 tokens a sequence, whose eviction takes a workspace."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    width = -(-max(kv) // page)
    c = dict(K_cache=torch.randn((B * width, H, page, d), generator=g, device="cuda").to(BF),
             V_cache=torch.randn((B * width, H, page, d), generator=g, device="cuda").to(BF),
             page_table=torch.randperm(B * width, generator=g, device="cuda").to(torch.int32)
             .view(B, width),
             kv_len=torch.tensor(kv, dtype=torch.int32, device="cuda"))
    w = torch.rand((B * width, H, page), generator=g, device="cuda")
    assert sp.sparsp_cache_evict_workspace_bytes(c["K_cache"], c["page_table"]) > 0
    return c, w


def test_memory_of_the_stream(gpu):
    """Outputs of a call on a side stream are not memory that the current stream has freed, and what
    the caller drops is not handed to the current stream."""
    s = torch.cuda.Stream()
    c, w = long_cache(1, (20000, 300))
    q = torch.randn(4, 2, 64, device="cuda").to(BF)
    off = torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda")
    # (as many bytes as the output has, so that the allocator would choose this block)
    keep = 5000
    x = torch.empty(2 * 2 * keep, dtype=torch.int32, device="cuda")
    freed = x.data_ptr()
    del x
    torch.cuda.synchronize()
    s.wait_stream(torch.cuda.current_stream())
    kept = sp.sparsp_cache_evict(weights=w, keep=keep, stream=s, **c)[1]
    O, lse = sp.sparsp_paged_attn(q, new_off=off, stream=s, **c)
    at = kept.data_ptr()
    assert at != freed
    shape = kept.shape
    del kept
    assert torch.empty(shape, dtype=torch.int32, device="cuda").data_ptr() != at
    torch.cuda.synchronize()


@pytest.mark.parametrize("side", [False, True])
def test_dropped_outputs(gpu, side):
    """Evictions of long caches on two streams at once, every output dropped and its size allocated
    and overwritten on the current stream at once: the result of one after the other."""
    want = []
    for seed in (1, 2):
        c, w = long_cache(seed, (30001, 17003))
        out, kept = sp.sparsp_cache_evict(weights=w, keep=9000, first=3, recent=100, **c)
        want.append([out, kept, c["K_cache"], c["V_cache"], w])
    caches = [long_cache(seed, (30001, 17003)) for seed in (1, 2)]
    streams = [torch.cuda.Stream() if side else torch.cuda.current_stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for (c, w), s in zip(caches, streams):
        out = sp.sparsp_cache_evict(weights=w, keep=9000, first=3, recent=100, stream=s, **c)[0]
        c["new"] = out
        for _ in range(3):
            torch.full((2, 2, 9000), -7, dtype=torch.int32, device="cuda")
            torch.full((1 << 18,), 255, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    for (c, w), ref in zip(caches, want):
        assert torch.equal(c["new"], ref[0])
        for a, b in zip((c["K_cache"], c["V_cache"], w), ref[2:]):
            assert torch.equal(a, b)


def test_a_step_on_a_side_stream(gpu):
    """Rope, append, attention, weights and eviction on a side stream, nothing passed for outputs:
    the same bits as on the current stream."""
    results = []
    for s in (None, torch.cuda.Stream()):
        c, w = long_cache(3, (16800, 40))
        g = torch.Generator(device="cuda").manual_seed(4)
        q, k, v = (torch.randn((h, 3, 64), generator=g, device="cuda").to(BF) for h in (4, 2, 2))
        off = torch.tensor([0, 1, 3], dtype=torch.int32, device="cuda")
        pos = torch.tensor([16799, 38, 39], dtype=torch.int32, device="cuda")
        f = torch.from_numpy(sp.sparsp_rope_frequencies(64)[0]).cuda()
        if s is not None:
            s.wait_stream(torch.cuda.current_stream())
        r = sp.sparsp_rope(sp.Rotary(64), k, pos, f, stream=s)
        q = sp.sparsp_paged_append(k, v, new_off=off, weights=w, rotary=sp.Rotary(64), positions=pos,
                                   inv_freq=f, Q=q, stream=s, **c)
        O, lse = sp.sparsp_paged_attn(q, new_off=off, stream=s, **c)
        t = dict(c)
        del t["V_cache"]
        sp.sparsp_paged_weights(q, lse, weights=w, new_off=off, stream=s, **t)
        out, kept = sp.sparsp_cache_evict(weights=w, keep=1000, recent=20, stream=s, **c)
        if s is not None:
            torch.cuda.current_stream().wait_stream(s)
        results.append([x.clone() for x in (r, q, O, lse, w, out, kept, c["K_cache"], c["V_cache"])])
    for a, b in zip(*results):
        assert torch.equal(a, b)


def test_the_four_calls_on_a_side_stream(gpu):
    """Scores, mask, gather and attention on a side stream, nothing passed for outputs and all but the
    last dropped: the same bits as on the current stream."""
    geom = sp.Geometry(2, 1000, 64, 64, 0, 16, sp.BF16)
    g = torch.Generator(device="cuda").manual_seed(5)
    q, k, v = (torch.randn((2, 1000, 64), generator=g, device="cuda").to(BF) for _ in range(3))

    def run(s):
        sc = sp.sparsp_block_scores(geom, q, k, stream=s)[2]
        mask, sel = sp.sparsp_topk_mask(geom, sc, 5, stream=s)
        o = sp.sparsp_demand_union_gather(geom, mask, k, v, stream=s)
        return sp.sparsp_block_sparse_attn(geom, q, sel, o["slot_of"], o["K_packed"], o["V_packed"],
                                           stream=s)

    want = run(None)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        got = run(s)
        torch.full((1 << 20,), 255, dtype=torch.uint8, device="cuda")
    torch.cuda.current_stream().wait_stream(s)
    # (rows behind the sequence's end are no one's)
    assert torch.equal(got[0][:, :1000], want[0][:, :1000])
    assert torch.equal(got[1][:, :1000], want[1][:, :1000])
