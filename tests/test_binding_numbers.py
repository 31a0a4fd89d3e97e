"""Numbers that the library takes in 32 bits: larger ones are refused, not cut to their low bits."""

import pytest
import torch

import paper_2609_32197_amd as sp
from paper_2609_32197_amd import paged
from tests.test_binding_streams import gpu

BIG = 2 ** 32


def calls():
    x = gpu(4, 3, 64)
    K, V, w = gpu(5, 2, 16, 64), gpu(5, 2, 16, 64), gpu(5, 2, 16, dtype=torch.float32)
    i32 = dict(dtype=torch.int32)
    table, off, kv = gpu(1, 2, **i32), gpu(2, **i32), gpu(1, **i32)
    lse = gpu(4, 3, dtype=torch.float32)
    attn = lambda **a: sp.sparsp_paged_attn(x, K, V, table, off, kv, **a)
    weigh = lambda **a: sp.sparsp_paged_weights(x, lse, K, table, off, kv, w, **a)
    evict = lambda keep=9, **a: sp.sparsp_cache_evict(K, V, w, table, kv, keep, **a)
    return [
        ("first", lambda: evict(first=BIG)),
        ("recent", lambda: evict(recent=BIG + 3)),
        ("keep", lambda: evict(keep=BIG + 9)),
        ("keep", lambda: evict(keep=-BIG + 9)),
        ("max_new", lambda: attn(max_new=BIG + 1)),
        ("max_kv", lambda: attn(max_kv=-BIG + 1)),
        ("out_dtype", lambda: attn(out_dtype=BIG + sp.BF16)),
        ("max_new", lambda: weigh(max_new=BIG + 1)),
        ("max_kv", lambda: weigh(max_kv=2 ** 31)),
        ("rot_dim", lambda: sp.sparsp_rope_frequencies(BIG + 64)),
        ("rot_dim", lambda: sp.sparsp_rope_frequencies(-BIG + 64)),
        ("tokens", lambda: sp.sparsp_paged_attn_workspace_bytes(K, table, BIG + 1, 2)),
        ("q_heads", lambda: sp.sparsp_paged_attn_workspace_bytes(K, table, 1, BIG + 2)),
        ("max_new", lambda: sp.sparsp_paged_attn_workspace_bytes(K, table, 1, 2, BIG + 2)),
        ("max_kv", lambda: sp.sparsp_paged_attn_workspace_bytes(K, table, 1, 2, 1, BIG + 2)),
    ]


@pytest.mark.parametrize("n", range(len(calls())))
def test_refused(monkeypatch, n):
    monkeypatch.setattr(paged, "_call", lambda *a: None)
    name, call = calls()[n]
    with pytest.raises(ValueError, match=name):
        call()
