"""Tensors that a call makes itself when it is given a stream (no GPU: tensors on the CPU that say
they are on one, and a library that launches nothing).

Memory that the current stream has freed may still be read and written there, and what is dropped while
another stream works on it would be handed out again by the stream it was made on. So what a
call makes for itself comes from the memory of the stream that it runs on, and its later use on the
current stream is told to the allocator.
"""

import contextlib

import pytest
import torch

import paper_2609_32197_amd as sp
from paper_2609_32197_amd import paged


class OnGpu(torch.Tensor):
    is_cuda = True
    recorded = ()

    def get_device(self):
        return 0

    def record_stream(self, stream):
        self.recorded = self.recorded + (stream,)


class Made:
    """What was made, and under which stream: (tensor, stream)."""

    def __init__(self, monkeypatch):
        self.now, self.all = "current", []

        @contextlib.contextmanager
        def under(stream):
            self.now, before = stream, self.now
            yield
            self.now = before

        def noting(make):
            def f(*args, **kw):
                t = make(*args, **kw).as_subclass(OnGpu)
                self.all.append((t, self.now))
                return t
            return f

        monkeypatch.setattr(torch.cuda, "stream", under)
        monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: self.now)
        for name in ("empty", "empty_like"):
            monkeypatch.setattr(torch, name, noting(getattr(torch, name)))
        monkeypatch.setattr(OnGpu, "new_empty", noting(torch.Tensor.new_empty), raising=False)

    def take(self):
        made, self.all = self.all, []
        return made


class Library:
    """Takes every call; an eviction wants a workspace."""

    def __getattr__(self, name):
        return lambda *a: 4096 if name.endswith("evict_workspace_bytes") else 0


def gpu(*shape, dtype=torch.bfloat16):
    return torch.zeros(*shape, dtype=dtype).as_subclass(OnGpu)


def paged_calls():
    x, k = gpu(4, 3, 64), gpu(2, 3, 64)
    K, V, w = gpu(5, 2, 16, 64), gpu(5, 2, 16, 64), gpu(5, 2, 16, dtype=torch.float32)
    i32 = dict(dtype=torch.int32)
    table, off, kv = gpu(1, 2, **i32), gpu(2, **i32), gpu(1, **i32)
    pos, f = gpu(3, **i32), gpu(32, dtype=torch.float32)
    rot = sp.Rotary(64)
    return {  # name: (call, tensors it makes)
        "rope": (lambda s: sp.sparsp_rope(rot, x, pos, f, X2=k, stream=s), 2),
        "append": (lambda s: sp.sparsp_paged_append(k, k, K, V, table, off, kv, rotary=rot,
                                                    positions=pos, inv_freq=f, Q=x, stream=s), 1),
        "attn": (lambda s: sp.sparsp_paged_attn(x, K, V, table, off, kv, stream=s), 2),
        "evict": (lambda s: sp.sparsp_cache_evict(K, V, w, table, kv, 9, stream=s), 3),
    }


def check(made, count, stream):
    assert len(made) == count
    for t, where in made:
        assert where == (stream or "current"), f"a {tuple(t.shape)} tensor was made on {where}"
        if stream:
            assert "current" in t.recorded
        else:
            assert not t.recorded


@pytest.mark.parametrize("name", list(paged_calls()))
@pytest.mark.parametrize("stream", [None, "side"])
def test_paged_cache(monkeypatch, name, stream):
    call, count = paged_calls()[name]
    monkeypatch.setattr(paged, "_call", lambda *a: None)
    monkeypatch.setattr(paged, "load_library", Library)
    made = Made(monkeypatch)
    call(stream)
    check(made.take(), count, stream)


def block_calls():
    g = sp.Geometry(2, 128, 64, 64, 0, 2, sp.BF16)
    f32, i32, i64 = (dict(dtype=t) for t in (torch.float32, torch.int32, torch.int64))
    q, sc, mask = gpu(2, 128, 64), gpu(2, 2, 2, **f32), gpu(2, 2, 1, **i64)
    sel, slot, kp, vp = gpu(2, 2, 2, **i32), gpu(2, 2, **i32), gpu(4, 64, 64), gpu(4, 64, 64)
    kept = (g, q, sel, slot, kp, vp)
    return {
        "scores": (lambda s: sp.sparsp_block_scores(g, q, q, stream=s), 3),
        "topk": (lambda s: sp.sparsp_topk_mask(g, sc, 1, stream=s), 2),
        "cdf": (lambda s: sp.sparsp_cdf_mask(g, sc, 0.9, stream=s), 3),
        "gather": (lambda s: sp.sparsp_demand_union_gather(g, mask, q, q, stream=s), 6),
        "attention": (lambda s: sp.sparsp_block_sparse_attn(*kept, stream=s), 2),
        "part": (lambda s: sp.sparsp_block_sparse_attn_part(*kept, (0, 2), (0, 2), stream=s), 2),
        "chunked": (lambda s: sp.sparsp_chunked_attn(*kept, [], stream=s), 2),
        "order": (lambda s: sp.sparsp_row_order(g, gpu(2, 2, **i32), stream=s), 1),
        "permute": (lambda s: sp.sparsp_permute_blocks(g, gpu(2, **i32), q, stream=s), 1),
        "pack": (lambda s: sp.sparsp_pack_for_consumers(g, gpu(2, 2, 1, **i64), 2, 0, q, q,
                                                        stream=s), 6),
    }


@pytest.mark.parametrize("name", list(block_calls()))
@pytest.mark.parametrize("stream", [None, "side"])
def test_block_calls(monkeypatch, name, stream):
    call, count = block_calls()[name]
    monkeypatch.setattr(sp, "_stream", lambda stream, device: None)
    monkeypatch.setattr(sp, "load_library", Library)
    made = Made(monkeypatch)
    call(stream)
    check(made.take(), count, stream)
