"""Binding of the bounded cache (include/sparsp_bounded.h): argument marshalling only.

    Cache4                    a cache held in 4 bits: codes and scales of K and V
    sparsp_paged_append4      new tokens' K and V into it, K and Q rotated on the way
    sparsp_paged_attn4        attention of the new tokens over it, with or without a window
    sparsp_paged_read4        what it holds of the new tokens, back as rows
    sparsp_pages_reserve      pages for the tokens that come next
    sparsp_pages_release      back what no later token sees
    sparsp_pages_fork         sequences continue others, ended ones go
    sparsp_pages_compact      the pages in use moved together
    sparsp_pages_copy         contents of pages to others

Attention with a window over a cache of rows is sparsp_paged_attn(window=, sinks=). Token tensors, page
tables, lengths, devices and streams are as for the paged cache (paged.py). No two tensors of a page
call of which it writes one may share memory.
"""

from __future__ import annotations

import ctypes
import struct
from dataclasses import dataclass
from typing import Any, Optional

from . import _SIGNATURES, _RESTYPES, _check, _torch, BF16, load_library
from .paged import (Rotary, _call, _dtype_code, _hints, _int, _like, _new, _on, _positions, _rows,
                    _scale, _window)

__all__ = [
    "Cache4",
    "sparsp_paged_append4",
    "sparsp_paged_attn4",
    "sparsp_paged_attn4_workspace_bytes",
    "sparsp_paged_read4",
    "paged_append4",
    "paged_attn4",
    "paged_attn4_workspace_bytes",
    "paged_read4",
    "sparsp_pages_reserve",
    "sparsp_pages_release",
    "sparsp_pages_fork",
    "sparsp_pages_compact",
    "sparsp_pages_copy",
    "sparsp_pages_workspace_bytes",
    "pages_reserve",
    "pages_release",
    "pages_fork",
    "pages_compact",
    "pages_copy",
    "pages_workspace_bytes",
]

_VP, _I32, _I64, _F32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float
_STRUCT = ctypes.c_char_p
_CACHE4 = struct.Struct("@PPPPPPPiiiiiiii")

_SIGNATURES.update({
    "sparsp_paged_append4": [_STRUCT, _I32, _I32, _STRUCT, _STRUCT, _STRUCT, _VP, _I32, _VP, _STRUCT,
                             _STRUCT, _VP],
    "sparsp_paged_attn4": [_STRUCT, _I32, _I32, _STRUCT, _STRUCT, _I32, _VP, _I32, _I32, _I32, _F32,
                           _I32, _I32, _VP, _I64, _VP],
    "sparsp_paged_attn4_workspace_bytes": [_STRUCT, _I32, _I32, _I32, _I32, _I32, _I32, _I32],
    "sparsp_paged_read4": [_STRUCT, _I32, _I32, _STRUCT, _STRUCT, _VP],
    "sparsp_pages_workspace_bytes": [_STRUCT, _I32],
    "sparsp_pages_reserve": [_STRUCT, _VP, _VP, _VP, _I64, _VP],
    "sparsp_pages_release": [_STRUCT, _I32, _I32, _VP],
    "sparsp_pages_fork": [_STRUCT, _VP, _I32, _STRUCT, _I32, _VP, _VP, _VP, _VP, _VP, _I64, _VP],
    "sparsp_pages_compact": [_STRUCT, _STRUCT, _I32, _VP, _VP, _VP, _VP, _I64, _VP],
    "sparsp_pages_copy": [_STRUCT, _I32, _I32, _VP, _VP, _I32, _VP],
})
_RESTYPES["sparsp_paged_attn4_workspace_bytes"] = _I64
_RESTYPES["sparsp_pages_workspace_bytes"] = _I64
_PAGES = struct.Struct("@PPPiiii")
_BUFFER = struct.Struct("@Pq")


@dataclass(frozen=True)
class Cache4:
    """K and V in 4 bits: codes uint8 [pages, H, page, d / 2] and scales uint8 [pages, H, d / 32, page].

    A code is sign and magnitude (0, 0.5, 1, 1.5, 2, 3, 4, 6), two to a byte, the even channel in its
    low half; 32 channels of a token share the scale 2^(byte - 127), 255 being NaN.
    """

    K: Any
    K_scales: Any
    V: Any
    V_scales: Any

    # Types and shapes are looked at once, when the cache is made, and sizes again in every call.
    def __post_init__(self):
        torch, K = _torch(), self.K
        for name, t in zip(("K", "K_scales", "V", "V_scales"), self.tensors):
            if not isinstance(t, torch.Tensor):
                raise TypeError(f"{name} must be a torch.Tensor")
            if t.dtype is not torch.uint8 or t.dim() != 4 or not t.is_contiguous():
                raise ValueError(f"{name} must be a contiguous uint8 tensor of four dimensions")
            if t.device != K.device:
                raise ValueError(f"{name} is on {t.device}, K on {K.device}")
        P, H, page, half = K.shape
        codes, scales = (P, H, page, half), (P, H, half // 16, page)
        for name, t, shape in (("K_scales", self.K_scales, scales), ("V", self.V, codes),
                               ("V_scales", self.V_scales, scales)):
            if t.shape != shape:
                raise ValueError(f"{name} must have shape {shape} (got {tuple(t.shape)})")
        # (frozen: set past the dataclass's own refusal)
        object.__setattr__(self, "_sizes", (P, H, page, 2 * half, K.numel(), self.K_scales.numel()))

    @classmethod
    def zeros(cls, pages: int, H: int, page: int, d: int, device="cuda") -> "Cache4":
        """A cache of zeros."""
        if d % 32:
            raise ValueError(f"d = {d} must be a multiple of 32")
        def make(*shape):
            return _torch().zeros(shape, dtype=_torch().uint8, device=device)
        codes, scales = (pages, H, page, d // 2), (pages, H, d // 32, page)
        return cls(make(*codes), make(*scales), make(*codes), make(*scales))

    @property
    def tensors(self) -> tuple:
        """The four tensors, all [pages, ...]: what the page calls copy."""
        return self.K, self.K_scales, self.V, self.V_scales

    @property
    def d(self) -> int:
        return self._sizes[3]


def _cache4(cache, page_table, new_off, kv_len):
    """(sparsp_cache4, GPU) of the cache and its sequences."""
    if not isinstance(cache, Cache4):
        raise TypeError("cache must be a Cache4")
    if not isinstance(page_table, _torch().Tensor) or page_table.dim() != 2:
        raise ValueError("page_table must be an int32 [B, width] tensor")
    K, Ks, V, Vs = cache.K, cache.K_scales, cache.V, cache.V_scales
    P, H, page, d, codes, scales = cache._sizes
    dev = K.get_device()
    if dev < 0:
        raise ValueError(f"the cache must be on the GPU (got {K.device})")
    if K.numel() != codes or V.numel() != codes or Ks.numel() != scales or Vs.numel() != scales:
        raise ValueError("the cache's tensors have been resized")
    B, width = page_table.shape
    i32 = _torch().int32
    return _CACHE4.pack(
        K.data_ptr(), Ks.data_ptr(), V.data_ptr(), Vs.data_ptr(),
        _on(page_table, "page_table", dev, i32), _on(new_off, "new_off", dev, i32, (B + 1,)),
        _on(kv_len, "kv_len", dev, i32, (B,)), P, H, page, d, width, B, 0, 0), dev


def sparsp_paged_append4(K, V, cache: Cache4, page_table, new_off, kv_len,
                         rotary: Optional[Rotary] = None, positions=None, inv_freq=None, Q=None,
                         Q_out=None, stream=None):
    """Writes the new tokens' K, V [H, tokens, d] into a cache of 4-bit values.

    K, V and Q are bfloat16 or float32. With a rotation K is rotated to its positions on the way, and
    so is Q, into Q_out (which may be Q). Returns Q_out, or None without Q.
    """
    c, dev = _cache4(cache, page_table, new_off, kv_len)
    code = _dtype_code(K, "K")
    if K.dim() != 3:
        raise ValueError("K must be [H, tokens, d]")
    H, n, d, dt = cache.K.shape[1], K.shape[1], cache.d, K.dtype
    rot, pos, bits, freq, q, qo = None, None, 32, None, None, None
    if rotary is not None:
        rot = rotary._pack(False)
        pos, bits, freq = _positions(rotary, positions, inv_freq, n, dev)
    if Q is not None:
        q = _rows(Q, "Q", dev, dt, n, d)
        if Q_out is None:
            Q_out = _like(Q, stream)
        qo = _rows(Q_out, "Q_out", dev, dt, n, d, Q.shape[0])
    elif Q_out is not None:
        raise ValueError("Q_out needs Q")
    _call(load_library().sparsp_paged_append4, dev, stream, c, n, code,
          _rows(K, "K", dev, dt, n, d, H), _rows(V, "V", dev, dt, n, d, H), rot, pos, bits, freq, q, qo)
    return Q_out


def sparsp_paged_read4(cache: Cache4, page_table, new_off, kv_len, tokens: int, dtype=None, K=None,
                       V=None, stream=None):
    """What the cache holds of the new tokens, as rows. Returns (K, V) [H, tokens, d].

    tokens is the number of columns (new_off[B]); with new_off as the running sums of kv_len the whole
    cache is read, token after token. dtype: torch.bfloat16 (the default) or torch.float32.
    """
    torch = _torch()
    c, dev = _cache4(cache, page_table, new_off, kv_len)
    dt = dtype or (torch.bfloat16 if K is None else K.dtype)
    n, H, d = _int(tokens, "tokens"), cache.K.shape[1], cache.d
    k, v = (x if x is not None else _new(cache.K, (H, max(n, 0), d), dt, stream) for x in (K, V))
    _call(load_library().sparsp_paged_read4, dev, stream, c, n, _dtype_code(k, "K"),
          _rows(k, "K", dev, dt, n, d, H), _rows(v, "V", dev, dt, n, d, H))
    return k, v


def _seen(window, sinks, causal):
    return (0, 0) if window is None and not sinks else _window(window, sinks, causal)


def sparsp_paged_attn4_workspace_bytes(cache: Cache4, page_table, tokens: int, q_heads: int,
                                       max_new: int = 0, max_kv: int = 0,
                                       window: Optional[int] = None, sinks: int = 0,
                                       dtype=None) -> int:
    """Workspace bytes that sparsp_paged_attn4 can use for these shapes (host). dtype: Q's, bfloat16 by
    default."""
    B, width = page_table.shape
    P, H, page, half = cache.K.shape
    c = _CACHE4.pack(0, 0, 0, 0, 0, 0, 0, P, H, page, 2 * half, width, B, 0, 0)
    code = BF16 if dtype is None else _dtype_code(_torch().empty(0, dtype=dtype), "dtype")
    n = int(load_library().sparsp_paged_attn4_workspace_bytes(
        c, _int(tokens, "tokens"), code, _int(q_heads, "q_heads"), *_checked(window, sinks, True),
        *_hints(max_new, max_kv)))
    _check(n if n < 0 else 0)
    return n


def _checked(window, sinks, causal):
    """(window, sinks) for the calls that take 0 for no window."""
    if window is not None and _int(window, "window") < 1:
        raise ValueError(f"window = {window} must be positive")
    return _seen(window, sinks, causal)


def sparsp_paged_attn4(Q, cache: Cache4, page_table, new_off, kv_len, causal: bool = True,
                       softmax_scale: Optional[float] = None, max_new: Optional[int] = None,
                       max_kv: Optional[int] = None, O=None, lse=None, want_lse: bool = True,
                       out_dtype: Optional[int] = None, workspace=None, stream=None,
                       window: Optional[int] = None, sinks: int = 0):
    """sparsp_paged_attn over a cache held in 4 bits: Q bfloat16 or float32 [heads, tokens, d].

    Returns (O, lse or None), O in Q's type unless out_dtype or O say otherwise.
    """
    torch = _torch()
    c, dev = _cache4(cache, page_table, new_off, kv_len)
    code = _dtype_code(Q, "Q")
    if Q.dim() != 3:
        raise ValueError("Q must be [heads, tokens, d]")
    d, (heads, n, _) = cache.d, Q.shape
    if out_dtype is None:
        out_dtype = code
    odt = torch.bfloat16 if out_dtype == BF16 else torch.float32
    o = O if O is not None else _new(Q, (heads, n, d), odt, stream)
    ls = lse
    if ls is None and want_lse:
        ls = _new(Q, (heads, n), torch.float32, stream)
    ws, nbytes = None, 0
    if workspace is not None:
        ws = _on(workspace, "workspace", dev)
        nbytes = workspace.numel() * workspace.element_size()
    _call(load_library().sparsp_paged_attn4, dev, stream, c, n, code, _rows(Q, "Q", dev, Q.dtype, n, d),
          _rows(o, "O", dev, odt, n, d, heads), _int(out_dtype, "out_dtype"),
          None if ls is None else _on(ls, "lse", dev, torch.float32, (heads, n)), bool(causal),
          *_checked(window, sinks, causal), _scale(softmax_scale, d), *_hints(max_new, max_kv), ws,
          nbytes)
    return o, ls


# ---------------------------------------------------------------------------
# pages
# ---------------------------------------------------------------------------


def _pages(refs, page_table, kv_len, page):
    """(sparsp_pages, GPU, its shape)."""
    torch = _torch()
    if not isinstance(page_table, torch.Tensor) or page_table.dim() != 2:
        raise ValueError("page_table must be an int32 [B, width] tensor")
    at = _on(refs, "refs", None, torch.int32)
    if refs.dim() != 1:
        raise ValueError("refs must be an int32 [pages] tensor")
    dev, (B, width) = refs.get_device(), page_table.shape
    return _PAGES.pack(at, _on(page_table, "page_table", dev, torch.int32),
                       0 if kv_len is None else _on(kv_len, "kv_len", dev, torch.int32, (B,)),
                       refs.shape[0], _int(page, "page"), width, B), dev


def _buffers(caches, pages, dev):
    """(sparsp_page_buffers, how many) of tensors [pages, ...] and Cache4s."""
    torch = _torch()
    if isinstance(caches, (torch.Tensor, Cache4)):
        caches = (caches,)
    packed, count = b"", 0
    for c in caches:
        for t in c.tensors if isinstance(c, Cache4) else (c,):
            at, shape = _on(t, "a cache", dev), t.shape
            if len(shape) < 2 or shape[0] != pages:
                raise ValueError(f"a cache must be [pages = {pages}, ...] (got {tuple(shape)})")
            packed += _BUFFER.pack(at, t.nbytes // max(pages, 1))  # (no pages: refused in the call)
            count += 1
    return packed or None, count


def _page_workspace(packed, rows, workspace, like, dev, stream):
    """Address and bytes of a page call's workspace, and the tensor that holds it."""
    if workspace is None:
        nbytes = load_library().sparsp_pages_workspace_bytes(packed, rows)
        _check(nbytes if nbytes < 0 else 0)
        workspace = _new(like, (nbytes,), _torch().uint8, stream)
        return workspace.data_ptr(), nbytes, workspace
    return _on(workspace, "workspace", dev), workspace.numel() * workspace.element_size(), workspace


def _out(t, name, like, shape, dev, stream):
    """(int32 tensor, address), made here unless given."""
    i32 = _torch().int32
    if t is None:
        t = _new(like, shape, i32, stream)
        return t, t.data_ptr()
    return t, _on(t, name, dev, i32, shape)


def sparsp_pages_workspace_bytes(refs, page_table, rows: int = 0) -> int:
    """Workspace bytes of the page calls for these shapes and a fork's rows (host)."""
    B, width = page_table.shape
    n = int(load_library().sparsp_pages_workspace_bytes(
        _PAGES.pack(0, 0, 0, refs.shape[0], 16, width, B), _int(rows, "rows")))
    _check(n if n < 0 else 0)
    return n


def sparsp_pages_reserve(refs, page_table, new_off, kv_len, page: int, left=None, workspace=None,
                         stream=None):
    """Pages for the new tokens of every sequence, where page_table names none: before their append.

    refs int32 [pages] counts the entries that name a page; it and page_table are changed in place.
    kv_len counts the new tokens. Returns left, int32 [1]: the free pages left, or minus the number
    that was missing. A workspace is allocated here unless one is given, like left. A fork's left is
    another tensor's: where that was negative, a row's last tokens have no page, and the one that they
    get here holds anything; torch.minimum of the two tells for both.
    """
    p, dev = _pages(refs, page_table, kv_len, page)
    B = page_table.shape[0]
    left, at = _out(left, "left", refs, (1,), dev, stream)
    ws, nbytes, workspace = _page_workspace(p, B, workspace, refs, dev, stream)
    _call(load_library().sparsp_pages_reserve, dev, stream, p,
          _on(new_off, "new_off", dev, _torch().int32, (B + 1,)), at, ws, nbytes)
    return left


def sparsp_pages_release(refs, page_table, kv_len, page: int, window: Optional[int] = None,
                         sinks: int = 0, stream=None):
    """Gives back, in place, the pages that no later token of the sequences sees.

    Those behind kv_len tokens (0 ends a sequence), and with a window those between the first `sinks`
    tokens and the window of the next one. Their entries become -1. Returns refs.
    """
    p, dev = _pages(refs, page_table, kv_len, page)
    _call(load_library().sparsp_pages_release, dev, stream, p, *_checked(window, sinks, True))
    return refs


def sparsp_pages_fork(refs, page_table, kv_len, parents, page: int, caches=(), page_table_out=None,
                      kv_len_out=None, refs_out=None, left=None, workspace=None, stream=None):
    """Row i of the new tables continues row parents[i] of the old ones (-1: an empty sequence).

    Full pages are shared, partly filled ones copied in all `caches` (tensors [pages, ...] or Cache4s)
    for all but the first row that continues a sequence; sequences that none continues end. Returns
    (page_table, kv_len, refs, left); the old tensors stay as they are, but copies may go to pages of
    sequences that end. To go back to the old table, count those once more in refs beforehand. left
    leaves out pages that were copied from and that nothing holds any longer; they are free now.
    Rows that share pages are not for sparsp_paged_weights or sparsp_cache_evict.
    """
    torch = _torch()
    p, dev = _pages(refs, page_table, kv_len, page)
    at = _on(parents, "parents", dev, torch.int32)
    if parents.dim() != 1:
        raise ValueError("parents must be an int32 [rows] tensor")
    rows, pages, width = parents.shape[0], refs.shape[0], page_table.shape[1]
    buffers, count = _buffers(caches, pages, dev)
    table, t = _out(page_table_out, "page_table_out", refs, (rows, width), dev, stream)
    kv, k = _out(kv_len_out, "kv_len_out", refs, (rows,), dev, stream)
    counts, r = _out(refs_out, "refs_out", refs, (pages,), dev, stream)
    left, l = _out(left, "left", refs, (1,), dev, stream)
    ws, nbytes, workspace = _page_workspace(p, rows, workspace, refs, dev, stream)
    _call(load_library().sparsp_pages_fork, dev, stream, p, at, rows, buffers, count, t, k, r, l, ws,
          nbytes)
    return table, kv, counts, left


def sparsp_pages_compact(refs, page_table, caches=(), page_table_out=None, refs_out=None, live=None,
                         workspace=None, stream=None):
    """Moves the pages in use together: of n, those numbered n and above into the free ones below.

    Contents move in all `caches` (tensors [pages, ...] or Cache4s). Returns (page_table, refs, live)
    with live int32 [1] = n; the old tensors stay as they are, and the old pages' contents too.
    """
    p, dev = _pages(refs, page_table, None, 16)
    (B, width), pages = page_table.shape, refs.shape[0]
    buffers, count = _buffers(caches, pages, dev)
    table, t = _out(page_table_out, "page_table_out", refs, (B, width), dev, stream)
    counts, r = _out(refs_out, "refs_out", refs, (pages,), dev, stream)
    live, l = _out(live, "live", refs, (1,), dev, stream)
    ws, nbytes, workspace = _page_workspace(p, B, workspace, refs, dev, stream)
    _call(load_library().sparsp_pages_compact, dev, stream, p, buffers, count, t, r, l, ws, nbytes)
    return table, counts, live


def sparsp_pages_copy(src, dst, caches, stream=None):
    """Page src[k] of every cache (tensors [pages, ...] or Cache4s) to page dst[k]; int32 tensors.

    Numbers of no page copy nothing. No page may be a source and a destination, nor a destination twice.
    """
    torch = _torch()
    s = _on(src, "src", None, torch.int32)
    dev, n = src.get_device(), src.numel()
    caches = (caches,) if isinstance(caches, (torch.Tensor, Cache4)) else tuple(caches)
    if not caches:
        raise ValueError("nothing to copy")
    first = caches[0]
    pages = (first.K if isinstance(first, Cache4) else first).shape[0]
    buffers, count = _buffers(caches, pages, dev)
    _call(load_library().sparsp_pages_copy, dev, stream, buffers, count, pages, s,
          _on(dst, "dst", dev, torch.int32, src.shape), n)


paged_append4 = sparsp_paged_append4
paged_attn4 = sparsp_paged_attn4
paged_attn4_workspace_bytes = sparsp_paged_attn4_workspace_bytes
paged_read4 = sparsp_paged_read4
pages_reserve = sparsp_pages_reserve
pages_release = sparsp_pages_release
pages_fork = sparsp_pages_fork
pages_compact = sparsp_pages_compact
pages_copy = sparsp_pages_copy
pages_workspace_bytes = sparsp_pages_workspace_bytes
