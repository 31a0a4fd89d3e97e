"""Binding of the bounded cache (include/sparsp_bounded.h): argument marshalling only.

    Cache4                    a cache held in 4 bits: codes and scales of K and V
    sparsp_paged_append4      new tokens' K and V into it, K and Q rotated on the way
    sparsp_paged_attn4        attention of the new tokens over it, with or without a window
    sparsp_paged_read4        what it holds of the new tokens, back as rows

Attention with a window over a cache of rows is sparsp_paged_attn(window=, sinks=). Token tensors, page
tables, lengths, devices and streams are as for the paged cache (paged.py).
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
})
_RESTYPES["sparsp_paged_attn4_workspace_bytes"] = _I64


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
        return self.K.shape[3] * 2


def _cache4(cache, page_table, new_off, kv_len):
    """(sparsp_cache4, GPU) of the cache and its sequences."""
    torch = _torch()
    if not isinstance(cache, Cache4):
        raise TypeError("cache must be a Cache4")
    if not isinstance(cache.K, torch.Tensor) or cache.K.dim() != 4:
        raise ValueError("codes must be uint8 [pages, H, page, d / 2]")
    if not isinstance(page_table, torch.Tensor) or page_table.dim() != 2:
        raise ValueError("page_table must be an int32 [B, width] tensor")
    P, H, page, half = cache.K.shape
    scales = (P, H, half // 16, page)
    B, width = page_table.shape
    u8, i32 = torch.uint8, torch.int32
    k = _on(cache.K, "K codes", None, u8)
    dev = cache.K.get_device()
    return _CACHE4.pack(
        k, _on(cache.K_scales, "K scales", dev, u8, scales),
        _on(cache.V, "V codes", dev, u8, cache.K.shape),
        _on(cache.V_scales, "V scales", dev, u8, scales), _on(page_table, "page_table", dev, i32),
        _on(new_off, "new_off", dev, i32, (B + 1,)), _on(kv_len, "kv_len", dev, i32, (B,)),
        P, H, page, 2 * half, width, B, 0, 0), dev


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


paged_append4 = sparsp_paged_append4
paged_attn4 = sparsp_paged_attn4
paged_attn4_workspace_bytes = sparsp_paged_attn4_workspace_bytes
paged_read4 = sparsp_paged_read4
