"""Binding of the paged cache (include/sparsp_cache.h): argument marshalling only.

    sparsp_rope_frequencies   frequencies of rotary positions, scaled for long contexts (host)
    sparsp_rope               rotary positions of Q and K, or back
    sparsp_paged_append       new tokens' K and V into the cache, K and Q rotated on the way
    sparsp_paged_attn         attention of the new tokens over the cache
    sparsp_paged_weights      attention weight per cached token
    sparsp_cache_evict        the cache cut to the tokens of most weight

Token tensors are [heads, tokens, d] with contiguous channels and any other strides: a
projection's [tokens, heads, d] is passed as x.transpose(0, 1). The cache is K_cache and
V_cache [pages, H, page, d]; page_table int32 [B, width], new_off int32 [B + 1] and kv_len
int32 [B] (with the new tokens) describe its sequences. Everything is on one GPU; the calls
run on that GPU's current stream, or on the stream given. What a call makes itself (outputs, a
workspace) comes from the memory of that stream: wait for it before the results are used on another.
"""

from __future__ import annotations

import ctypes
import math
import struct
from dataclasses import dataclass
from typing import Optional, Sequence

from . import _SIGNATURES, _RESTYPES, _check, _make, _torch, BF16, F32, load_library

__all__ = [
    "Rotary",
    "sparsp_rope_frequencies",
    "sparsp_rope",
    "sparsp_paged_append",
    "sparsp_paged_attn",
    "sparsp_paged_attn_workspace_bytes",
    "sparsp_paged_weights",
    "sparsp_cache_evict",
    "sparsp_cache_evict_workspace_bytes",
    "rope_frequencies",
    "rope",
    "paged_append",
    "paged_attn",
    "paged_attn_workspace_bytes",
    "paged_weights",
    "cache_evict",
    "cache_evict_workspace_bytes",
]

_VP, _I32, _I64, _F32, _F64 = (ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float,
                               ctypes.c_double)
# The structures are packed as bytes, which costs a call less than ctypes fields do.
_STRUCT = ctypes.c_char_p
_ROWS = struct.Struct("@Pqqii")
_ROTARY = struct.Struct("@iiiiiifi")
_CACHE = struct.Struct("@PPPPPPiiiiiiii")

_SIGNATURES.update({
    "sparsp_rope_frequencies": [_I32, _F64, _I32, _F64, _F64, _F64, _F64, _VP, _VP],
    "sparsp_rope": [_STRUCT, _I32, _I32, _I32, _STRUCT, _STRUCT, _I32, _VP, _I32, _VP, _VP],
    "sparsp_paged_append": [_STRUCT, _I32, _STRUCT, _STRUCT, _STRUCT, _VP, _I32, _VP, _STRUCT,
                            _STRUCT, _VP],
    "sparsp_paged_attn": [_STRUCT, _I32, _STRUCT, _STRUCT, _I32, _VP, _I32, _F32, _I32, _I32, _VP,
                          _I64, _VP],
    "sparsp_paged_attn_workspace_bytes": [_STRUCT, _I32, _I32, _I32, _I32],
    "sparsp_paged_attn_window": [_STRUCT, _I32, _STRUCT, _STRUCT, _I32, _VP, _I32, _I32, _F32, _I32,
                                 _I32, _VP, _I64, _VP],
    "sparsp_paged_attn_window_workspace_bytes": [_STRUCT, _I32, _I32, _I32, _I32, _I32, _I32],
    "sparsp_paged_weights": [_STRUCT, _I32, _STRUCT, _VP, _I32, _F32, _I32, _I32, _I32, _VP],
    "sparsp_cache_evict": [_STRUCT, _I32, _I32, _I32, _VP, _I32, _VP, _VP, _VP, _I64, _VP],
    "sparsp_cache_evict_workspace_bytes": [_STRUCT],
})
_RESTYPES["sparsp_paged_attn_workspace_bytes"] = _I64
_RESTYPES["sparsp_paged_attn_window_workspace_bytes"] = _I64
_RESTYPES["sparsp_cache_evict_workspace_bytes"] = _I64

_LAYOUTS = {"half": 0, "interleaved": 1}
_SCALINGS = {"plain": 0, "linear": 1, "base": 2, "parts": 3}


@dataclass(frozen=True)
class Rotary:
    """sparsp_rotary: the first rot_dim channels of a row turn in pairs.

    layout "half" pairs channels (p, p + rot_dim/2), "interleaved" (2p, 2p + 1). axis_pairs
    is the number of pairs that turn with each axis of the positions (None: one axis).
    """

    rot_dim: int
    layout: str = "half"
    axis_pairs: Optional[Sequence[int]] = None
    factor: float = 1.0

    @property
    def axes(self) -> int:
        return 1 if self.axis_pairs is None else len(self.axis_pairs)

    def _pack(self, inverse: bool) -> bytes:
        if self.layout not in _LAYOUTS:
            raise ValueError(f"layout must be one of {sorted(_LAYOUTS)} (got {self.layout!r})")
        pairs = (self.rot_dim // 2,) if self.axis_pairs is None else tuple(self.axis_pairs)
        if len(pairs) > 3:
            raise ValueError("at most three axes")
        a, b, c = pairs + (0,) * (3 - len(pairs))
        return _ROTARY.pack(self.rot_dim, _LAYOUTS[self.layout], len(pairs), a, b, c, self.factor,
                            inverse)


def _int(x, name):
    """x as an int of 32 bits; ctypes would cut a larger one to its low bits."""
    x = int(x)
    if not -0x80000000 <= x < 0x80000000:
        raise ValueError(f"{name} = {x} does not fit into 32 bits")
    return x


def _hints(max_new, max_kv):
    return _int(max_new or 0, "max_new"), _int(max_kv or 0, "max_kv")


def _like(t, stream):
    if stream is None:
        return _torch().empty_like(t)
    return _make(stream, _torch().empty_like, t)


def _new(t, shape, dtype, stream):
    if stream is None:
        return t.new_empty(shape, dtype=dtype)
    return _make(stream, t.new_empty, shape, dtype=dtype)


def _dtype_code(t, name):
    torch = _torch()
    if t.dtype == torch.bfloat16:
        return BF16
    if t.dtype == torch.float32:
        return F32
    raise ValueError(f"{name} must be bfloat16 or float32 (got {t.dtype})")


# (Host time is what the smallest calls are bound by. get_device() is the device's index, -1
# off the GPU, at a fraction of what comparing device objects costs.)
def _on(t, name, index, dtype=None, shape=None):
    """Address of a contiguous tensor on GPU `index` (None: any)."""
    try:
        at = t.get_device()
    except AttributeError:
        raise TypeError(f"{name} must be a torch.Tensor") from None
    if at < 0 or (at != index and index is not None):
        raise ValueError(f"{name} must be on the GPU" + (
            "" if index is None else f" cuda:{index}") + f" (got {t.device})")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if dtype is not None and t.dtype is not dtype:
        raise ValueError(f"{name} must be {dtype} (got {t.dtype})")
    if shape is not None and t.shape != shape:
        raise ValueError(f"{name} must have shape {tuple(shape)} (got {tuple(t.shape)})")
    return t.data_ptr()


def _rows(t, name, index, dtype, tokens, d, heads=None):
    """sparsp_rows of a [heads, tokens, d] tensor."""
    try:
        at, shape = t.get_device(), t.shape
    except AttributeError:
        raise TypeError(f"{name} must be a torch.Tensor") from None
    if len(shape) != 3 or at != index or t.dtype is not dtype:
        raise ValueError(f"{name} must be a [heads, tokens, d] {dtype} tensor on the GPU "
                         f"cuda:{index} (got {tuple(shape)} {t.dtype} on {t.device})")
    h, n, c = shape
    if n != tokens or c != d or (heads is not None and h != heads):
        raise ValueError(f"{name} must have shape {(heads or h, tokens, d)} (got {tuple(shape)})")
    sh, st, sc = t.stride()
    if sc != 1:
        raise ValueError(f"{name} must have contiguous channels")
    # An axis of one entry, or a tensor of none, is never stepped along.
    if n <= 1:
        st = d
    if h <= 1 or not n:
        sh = d
    return _ROWS.pack(t.data_ptr() or 16, sh, st, h, 0)


def _call(fn, index, stream, *args):
    """The library call on GPU `index`, which launches need to be current, and its stream."""
    cuda = _torch()._C
    if stream is None:
        raw = cuda._cuda_getCurrentRawStream(index)
    elif stream.device.index != index:
        raise ValueError(f"the stream is on {stream.device}, the tensors on cuda:{index}")
    else:
        raw = stream.cuda_stream
    if cuda._cuda_getDevice() == index:
        rc = fn(*args, raw)
    else:
        with _torch().cuda.device(index):
            rc = fn(*args, raw)
    if rc < 0:
        _check(rc)


def _positions(rotary, positions, inv_freq, tokens, index):
    torch = _torch()
    if not isinstance(positions, torch.Tensor):
        raise TypeError("positions must be a torch.Tensor")
    if positions.dtype not in (torch.int32, torch.int64):
        raise ValueError(f"positions must be int32 or int64 (got {positions.dtype})")
    p = positions if positions.dim() == 2 else positions.view(1, -1)
    return (_on(p, "positions", index, None, (rotary.axes, tokens)) or 16,
            32 if positions.dtype == torch.int32 else 64,
            _on(inv_freq, "inv_freq", index, torch.float32, (rotary.rot_dim // 2,)))


def sparsp_rope_frequencies(rot_dim: int, theta: float = 10000.0, scaling: str = "plain",
                            scale: float = 1.0, trained: float = 0.0, low: float = 1.0,
                            high: float = 32.0) -> tuple:
    """Frequencies of rot_dim // 2 pairs (host). Returns (inv_freq float32 numpy, factor).

    scaling: "plain", "linear" (all frequencies over scale), "base" (the base raised so that the
    lowest frequency is divided by scale) or "parts" (frequencies of fewer than `low` turns over
    `trained` tokens divided, of more than `high` kept, a ramp between; factor 0.1 ln scale + 1).
    """
    import numpy as np
    if scaling not in _SCALINGS:
        raise ValueError(f"scaling must be one of {sorted(_SCALINGS)} (got {scaling!r})")
    rot_dim = _int(rot_dim, "rot_dim")
    f = np.empty(min(max(1, rot_dim // 2), 128), dtype=np.float32)  # (longer ones are refused)
    factor = ctypes.c_float()
    _check(load_library().sparsp_rope_frequencies(rot_dim, float(theta), _SCALINGS[scaling],
                                                  float(scale), float(trained), float(low),
                                                  float(high), f.ctypes.data,
                                                  ctypes.addressof(factor)))
    return f, factor.value


def sparsp_rope(rotary: Rotary, X, positions, inv_freq, X2=None, Y=None, Y2=None,
                inverse: bool = False, stream=None):
    """X [heads, tokens, d] rotated to positions [axes, tokens] (or [tokens]); X2 alike.

    Returns Y (in X's order of heads and tokens, unless given), or (Y, Y2) with X2. Y may be X (in
    place). With inverse the transposed rotation: it turns back (times factor squared), and
    carries a gradient of Y to one of X.
    """
    torch = _torch()
    if not isinstance(X, torch.Tensor):
        raise TypeError("X must be a torch.Tensor")
    code = _dtype_code(X, "X")
    if X.dim() != 3 or not X.is_cuda:
        raise ValueError("X must be a [heads, tokens, d] tensor on the GPU")
    dev, (_, n, d) = X.get_device(), X.shape
    y = Y if Y is not None else _like(X, stream)
    x, count = _rows(X, "X", dev, X.dtype, n, d), 1
    o = _rows(y, "Y", dev, X.dtype, n, d, X.shape[0])
    y2 = None
    if X2 is not None:
        x += _rows(X2, "X2", dev, X.dtype, n, d)
        y2 = Y2 if Y2 is not None else _like(X2, stream)
        o += _rows(y2, "Y2", dev, X.dtype, n, d, X2.shape[0])
        count = 2
    elif Y2 is not None:
        raise ValueError("Y2 needs X2")
    pos, bits, freq = _positions(rotary, positions, inv_freq, n, dev)
    _call(load_library().sparsp_rope, dev, stream, rotary._pack(inverse), n, d, code, x, o, count,
          pos, bits, freq)
    return y if X2 is None else (y, y2)


def _cache(K_cache, V_cache, weights, page_table, new_off, kv_len):
    """(sparsp_cache, GPU) of the cache's tensors; V_cache, weights, new_off may be None."""
    torch = _torch()
    if not isinstance(K_cache, torch.Tensor):
        raise TypeError("K_cache must be a torch.Tensor")
    if K_cache.dim() != 4:
        raise ValueError("K_cache must be [pages, H, page, d]")
    shape, i32 = K_cache.shape, torch.int32
    if not isinstance(page_table, torch.Tensor) or page_table.dim() != 2:
        raise ValueError("page_table must be an int32 [B, width] tensor")
    B, width = page_table.shape
    k = _on(K_cache, "K_cache", None)
    dev = K_cache.get_device()
    v = 0 if V_cache is None else _on(V_cache, "V_cache", dev, K_cache.dtype, shape)
    w = 0 if weights is None else _on(weights, "weights", dev, torch.float32, shape[:3])
    return _CACHE.pack(
        k, v, w, _on(page_table, "page_table", dev, i32),
        0 if new_off is None else _on(new_off, "new_off", dev, i32, (B + 1,)),
        _on(kv_len, "kv_len", dev, i32, (B,)), shape[0], shape[1], shape[2], shape[3],
        _dtype_code(K_cache, "K_cache"), width, B, 0), dev


def sparsp_paged_append(K, V, K_cache, V_cache, page_table, new_off, kv_len, weights=None,
                        rotary: Optional[Rotary] = None, positions=None, inv_freq=None, Q=None,
                        Q_out=None, stream=None):
    """Writes the new tokens' K, V [H, tokens, d] into the cache (and 0 into weights, if given).

    With a rotation K is rotated to its positions on the way, and so is Q, into Q_out (which may
    be Q). Returns Q_out, or None without Q.
    """
    c, dev = _cache(K_cache, V_cache, weights, page_table, new_off, kv_len)
    if K.dim() != 3:
        raise ValueError("K must be [H, tokens, d]")
    H, n, d, dt = K_cache.shape[1], K.shape[1], K_cache.shape[3], K_cache.dtype
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
    _call(load_library().sparsp_paged_append, dev, stream, c, n, _rows(K, "K", dev, dt, n, d, H),
          _rows(V, "V", dev, dt, n, d, H), rot, pos, bits, freq, q, qo)
    return Q_out


def sparsp_paged_attn_workspace_bytes(K_cache, page_table, tokens: int, q_heads: int,
                                      max_new: int = 0, max_kv: int = 0,
                                      window: Optional[int] = None, sinks: int = 0) -> int:
    """Workspace bytes that sparsp_paged_attn can use for these shapes (host)."""
    B, width = page_table.shape
    P, H, page, d = K_cache.shape
    c = _CACHE.pack(0, 0, 0, 0, 0, 0, P, H, page, d, _dtype_code(K_cache, "K_cache"), width, B, 0)
    c = (c, _int(tokens, "tokens"), _int(q_heads, "q_heads"))
    if window is None and not sinks:
        n = load_library().sparsp_paged_attn_workspace_bytes(*c, *_hints(max_new, max_kv))
    else:
        n = load_library().sparsp_paged_attn_window_workspace_bytes(
            *c, *_window(window, sinks, True), *_hints(max_new, max_kv))
    n = int(n)
    _check(n if n < 0 else 0)
    return n


def _window(window, sinks, causal):
    if window is None or not causal:
        raise ValueError("sinks need a window" if window is None else
                         "a window needs causal attention")
    return _int(window, "window"), _int(sinks, "sinks")


def _scale(softmax_scale, d):
    return 1.0 / math.sqrt(d) if softmax_scale is None else float(softmax_scale)


def sparsp_paged_attn(Q, K_cache, V_cache, page_table, new_off, kv_len, causal: bool = True,
                      softmax_scale: Optional[float] = None, max_new: Optional[int] = None,
                      max_kv: Optional[int] = None, O=None, lse=None, want_lse: bool = True,
                      out_dtype: Optional[int] = None, workspace=None, stream=None,
                      window: Optional[int] = None, sinks: int = 0):
    """Attention of the new tokens Q [heads, tokens, d] over the cache. Returns (O, lse or None).

    O is [heads, tokens, d] (contiguous unless given), lse float32 [heads, tokens]. max_new and
    max_kv, the largest numbers of new and of cached tokens if the caller knows them, size the
    launch. With workspace (any device tensor, e.g. of sparsp_paged_attn_workspace_bytes bytes)
    long caches are split among workgroups; without, one workgroup walks a sequence's keys.

    window: a token sees itself and the window - 1 tokens before it, and the sequence's first
    `sinks` ones. Pages that no row sees are not read; their table entries may name no page. The lse
    is then not one for sparsp_paged_weights, whose rows see the whole cache.
    """
    torch = _torch()
    c, dev = _cache(K_cache, V_cache, None, page_table, new_off, kv_len)
    d, dt = K_cache.shape[3], K_cache.dtype
    if Q.dim() != 3:
        raise ValueError("Q must be [heads, tokens, d]")
    heads, n = Q.shape[0], Q.shape[1]
    if out_dtype is None:
        out_dtype = _dtype_code(K_cache, "K_cache")
    odt = torch.bfloat16 if out_dtype == BF16 else torch.float32
    o = O if O is not None else _new(Q, (heads, n, d), odt, stream)
    ls = lse
    if ls is None and want_lse:
        ls = _new(Q, (heads, n), torch.float32, stream)
    ws, nbytes = None, 0
    if workspace is not None:
        ws = _on(workspace, "workspace", dev)
        nbytes = workspace.numel() * workspace.element_size()
    if window is None and not sinks:
        fn, seen = load_library().sparsp_paged_attn, (bool(causal),)
    else:
        fn, seen = load_library().sparsp_paged_attn_window, _window(window, sinks, causal)
    _call(fn, dev, stream, c, n, _rows(Q, "Q", dev, dt, n, d),
          _rows(o, "O", dev, odt, n, d, heads), _int(out_dtype, "out_dtype"),
          None if ls is None else _on(ls, "lse", dev, torch.float32, (heads, n)),
          *seen, _scale(softmax_scale, d), *_hints(max_new, max_kv), ws, nbytes)
    return o, ls


def sparsp_paged_weights(Q, lse, K_cache, page_table, new_off, kv_len, weights,
                         causal: bool = True, softmax_scale: Optional[float] = None,
                         accumulate: bool = True, max_new: Optional[int] = None,
                         max_kv: Optional[int] = None, stream=None):
    """Adds (or with accumulate=False writes) the attention weight of every cached token.

    Q, lse and the other arguments as given to and returned by sparsp_paged_attn; weights
    float32 [pages, H, page]. Returns weights. No two sequences may share a page (as they do after
    sparsp_pages_fork).
    """
    torch = _torch()
    c, dev = _cache(K_cache, None, weights, page_table, new_off, kv_len)
    if Q.dim() != 3:
        raise ValueError("Q must be [heads, tokens, d]")
    heads, n, d = Q.shape
    if d != K_cache.shape[3]:
        raise ValueError(f"Q must have d = {K_cache.shape[3]} (got {d})")
    if weights is None:
        raise TypeError("weights must be a torch.Tensor")
    _call(load_library().sparsp_paged_weights, dev, stream, c, n,
          _rows(Q, "Q", dev, K_cache.dtype, n, d),
          _on(lse, "lse", dev, torch.float32, (heads, n)) or 16, bool(causal),
          _scale(softmax_scale, d), bool(accumulate), *_hints(max_new, max_kv))
    return weights


def sparsp_cache_evict(K_cache, V_cache, weights, page_table, kv_len, keep: int, first: int = 0,
                       recent: int = 0, dst_table=None, kv_len_out=None, kept=None, workspace=None,
                       stream=None):
    """Cuts every sequence of more than `keep` tokens to `keep`: its first and recent ones, and
    of the others, per head, those of most weight. Returns (kv_len_out [B], kept [B, H, keep]).

    The kept tokens move to the front of the sequence's pages, or into the pages of dst_table
    (int32 [B, width], none of them in page_table). kept lists them, ascending, then -1. Few long
    sequences use a workspace (sparsp_cache_evict_workspace_bytes bytes), which is allocated here
    unless one is given, like the outputs. No two sequences may share a page (as they do after
    sparsp_pages_fork): cutting one would move the other's tokens.
    """
    torch = _torch()
    c, dev = _cache(K_cache, V_cache, weights, page_table, None, kv_len)
    B, H = page_table.shape[0], K_cache.shape[1]
    keep, first, recent = _int(keep, "keep"), _int(first, "first"), _int(recent, "recent")
    out = kv_len_out if kv_len_out is not None else _like(kv_len, stream)
    lst = kept if kept is not None else _new(kv_len, (B, H, max(keep, 0)), torch.int32, stream)
    dst, dst_width = None, 0
    if dst_table is not None:
        if dst_table.dim() != 2 or dst_table.shape[0] != B:
            raise ValueError(f"dst_table must be an int32 [{B}, width] tensor")
        dst, dst_width = _on(dst_table, "dst_table", dev, torch.int32), dst_table.shape[1]
    lib = load_library()
    if workspace is None:
        nbytes = lib.sparsp_cache_evict_workspace_bytes(c)
        if nbytes > 0:
            workspace = _new(K_cache, (nbytes,), torch.uint8, stream)
    ws = None if workspace is None else _on(workspace, "workspace", dev)
    nbytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _call(lib.sparsp_cache_evict, dev, stream, c, keep, first, recent, dst, dst_width,
          _on(out, "kv_len_out", dev, torch.int32, (B,)),
          _on(lst, "kept", dev, torch.int32, (B, H, max(keep, 0))), ws, nbytes)
    return out, lst


def sparsp_cache_evict_workspace_bytes(K_cache, page_table) -> int:
    """Workspace bytes that sparsp_cache_evict can use for these shapes (host)."""
    B, width = page_table.shape
    P, H, page, d = K_cache.shape
    c = _CACHE.pack(0, 0, 0, 0, 0, 0, P, H, page, d, _dtype_code(K_cache, "K_cache"), width, B, 0)
    n = int(load_library().sparsp_cache_evict_workspace_bytes(c))
    _check(n if n < 0 else 0)
    return n


rope_frequencies = sparsp_rope_frequencies
rope = sparsp_rope
paged_append = sparsp_paged_append
paged_attn = sparsp_paged_attn
paged_attn_workspace_bytes = sparsp_paged_attn_workspace_bytes
paged_weights = sparsp_paged_weights
cache_evict = sparsp_cache_evict
cache_evict_workspace_bytes = sparsp_cache_evict_workspace_bytes
