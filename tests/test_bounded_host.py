"""The bounded cache without a GPU: what its entry points refuse before anything is launched."""

import os
import re

import pytest
import torch

import paper_2609_32197_amd as sp
from paper_2609_32197_amd.paged import _CACHE, _ROWS

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
AT = 1 << 20  # an address that no refused call touches


def cache(**kw):
    v = dict(K=AT, V=2 * AT, weights=0, table=AT, new_off=AT, kv_len=AT, pages=9, H=2, page=16, d=64,
             dtype=sp.BF16, width=4, B=3, reserved=0)
    v.update(kw)
    return _CACHE.pack(*v.values())


def rows(at=3 * AT, heads=4, tokens=5, d=64):
    return _ROWS.pack(at, tokens * d, d, heads, 0)


def status(rc):
    assert rc < 0, "not refused"
    return sp.STATUS[rc], sp.load_library().sparsp_last_error().decode()


def test_library_exports_every_declared_symbol():
    text = open(os.path.join(ROOT, "include", "sparsp_bounded.h")).read()
    names = re.findall(r"^(?:int|int64_t)\s+(sparsp_\w+)\s*\(", text, re.M)
    assert names
    for name in names:
        assert hasattr(sp.load_library(), name), name


def window_call(c=None, Q=None, O=None, window=5, sinks=1, scale=0.1, tokens=5, max_kv=0, ws=0,
                nbytes=0, out=sp.BF16):
    return sp.load_library().sparsp_paged_attn_window(
        c or cache(), tokens, Q or rows(), O or rows(5 * AT), out, None, window, sinks, scale, 0,
        max_kv, ws, nbytes, None)


@pytest.mark.parametrize("kw,code,word", [
    (dict(window=0), "SPARSP_E_INVALID", "window"),
    (dict(window=-2 ** 31), "SPARSP_E_INVALID", "window"),
    (dict(sinks=-1), "SPARSP_E_INVALID", "sinks"),
    (dict(c=cache(H=3)), "SPARSP_E_INVALID", "query heads"),
    (dict(c=cache(page=24)), "SPARSP_E_UNSUPPORTED", "page"),
    (dict(c=cache(kv_len=0)), "SPARSP_E_INVALID", "NULL"),
    (dict(scale=0.0), "SPARSP_E_INVALID", "scale"),
    (dict(O=rows()), "SPARSP_E_INVALID", "O may not be Q"),
    (dict(out=7), "SPARSP_E_DTYPE", "out_dtype"),
    (dict(ws=AT + 4, nbytes=64), "SPARSP_E_INVALID", "aligned"),
    (dict(max_kv=-1), "SPARSP_E_INVALID", "max_"),
])
def test_window_refused(kw, code, word):
    got, message = status(window_call(**kw))
    assert got == code and word in message


def test_window_without_tokens_does_nothing():
    assert window_call(tokens=0, Q=rows(tokens=1), O=rows(5 * AT, tokens=1)) == 0


def test_window_workspace():
    c, t = torch.zeros(4, 2, 16, 64), torch.zeros(2, 3000, dtype=torch.int32)
    whole = sp.sparsp_paged_attn_workspace_bytes(c, t, 2, 4, 1)
    n = [sp.sparsp_paged_attn_workspace_bytes(c, t, 2, 4, 1, window=w, sinks=s)
         for w, s in ((10, 0), (4000, 4), (2 ** 31 - 1, 2 ** 31 - 1))]
    assert n[0] == 0 < n[1] < whole == n[2]
    for kw in (dict(window=0), dict(window=3, sinks=-1)):
        with pytest.raises(sp.SparspError):
            sp.sparsp_paged_attn_workspace_bytes(c, t, 2, 4, 1, **kw)
    with pytest.raises(ValueError):
        sp.sparsp_paged_attn_workspace_bytes(c, t, 2, 4, 1, sinks=3)


def test_binding_refuses_a_window_without_a_gpu():
    x, c = torch.zeros(2, 3, 64), torch.zeros(4, 2, 16, 64)
    i = torch.zeros(1, 4, dtype=torch.int32)
    off, kv = torch.zeros(2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError, match="GPU"):
        sp.sparsp_paged_attn(x, c, c, i, off, kv, window=5)
