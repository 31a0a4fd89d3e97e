"""The bounded cache without a GPU: what its entry points refuse before anything is launched."""

import os
import re
import shutil
import subprocess

import pytest
import torch

import paper_2609_32197_amd as sp
from paper_2609_32197_amd.bounded import _BUFFER, _CACHE4, _PAGES
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


def test_abi_under_asan_and_ubsan(tmp_path):
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    cxx = os.environ.get("CXX") or shutil.which("g++")
    if not cxx or not os.path.exists(os.path.join(rocm, "include", "hip", "hip_runtime_api.h")):
        pytest.skip("needs g++ and the HIP runtime API headers")
    exe = str(tmp_path / "bounded_host_check")
    csrc = os.path.join(ROOT, "paper_2609_32197_amd", "csrc")
    srcs = [os.path.join(csrc, f) for f in ("api.cpp", "api_cache.cpp", "api_bounded.cpp",
                                            "host_plan.cpp")]
    srcs += [os.path.join(ROOT, "tests", "hostcheck", f)
             for f in ("stub_launchers.cpp", "cache_stub_launchers.cpp", "bounded_stub_launchers.cpp",
                       "bounded_host_check.cpp")]
    r = subprocess.run([cxx, "-std=c++17", "-O1", "-g", "-fno-omit-frame-pointer",
                        "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
                        "-D__HIP_PLATFORM_AMD__", f"-I{os.path.join(rocm, 'include')}", *srcs, "-o",
                        exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, (r.stdout + r.stderr)[-4000:]
    assert " 0 failures" in r.stdout


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


# ---------------------------------------------------------------------------
# the 4-bit cache
# ---------------------------------------------------------------------------


def cache4(**kw):
    v = dict(K=AT, Ks=2 * AT, V=3 * AT, Vs=4 * AT, table=AT, new_off=AT, kv_len=AT, pages=9, H=2,
             page=16, d=64, width=4, B=3, r0=0, r1=0)
    v.update(kw)
    return _CACHE4.pack(*v.values())


ROTARY = sp.Rotary(64)._pack(False)


def append4(c=None, dtype=sp.BF16, K=None, V=None, r=ROTARY, pos=AT, bits=32, Q=None, Qo=None, tokens=5):
    return sp.load_library().sparsp_paged_append4(
        c or cache4(), tokens, dtype, K or rows(heads=2), V or rows(6 * AT, heads=2), r, pos, bits, AT,
        Q, Qo, None)


@pytest.mark.parametrize("kw,code,word", [
    (dict(c=cache4(d=48)), "SPARSP_E_UNSUPPORTED", "multiple of 32"),
    (dict(c=cache4(d=160)), "SPARSP_E_UNSUPPORTED", "multiple of 32"),
    (dict(c=cache4(d=0)), "SPARSP_E_INVALID", "d = 0"),
    (dict(c=cache4(page=8)), "SPARSP_E_UNSUPPORTED", "page"),
    (dict(c=cache4(Ks=0)), "SPARSP_E_INVALID", "NULL"),
    (dict(c=cache4(Vs=AT + 8)), "SPARSP_E_INVALID", "aligned"),
    (dict(c=cache4(V=AT)), "SPARSP_E_INVALID", "same memory"),
    (dict(c=cache4(Vs=2 * AT)), "SPARSP_E_INVALID", "same memory"),
    (dict(dtype=5), "SPARSP_E_DTYPE", "dtype"),
    (dict(K=rows(heads=3)), "SPARSP_E_INVALID", "heads"),
    (dict(K=rows(3 * AT + 2, heads=2)), "SPARSP_E_INVALID", "16 bytes"),
    (dict(bits=16), "SPARSP_E_DTYPE", "position_bits"),
    (dict(pos=0), "SPARSP_E_INVALID", "positions"),
    (dict(Q=rows(7 * AT)), "SPARSP_E_INVALID", "Q_out"),
    (dict(Q=rows(7 * AT), Qo=rows(8 * AT), r=None), "SPARSP_E_INVALID", "rotation"),
    (dict(Q=rows(7 * AT), Qo=rows(3 * AT)), "SPARSP_E_INVALID", "Q_out"),
    (dict(Q=rows(7 * AT), Qo=rows(8 * AT, heads=5)), "SPARSP_E_INVALID", "heads"),
    (dict(Q=rows(7 * AT), Qo=_ROWS.pack(8 * AT, 64, 64, 4, 0)), "SPARSP_E_INVALID", "overlap"),
    (dict(tokens=-1), "SPARSP_E_INVALID", "tokens"),
])
def test_append4_refused(kw, code, word):
    got, message = status(append4(**kw))
    assert got == code and word in message


@pytest.mark.parametrize("K,V,word", [
    (rows(heads=2), rows(heads=2), "same memory"),
    (rows(heads=1), rows(6 * AT, heads=2), "heads"),
    (rows(heads=2), _ROWS.pack(6 * AT, 64, 64, 2, 0), "overlap"),
])
def test_read4_refused(K, V, word):
    _, message = status(sp.load_library().sparsp_paged_read4(cache4(), 5, sp.F32, K, V, None))
    assert word in message


def attn4(c=None, dtype=sp.BF16, O=None, out=sp.BF16, causal=1, window=0, sinks=0, nbytes=0):
    return sp.load_library().sparsp_paged_attn4(
        c or cache4(), 5, dtype, rows(), O or rows(5 * AT), out, None, causal, window, sinks, 0.1, 0, 0,
        None, nbytes, None)


@pytest.mark.parametrize("kw,code,word", [
    (dict(window=-1), "SPARSP_E_INVALID", "window"),
    (dict(window=4, sinks=-1), "SPARSP_E_INVALID", "sinks"),
    (dict(sinks=4), "SPARSP_E_INVALID", "sinks need a window"),
    (dict(window=4, causal=0), "SPARSP_E_INVALID", "causal"),
    (dict(dtype=sp.F32), "SPARSP_E_DTYPE", "f32"),
    (dict(c=cache4(H=3)), "SPARSP_E_INVALID", "query heads"),
    (dict(c=cache4(V=0)), "SPARSP_E_INVALID", "NULL"),
    (dict(O=rows()), "SPARSP_E_INVALID", "O may not be Q"),
    (dict(nbytes=-1), "SPARSP_E_INVALID", "workspace_bytes"),
])
def test_attn4_refused(kw, code, word):
    got, message = status(attn4(**kw))
    assert got == code and word in message


def test_nothing_to_do():
    one = rows(heads=2, tokens=1), rows(6 * AT, heads=2, tokens=1)
    assert append4(tokens=0, K=one[0], V=one[1]) == 0
    assert sp.load_library().sparsp_paged_read4(cache4(), 0, sp.F32, *one, None) == 0


def test_attn4_workspace():
    c = sp.Cache4.zeros(4, 2, 16, 64, device="cpu")
    t = torch.zeros(2, 3000, dtype=torch.int32)
    whole = sp.sparsp_paged_attn4_workspace_bytes(c, t, 2, 4, 1)
    some = sp.sparsp_paged_attn4_workspace_bytes(c, t, 2, 4, 1, window=4000)
    assert 0 < some < whole
    assert sp.sparsp_paged_attn4_workspace_bytes(c, t, 2, 4, 1, 100, dtype=torch.float32) == 0
    with pytest.raises(sp.SparspError):
        sp.sparsp_paged_attn4_workspace_bytes(c, t, 2, 3)
    for kw in (dict(window=0), dict(sinks=1), dict(dtype=torch.float16)):
        with pytest.raises(ValueError):
            sp.sparsp_paged_attn4_workspace_bytes(c, t, 2, 4, **kw)


def test_binding_of_the_4_bit_cache_wants_the_gpu():
    c = sp.Cache4.zeros(4, 2, 16, 64, device="cpu")
    x = torch.zeros(2, 3, 64, dtype=torch.bfloat16)
    i = torch.zeros(1, 4, dtype=torch.int32)
    off, kv = torch.zeros(2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    for call in (lambda: sp.sparsp_paged_append4(x, x, c, i, off, kv),
                 lambda: sp.sparsp_paged_read4(c, i, off, kv, 3),
                 lambda: sp.sparsp_paged_attn4(x, c, i, off, kv)):
        with pytest.raises(ValueError, match="GPU"):
            call()
    with pytest.raises(TypeError):
        sp.sparsp_paged_attn4(x, c.K, i, off, kv)
    with pytest.raises(ValueError):
        sp.Cache4.zeros(4, 2, 16, 48, device="cpu")


# ---------------------------------------------------------------------------
# pages
# ---------------------------------------------------------------------------


def pages(**kw):
    v = dict(refs=AT, table=2 * AT, kv_len=3 * AT, pages=9, page=16, width=4, B=3)
    v.update(kw)
    return _PAGES.pack(*v.values())


def buffers(*pairs):
    return b"".join(_BUFFER.pack(*x) for x in pairs)


def fork(p=None, parents=AT, n=3, b=buffers((AT, 64)), count=1, out=(4 * AT, 5 * AT, 6 * AT, 7 * AT),
         ws=8 * AT, nbytes=1 << 20):
    return sp.load_library().sparsp_pages_fork(p or pages(), parents, n, b, count, *out, ws, nbytes, None)


@pytest.mark.parametrize("kw,code,word", [
    (dict(p=pages(refs=0)), "SPARSP_E_INVALID", "NULL"),
    (dict(p=pages(kv_len=0)), "SPARSP_E_INVALID", "NULL"),
    (dict(p=pages(pages=0)), "SPARSP_E_INVALID", "positive"),
    (dict(p=pages(page=48)), "SPARSP_E_UNSUPPORTED", "page"),
    (dict(p=pages(width=1 << 27)), "SPARSP_E_UNSUPPORTED", "2^30"),
    (dict(p=pages(width=1 << 16, B=1 << 15)), "SPARSP_E_UNSUPPORTED", "2^30"),
    (dict(parents=0), "SPARSP_E_INVALID", "NULL"),
    (dict(n=0), "SPARSP_E_UNSUPPORTED", "rows"),
    (dict(n=65537), "SPARSP_E_UNSUPPORTED", "rows"),
    (dict(count=9), "SPARSP_E_INVALID", "buffers"),
    (dict(b=None), "SPARSP_E_INVALID", "buffers"),
    (dict(b=buffers((AT, 24))), "SPARSP_E_INVALID", "multiple of 16"),
    (dict(b=buffers((AT, 0))), "SPARSP_E_INVALID", "multiple of 16"),
    (dict(b=buffers((AT + 4, 32))), "SPARSP_E_INVALID", "aligned"),
    (dict(b=buffers((AT, 32), (2 * AT, 32), (AT, 32)), count=3), "SPARSP_E_INVALID", "same memory"),
    (dict(out=(2 * AT, 5 * AT, 6 * AT, 7 * AT)), "SPARSP_E_INVALID", "inputs"),
    (dict(out=(4 * AT, 3 * AT, 6 * AT, 7 * AT)), "SPARSP_E_INVALID", "inputs"),
    (dict(out=(4 * AT, 5 * AT, AT, 7 * AT)), "SPARSP_E_INVALID", "inputs"),
    (dict(out=(4 * AT, 5 * AT, 6 * AT, 0)), "SPARSP_E_INVALID", "NULL"),
    (dict(ws=0), "SPARSP_E_INVALID", "workspace"),
    (dict(nbytes=100), "SPARSP_E_CAPACITY", "workspace"),
])
def test_fork_refused(kw, code, word):
    got, message = status(fork(**kw))
    assert got == code and word in message


def test_other_page_calls_refused():
    lib = sp.load_library()
    for call, word in (
            (lambda: lib.sparsp_pages_reserve(pages(), 0, AT, AT, 1 << 20, None), "NULL"),
            (lambda: lib.sparsp_pages_reserve(pages(), AT, 0, AT, 1 << 20, None), "NULL"),
            (lambda: lib.sparsp_pages_reserve(pages(), AT, AT, AT, 8, None), "workspace"),
            (lambda: lib.sparsp_pages_release(pages(), -1, 0, None), "window"),
            (lambda: lib.sparsp_pages_release(pages(), 0, 4, None), "sinks"),
            (lambda: lib.sparsp_pages_compact(pages(), None, 0, 2 * AT, 5 * AT, 6 * AT, AT, 1 << 20, None),
             "inputs"),
            (lambda: lib.sparsp_pages_compact(pages(), None, 0, 4 * AT, 5 * AT, 0, AT, 1 << 20, None), "NULL"),
            (lambda: lib.sparsp_pages_copy(buffers((AT, 16)), 0, 9, AT, AT, 3, None), "nothing"),
            (lambda: lib.sparsp_pages_copy(buffers((AT, 16)), 1, 0, AT, AT, 3, None), "pages"),
            (lambda: lib.sparsp_pages_copy(buffers((AT, 16)), 1, 9, AT, AT, -1, None), "moves"),
            (lambda: lib.sparsp_pages_copy(buffers((AT, 16)), 1, 9, 0, AT, 3, None), "NULL"),
            (lambda: lib.sparsp_pages_workspace_bytes(pages(page=8), 0), "page"),
            (lambda: lib.sparsp_pages_workspace_bytes(pages(), -1), "rows")):
        assert word in status(call())[1]
    assert lib.sparsp_pages_copy(buffers((AT, 16)), 1, 9, 0, 0, 0, None) == 0


def test_page_workspace_holds_its_lists():
    """counts, three lists of pages and one of rows, each on 4 bytes."""
    refs, table = torch.zeros(20000, dtype=torch.int32), torch.zeros(5, 7, dtype=torch.int32)
    for rows_ in (0, 5, 3000):
        n = sp.sparsp_pages_workspace_bytes(refs, table, rows_)
        assert n >= 4 * (3 * 20000 + max(rows_, 5) + 2 + -(-max(rows_, 5) // 1024) + 1)


def test_page_calls_want_the_gpu():
    i = torch.zeros(9, dtype=torch.int32)
    t, kv = torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    for call in (lambda: sp.sparsp_pages_reserve(i, t, i[:3], kv, 16),
                 lambda: sp.sparsp_pages_release(i, t, kv, 16),
                 lambda: sp.sparsp_pages_fork(i, t, kv, kv, 16),
                 lambda: sp.sparsp_pages_compact(i, t),
                 lambda: sp.sparsp_pages_copy(kv, kv, torch.zeros(9, 8))):
        with pytest.raises(ValueError, match="GPU"):
            call()
