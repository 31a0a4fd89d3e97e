"""The paged cache without a GPU: the C ABI's checks under sanitizers, the rotary frequencies, and
what the binding refuses."""

import math
import os
import re
import shutil
import subprocess

import numpy as np
import pytest
import torch

import paper_2609_32197_amd as sp

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2609_32197_amd", "csrc")
CHECK = os.path.join(ROOT, "tests", "hostcheck")
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")


def test_abi_under_asan_and_ubsan(tmp_path):
    cxx = os.environ.get("CXX") or shutil.which("g++")
    if not cxx or not os.path.exists(os.path.join(ROCM, "include", "hip", "hip_runtime_api.h")):
        pytest.skip("needs g++ and the HIP runtime API headers")
    exe = str(tmp_path / "cache_host_check")
    srcs = [os.path.join(CSRC, f) for f in ("api.cpp", "api_cache.cpp", "host_plan.cpp")]
    srcs += [os.path.join(CHECK, f) for f in ("stub_launchers.cpp", "cache_stub_launchers.cpp",
                                              "cache_host_check.cpp")]
    r = subprocess.run([cxx, "-std=c++17", "-O1", "-g", "-fno-omit-frame-pointer",
                        "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
                        "-D__HIP_PLATFORM_AMD__", f"-I{os.path.join(ROCM, 'include')}", *srcs, "-o",
                        exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, (r.stdout + r.stderr)[-4000:]
    assert " 0 failures" in r.stdout


def test_library_exports_every_declared_symbol():
    text = open(os.path.join(ROOT, "include", "sparsp_cache.h")).read()
    names = re.findall(r"^(?:int|int64_t)\s+(sparsp_\w+)\s*\(", text, re.M)
    assert len(names) == 8
    for name in names:
        assert hasattr(sp.load_library(), name), name


@pytest.mark.parametrize("rot,theta", [(2, 10000.0), (64, 10000.0), (128, 500000.0)])
def test_frequencies(rot, theta):
    p = np.arange(rot // 2, dtype=np.float64)
    plain = theta ** (-2 * p / rot)
    f, s = sp.sparsp_rope_frequencies(rot, theta)
    assert s == 1.0 and f.dtype == np.float32
    np.testing.assert_allclose(f, plain, rtol=1.01 * 2.0 ** -24)
    f, s = sp.sparsp_rope_frequencies(rot, theta, "linear", 8.0)
    np.testing.assert_allclose(f, plain / 8, rtol=1.01 * 2.0 ** -24)
    if rot > 2:
        f, s = sp.sparsp_rope_frequencies(rot, theta, "base", 8.0)
        # The highest frequency stays 1, the lowest is divided by the scale.
        assert f[0] == 1.0 and s == 1.0
        np.testing.assert_allclose(f[-1], plain[-1] / 8, rtol=2.0 ** -23)
    f, s = sp.sparsp_rope_frequencies(rot, theta, "parts", 8.0, trained=4096, low=1, high=32)
    turns = 4096 * plain / (2 * math.pi)
    g = np.clip((turns - 1) / 31, 0, 1)
    np.testing.assert_allclose(f, plain * (g + (1 - g) / 8), rtol=2.0 ** -23)
    assert abs(s - (0.1 * math.log(8.0) + 1)) < 2.0 ** -23
    assert (f[turns > 32] == plain[turns > 32].astype(np.float32)).all()


def test_frequencies_refused():
    for kw in (dict(rot_dim=7), dict(rot_dim=0), dict(rot_dim=300), dict(rot_dim=8, theta=-1.0),
               dict(rot_dim=8, scaling="linear", scale=0.0), dict(rot_dim=2, scaling="base", scale=2),
               dict(rot_dim=8, scaling="parts", scale=2)):
        with pytest.raises(sp.SparspError):
            sp.sparsp_rope_frequencies(**kw)
    with pytest.raises(ValueError):
        sp.sparsp_rope_frequencies(8, scaling="other")


def test_binding_wants_the_gpu():
    x = torch.zeros(2, 3, 64)
    i = torch.zeros(1, 4, dtype=torch.int32)
    c = torch.zeros(4, 2, 16, 64)
    off, kv = torch.zeros(2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError, match="GPU"):
        sp.sparsp_rope(sp.Rotary(64), x, torch.zeros(3, dtype=torch.int32), torch.zeros(32))
    for call in (lambda: sp.sparsp_paged_append(x, x, c, c, i, off, kv),
                 lambda: sp.sparsp_paged_attn(x, c, c, i, off, kv),
                 lambda: sp.sparsp_paged_weights(x, x[..., 0], c, i, off, kv, c[..., 0].contiguous()),
                 lambda: sp.sparsp_cache_evict(c, c, c[..., 0].contiguous(), i, kv, 3)):
        with pytest.raises(ValueError, match="GPU"):
            call()


def test_rotary_refused():
    with pytest.raises(ValueError, match="layout"):
        sp.Rotary(64, "other")._pack(False)
    with pytest.raises(ValueError, match="axes"):
        sp.Rotary(64, "half", (8, 8, 8, 8))._pack(False)


def test_workspace_bytes():
    c, t = torch.zeros(4, 2, 16, 64), torch.zeros(2, 300, dtype=torch.int32)
    assert sp.sparsp_paged_attn_workspace_bytes(c, t, 2, 4, 1, 100) == 0  # short: no split
    n = sp.sparsp_paged_attn_workspace_bytes(c, t, 2, 4, 1)
    assert n > 0 and n % (2 * 4 * 65 * 4) == 0
    with pytest.raises(sp.SparspError):
        sp.sparsp_paged_attn_workspace_bytes(c, t, 2, 3)
    assert sp.sparsp_cache_evict_workspace_bytes(c, t) == 0  # 4,800 tokens: one workgroup each
    long = torch.zeros(2, 3000, dtype=torch.int32)
    n = sp.sparsp_cache_evict_workspace_bytes(c, long)
    assert n >= 4 * 2 * 2 * 48000 and n % 16 == 0
