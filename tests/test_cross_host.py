"""Host code of cross attention, read-back and page-scaled pools, on the CPU: refusals, coverage of
the (query, key) pairs by a call's units, streams and devices, over a stand-in for the HIP
runtime (tests/sanitize/cross_calls.cpp, built with AddressSanitizer and
UndefinedBehaviorSanitizer); and the binding's own checks."""

import os
import shutil
import subprocess

import numpy as np
import pytest
import torch

from paper_2609_32278_amd import kvx

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SAN = ["-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-fno-omit-frame-pointer"]


@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    if shutil.which("g++") is None or not os.path.exists("/opt/rocm/include/hip/hip_runtime.h"):
        pytest.skip("g++ or the HIP headers not installed")
    exe = str(tmp_path_factory.mktemp("cross") / "cross_calls")
    cmd = ["g++", "-std=c++17", *SAN, "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-I" + os.path.join(ROOT, "include"),
           "-I" + os.path.join(ROOT, "paper_2609_32278_amd", "csrc"),
           os.path.join(ROOT, "tests", "sanitize", "cross_calls.cpp"), "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        if "asan" in r.stderr.lower() or "ubsan" in r.stderr.lower():
            pytest.skip("sanitizer runtime not available: " + r.stderr[-300:])
        raise AssertionError(r.stderr[-3000:])
    return exe


@pytest.mark.parametrize("check", ["coverage", "drafts", "limits", "refusals", "streams", "pools", "memory"])
def test_host_calls(driver, check, tmp_path):
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1")
    run = subprocess.run([driver, check], capture_output=True, text=True, env=env, timeout=300, cwd=tmp_path)
    assert run.returncode == 0, run.stdout[-2000:] + run.stderr[-4000:]
    assert check + " passed" in run.stdout


@pytest.fixture
def geometry(monkeypatch):
    """A pool of 2 KV heads of 64 as the binding sees one; calls into the library are kept."""
    called = []

    class Lib:
        def __getattr__(self, name):
            return lambda *a: called.append(name) or 0

    monkeypatch.setattr(kvx, "lib", lambda: Lib())
    monkeypatch.setattr(kvx, "_geometry", lambda pool: (2, 64, 1))
    return called


def test_binding_refuses_wrong_buffers(geometry):
    b = kvx.Batch([20, 5], [3, 2], [0, 2, 3], 0x1000)
    bf16 = dict(dtype=torch.bfloat16)
    q, short, half = torch.zeros(5, 6, 64, **bf16), torch.zeros(5, 6, 63, **bf16), torch.zeros(5, 6, 64).half()
    for args in ((short, 0x10), (0x10, short), (half, 0x10), (0x10, half), (q.float(), 0x10)):
        with pytest.raises(ValueError):
            kvx.cross_attention(None, b, args[0], 6, 0.1, args[1])
    for lse in (torch.zeros(5, 6, dtype=torch.float64), torch.zeros(5, 5), torch.zeros(5, 6, dtype=torch.int32)):
        with pytest.raises(ValueError):
            kvx.cross_attention(None, b, 0x10, 6, 0.1, 0x10, lse)
    rows = torch.zeros(5, 2, 64, **bf16)
    for args in ((rows[:4], 0x10), (0x10, rows[:4]), (rows.float(), 0x10), (rows.half(), 0x10)):
        with pytest.raises(ValueError):
            kvx.load_kv(None, b, *args)
    with pytest.raises(ValueError):  # host memory
        kvx.cross_attention(None, b, q, 6, 0.1, 0x10)
    assert geometry == []
    kvx.cross_attention(None, b, 0x10, 6, 0.1, 0x20)
    kvx.load_kv(None, b, 0x10, 0x20)
    assert geometry == ["cross_attention", "load_kv"]


def test_raw_page_buffers_of_a_page_scaled_pool_hold_the_scales(monkeypatch):
    lay = {"num_kv_heads": 2, "head_dim": 64, "elem_bytes": 1, "kv_dtype": kvx.KVX_KV_FP8_PAGE}
    monkeypatch.setattr(kvx, "kv_pool_layout", lambda pool: lay)
    n = 3 * 2 * (16 * 64 + 4)
    enough, short = torch.zeros(n, dtype=torch.uint8), torch.zeros(n - 1, dtype=torch.uint8)
    kvx._page_buffers(None, 3, enough, enough)
    with pytest.raises(ValueError):
        kvx._page_buffers(None, 3, enough, short)
    lay["kv_dtype"] = kvx.KVX_KV_FP8_E4M3
    kvx._page_buffers(None, 3, short, short)


def test_calls_without_a_pool():
    b = kvx.Batch([16], [4], [0, 2], 0x1000)
    for call in (lambda: kvx.load_kv(None, b, 1, 1), lambda: kvx.cross_attention(None, b, 1, 4, 0.125, 1)):
        with pytest.raises(kvx.KvxError) as e:
            call()
        assert e.value.status == kvx.KVX_EINVAL
    for scales in ((np.ones(2), np.ones(2)), (None, np.ones(2))):
        with pytest.raises(kvx.KvxError) as e:
            kvx.kv_pool_create(8, 16, 2, 64, kvx.KVX_KV_FP8_PAGE, *scales)
        assert e.value.status == kvx.KVX_EINVAL
