"""Latent attention on the CPU: what the entry points refuse, how batches are planned, and the
binding's own checks.  tests/sanitize/latent_calls.cpp holds the checks that need the host code
itself, built with AddressSanitizer and UndefinedBehaviorSanitizer."""

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
    if shutil.which("g++") is None or not os.path.exists("/opt/rocm/lib/libamdhip64.so"):
        pytest.skip("g++ or the HIP runtime library not installed")
    exe = str(tmp_path_factory.mktemp("latent") / "latent_calls")
    cmd = ["g++", "-std=c++17", *SAN, "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-I" + os.path.join(ROOT, "include"),
           "-I" + os.path.join(ROOT, "paper_2609_32278_amd", "csrc"),
           os.path.join(ROOT, "tests", "sanitize", "latent_calls.cpp"),
           "-L/opt/rocm/lib", "-lamdhip64", "-Wl,-rpath,/opt/rocm/lib", "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        if "asan" in r.stderr.lower() or "ubsan" in r.stderr.lower():
            pytest.skip("sanitizer runtime not available: " + r.stderr[-300:])
        raise AssertionError(r.stderr[-3000:])
    return exe


@pytest.mark.parametrize("check", ["refusals", "absorbed", "expanded", "orders", "forms"])
def test_host(driver, check, tmp_path):
    # no leak check: the HIP runtime keeps what it allocated
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1")
    run = subprocess.run([driver, check], capture_output=True, text=True, env=env, timeout=300, cwd=tmp_path)
    assert run.returncode == 0, run.stdout[-2000:] + run.stderr[-4000:]
    assert check + " passed" in run.stdout


def test_binding_refuses_before_the_library(monkeypatch):
    """Tensors that are too small, of another size of element or not on the device never reach
    a kernel."""
    monkeypatch.setattr(kvx, "_latent_row", lambda pool: (512, 64))
    b = kvx.Batch([16], [4], [0, 2], 0x1000)
    cpu = torch.zeros(4, 576, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="device"):
        kvx.store_latent(None, b, cpu)
    with pytest.raises(ValueError, match="bf16"):
        kvx.store_latent(None, b, cpu.float())
    with pytest.raises(ValueError, match="bytes"):
        kvx.latent_attention(None, b, torch.zeros(3, 16, 576, dtype=torch.bfloat16), 16, 0.1, None)
    with pytest.raises(ValueError, match="float32"):
        kvx.latent_attention(None, b, 1, 16, 0.1, 1, torch.zeros(4, 16, dtype=torch.bfloat16))
    w = torch.zeros(16, 128, 256, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="expected"):
        kvx.latent_extend_attention(None, b, 1, w, w, 0.1, 1)
    with pytest.raises(ValueError, match="inv_freq"):
        kvx.store_latent_rope(None, b, 1, inv_freq=np.zeros(31))
    with pytest.raises(ValueError, match="q_dim"):
        kvx.store_latent_rope(None, b, 1, q=1, q_out=1, num_q_heads=2)


def test_absent_pool_is_reported():
    b = kvx.Batch([16], [4], [0, 2], 0x1000)
    for call in (lambda: kvx.store_latent(None, b, 1), lambda: kvx.load_latent(None, b, 1),
                 lambda: kvx.latent_attention(None, b, 1, 16, 0.1, 1),
                 lambda: kvx.latent_pool_set_split_keys(None, 64), lambda: kvx.latent_pool_layout(None)):
        with pytest.raises(kvx.KvxError) as e:
            call()
        assert e.value.status == kvx.KVX_EINVAL and "NULL" in kvx.kvx_last_error()


def test_header_is_c(tmp_path):
    if shutil.which("gcc") is None:
        pytest.skip("gcc not installed")
    src = tmp_path / "user.c"
    src.write_text('#include "kvx_latent.h"\n'
                   "int use(kvx_latent_pool *p, const kvx_batch *b, const kvx_latent_proj *w, void *x) {\n"
                   "    kvx_latent_layout l;\n"
                   "    return latent_pool_layout(p, &l) + store_latent(p, b, x, 576, 0) +\n"
                   "           latent_extend_attention(p, b, w, x, 0.1f, x, 0, KVX_LATENT_AUTO, 0);\n"
                   "}\n")
    r = subprocess.run(["gcc", "-std=c99", "-pedantic", "-Wall", "-Wextra", "-Werror", "-fsyntax-only",
                        "-I" + os.path.join(ROOT, "include"), str(src)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr


def test_binding_refuses_types_of_the_same_width(monkeypatch):
    """16-bit floats that are not bf16, and 32-bit integers for lse, are not taken for their bits."""
    monkeypatch.setattr(kvx, "_latent_row", lambda pool: (512, 64))
    b = kvx.Batch([16], [4], [0, 2], 0x1000)
    half, ints = torch.zeros(4, 576, dtype=torch.float16), torch.zeros(4, 16, dtype=torch.int32)
    w, q = torch.zeros(16, 128, 512, dtype=torch.bfloat16), torch.zeros(4, 16, 192, dtype=torch.float16)
    for call in (lambda: kvx.store_latent(None, b, half), lambda: kvx.load_latent(None, b, half),
                 lambda: kvx.store_latent_rope(None, b, half), lambda: kvx.store_latent_rope(None, b, 1, norm=half),
                 lambda: kvx.store_latent_rope(None, b, 1, q=q, q_out=q, num_q_heads=16),
                 lambda: kvx.latent_attention(None, b, half, 1, 0.1, 1), lambda: kvx.latent_attention(None, b, 1, 1, 0.1, half),
                 lambda: kvx.latent_extend_attention(None, b, q, w, w, 0.1, 1),
                 lambda: kvx.latent_extend_attention(None, b, 1, w.half(), w, 0.1, 1),
                 lambda: kvx.latent_extend_attention(None, b, 1, w, w.half(), 0.1, 1)):
        with pytest.raises(ValueError, match="float16 elements; expected bf16"):
            call()
    with pytest.raises(ValueError, match="int32 elements; expected float32"):
        kvx.latent_attention(None, b, 1, 16, 0.1, 1, ints)
    # the bits of bf16 as integers pass (and are then not on the device)
    with pytest.raises(ValueError, match="device"):
        kvx.store_latent(None, b, half.view(torch.int16))
