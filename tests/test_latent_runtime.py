"""Latent attention's use of the runtime, on the CPU: streams, devices and failing allocations
over a stand-in for the HIP runtime (tests/sanitize/latent_runtime.cpp, built with
AddressSanitizer and UndefinedBehaviorSanitizer), and the stream that the binding chooses."""

import os
import shutil
import subprocess
from types import SimpleNamespace

import pytest
import torch

from paper_2609_32278_amd import kvx

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SAN = ["-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-fno-omit-frame-pointer"]


@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    if shutil.which("g++") is None or not os.path.exists("/opt/rocm/include/hip/hip_runtime.h"):
        pytest.skip("g++ or the HIP headers not installed")
    exe = str(tmp_path_factory.mktemp("latent") / "latent_runtime")
    cmd = ["g++", "-std=c++17", *SAN, "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-I" + os.path.join(ROOT, "include"),
           "-I" + os.path.join(ROOT, "paper_2609_32278_amd", "csrc"),
           os.path.join(ROOT, "tests", "sanitize", "latent_runtime.cpp"), "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        if "asan" in r.stderr.lower() or "ubsan" in r.stderr.lower():
            pytest.skip("sanitizer runtime not available: " + r.stderr[-300:])
        raise AssertionError(r.stderr[-3000:])
    return exe


def run_check(driver, check, tmp_path):
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1")
    run = subprocess.run([driver, check], capture_output=True, text=True, env=env, timeout=300, cwd=tmp_path)
    assert run.returncode == 0, run.stdout[-2000:] + run.stderr[-4000:]
    assert check + " passed" in run.stdout


def test_streams_and_devices(driver, tmp_path):
    run_check(driver, "streams", tmp_path)


def test_uploads_that_find_no_memory(driver, tmp_path):
    run_check(driver, "staging", tmp_path)


def test_more_tokens_than_one_call_expands(driver, tmp_path):
    run_check(driver, "tokens", tmp_path)


def test_automatic_form_is_the_faster_one(driver, tmp_path):
    run_check(driver, "choices", tmp_path)


def test_outputs_over_inputs_are_refused(driver, tmp_path):
    run_check(driver, "overlaps", tmp_path)


class OnSecond:
    """What the binding asks of a tensor, of one on the second device."""

    dtype, is_cuda, device = torch.bfloat16, True, torch.device("cuda", 1)

    def __init__(self, *shape):
        self.shape = shape

    def dim(self):
        return len(self.shape)

    def stride(self, i):
        return 1 if i == len(self.shape) - 1 else self.shape[-1]

    def numel(self):
        return torch.Size(self.shape).numel()

    def element_size(self):
        return 2

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 0x10000


def test_binding_takes_the_stream_of_the_tensors_device(monkeypatch):
    """Where no stream is given, it is the current one of the device that the tensors are on, which
    need not be the current device."""
    streams = {None: 0x100, torch.device("cuda", 1): 0x200}
    got = []
    names = ("store_latent", "store_latent_rope", "load_latent", "latent_attention", "latent_extend_attention")
    fake = SimpleNamespace(**{n: lambda *a: got.append(a[-1].value) or 0 for n in names})
    monkeypatch.setattr(kvx, "lib", lambda: fake)
    monkeypatch.setattr(kvx, "_latent_row", lambda pool: (256, 64))
    monkeypatch.setattr(torch.cuda, "is_initialized", lambda: True)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda d=None: SimpleNamespace(cuda_stream=streams[d]))
    b = kvx.Batch([16], [4], [0, 2], 0x1000)
    rows, q, o, w = OnSecond(4, 320), OnSecond(4, 2, 320), OnSecond(4, 2, 256), OnSecond(2, 64, 256)
    qs, os_ = OnSecond(4, 2, 128), OnSecond(4, 2, 64)
    kvx.store_latent(None, b, rows)
    kvx.store_latent_rope(None, b, rows)
    kvx.store_latent_rope(None, b, 0x1000, q=qs, num_q_heads=2, q_out=qs)
    kvx.load_latent(None, b, rows)
    kvx.latent_attention(None, b, q, 2, 0.1, o)
    kvx.latent_attention(None, b, 0x1000, 2, 0.1, o)
    kvx.latent_extend_attention(None, b, qs, w, w, 0.1, os_)
    assert got == [0x200] * 7
    got.clear()
    kvx.store_latent(None, b, 0x1000)  # addresses only: the current device's stream, as before
    kvx.latent_attention(None, b, 0x1000, 2, 0.1, 0x2000, stream=0x300)
    assert got == [0x100, 0x300]
