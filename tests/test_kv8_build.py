"""The 8-bit cache's objects as they were built: registers that leave room for the workgroups their launches assume, and all their host code under
AddressSanitizer and UndefinedBehaviorSanitizer (host code only; device code is compiled as usual and never runs here)."""
import os
import re
import shutil
import subprocess
from concurrent.futures import ThreadPoolExecutor

import pytest

from test_host_sanitizers import CSRC, HIP, OUT, ROOT, SAN
from test_kernel_registers import kernels


def test_registers_of_the_attention_kernels(tmp_path):
    """Two waves a SIMD, whether of one workgroup of eight or of two of four: at most 256 registers, nothing in scratch memory."""
    found = {k: v for k, v in kernels("kv8_attention", tmp_path).items() if "kv8_attn_kernel" in k}
    assert len(found) == 2 * 2 * 2 * 3 + 2 * 2 * 2      # channels, formats, parts, tiles; of 128 channels two and three tiles with eight waves
    for k, (registers, spilled, scratch) in found.items():
        assert registers <= 256 and spilled == 0 and scratch == 0, (k, registers, spilled, scratch)


def test_registers_of_the_store_kernels(tmp_path):
    """Rows of a prompt are many small workgroups: five waves a SIMD for an append of several heads a workgroup, six for the others."""
    found = kernels("kv8_store", tmp_path)
    assert len(found) == 8 + 4 + 4 + 1 + 1              # append by channels, format, one head or several; read, commit; the advance of lens, the rotation
    for k, (registers, spilled, scratch) in found.items():
        assert registers <= (96 if "append_kernel" in k and "Lb1" in k else 80) and spilled == 0 and scratch == 0, (k, registers, spilled, scratch)


def _compile(job):
    cmd, obj = job
    subprocess.run(cmd + ["-o", obj], check=True, stdout=subprocess.PIPE, stderr=subprocess.STDOUT)
    return obj


@pytest.mark.timeout(900)
def test_host_code_is_clean_under_asan_and_ubsan():
    if shutil.which("hipcc") is None:
        pytest.skip("hipcc not on PATH")
    out = os.path.join(OUT, "kv8")
    os.makedirs(out, exist_ok=True)
    jobs = [(HIP + ["-c", os.path.join(CSRC, src)], os.path.join(out, src + ".o")) for src in ("kv8_attention.hip", "kv8_store.hip", "kv8_api.hip")]
    jobs.append((HIP + ["-c", os.path.join(ROOT, "tests", "sanitize", "kv8_san.hip")], os.path.join(out, "kv8_san.o")))
    with ThreadPoolExecutor(max_workers=4) as ex:
        objs = list(ex.map(_compile, jobs))
    exe = os.path.join(out, "kv8_san")
    subprocess.run(["hipcc", "--offload-arch=gfx950", "-fno-gpu-sanitize", *SAN, *objs, "-lm", "-o", exe], check=True)
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1")
    run = subprocess.run([exe], env=env, stdout=subprocess.PIPE, stderr=subprocess.PIPE, text=True, timeout=600)
    print(run.stdout, run.stderr[-4000:])
    assert run.returncode == 0, run.stderr[-4000:]
    assert "ERROR: AddressSanitizer" not in run.stderr and "runtime error:" not in run.stderr
    assert re.search(r"host self-test passed", run.stdout)
