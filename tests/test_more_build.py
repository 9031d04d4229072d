"""Shared prefixes, pages and log-probabilities as they were built: registers that leave room for the workgroups their launches assume, and all their host code under
AddressSanitizer and UndefinedBehaviorSanitizer (host code only; device code is compiled as usual and never runs here)."""
import os
import re
import shutil
import subprocess
from concurrent.futures import ThreadPoolExecutor

import pytest

from test_host_sanitizers import CSRC, HIP, OUT, ROOT, SAN
from test_kernel_registers import kernels


def test_registers_of_the_shared_attention(tmp_path):
    """Two workgroups of four waves a compute unit: at most 256 registers; nothing in scratch memory but three words of the form of two row tiles a wave with a step's rows in two or
    three tiles."""
    found = {k: v for k, v in kernels("kv8_shared", tmp_path).items() if "kv8_shared_kernel" in k}
    assert len(found) == 2 * 2 * (4 + 3) * 3      # channels, formats; kinds of a prefix's workgroups for bf16 and float32; row tiles of the rest
    for k, (registers, spilled, scratch) in found.items():
        hd, _, parts, tiles, few, rest = (int(x) for x in re.search(r"ILi(\d+)ELi(\d)ELi(\d)ELi(\d)ELb(\d)ELi(\d)E", k).groups())
        allowed = 16 if (hd, parts, tiles, few) == (128, 1, 2, 0) and rest > 1 else 0
        assert registers <= 256 and scratch <= allowed, (k, registers, spilled, scratch)


def test_registers_of_sequences_by_themselves(tmp_path):
    """As those of a batch that shares nothing: two waves a SIMD, nothing in scratch memory."""
    found = {k: v for k, v in kernels("kv8_apart", tmp_path).items() if "kv8_attn_kernel" in k}
    assert len(found) == 2 * 2 * 2 * 3 + 2 * 2 * 2
    for k, (registers, spilled, scratch) in found.items():
        assert registers <= 256 and spilled == 0 and scratch == 0, (k, registers, spilled, scratch)


def test_registers_of_log_probabilities(tmp_path):
    """Six workgroups of four waves on a compute unit: 1536 rows at once."""
    found = {k: v for k, v in kernels("logprobs", tmp_path).items() if "logprob_kernel" in k}
    assert len(found) == 4
    for k, (registers, spilled, scratch) in found.items():
        assert registers <= 80 and scratch <= 8, (k, registers, spilled, scratch)


def _compile(job):
    cmd, obj = job
    subprocess.run(cmd + ["-o", obj], check=True, stdout=subprocess.PIPE, stderr=subprocess.STDOUT)
    return obj


@pytest.mark.timeout(900)
def test_host_code_is_clean_under_asan_and_ubsan():
    if shutil.which("hipcc") is None:
        pytest.skip("hipcc not on PATH")
    out = os.path.join(OUT, "more")
    os.makedirs(out, exist_ok=True)
    jobs = [(HIP + ["-c", os.path.join(CSRC, src)], os.path.join(out, src + ".o"))
            for src in ("kv8_shared.hip", "kv8_apart.hip", "kv8_attention.hip", "kv8_store.hip", "kv8_api.hip", "kv8_pages.hip", "logprobs.hip")]
    jobs.append((HIP + ["-c", os.path.join(ROOT, "tests", "sanitize", "more_san.hip")], os.path.join(out, "more_san.o")))
    with ThreadPoolExecutor(max_workers=4) as ex:
        objs = list(ex.map(_compile, jobs))
    exe = os.path.join(out, "more_san")
    subprocess.run(["hipcc", "--offload-arch=gfx950", "-fno-gpu-sanitize", *SAN, *objs, "-lm", "-o", exe], check=True)
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1")
    run = subprocess.run([exe], env=env, stdout=subprocess.PIPE, stderr=subprocess.PIPE, text=True, timeout=600)
    print(run.stdout, run.stderr[-4000:])
    assert run.returncode == 0, run.stderr[-4000:]
    assert "ERROR: AddressSanitizer" not in run.stderr and "runtime error:" not in run.stderr
    assert re.search(r"host self-test passed", run.stdout)
