"""The loop over blocks of the 8-bit attention as it was built: a block waits for what it needs of the cache, not for everything under way.  The loads of the next block are on their way
while this one is multiplied, so a wait for all loads inside that loop would undo the overlap; the compiler puts one there as soon as registers that a load fills are moved on the way
round."""
import os
import re
import shutil
import subprocess

import pytest

from test_kernel_registers import BUILD, LLVM


def code_of(source, tmp_path):
    """{mangled name: [(address, instruction)]} of the object built from `source`.hip."""
    obj = os.path.join(BUILD, source + ".o")
    if not os.path.exists(obj) or not os.path.exists(os.path.join(LLVM, "llvm-objdump")):
        pytest.skip("needs the built objects and the ROCm LLVM tools")
    bundle, code = str(tmp_path / "bundle"), str(tmp_path / "code")
    copy = shutil.copy(obj, str(tmp_path / "obj.o"))
    subprocess.run([LLVM + "/llvm-objcopy", "--dump-section", ".hip_fatbin=" + bundle, copy], check=True)
    subprocess.run([LLVM + "/clang-offload-bundler", "--unbundle", "--type=o", "--targets=hipv4-amdgcn-amd-amdhsa--gfx950",
                    "--input=" + bundle, "--output=" + code], check=True)
    text = subprocess.run([LLVM + "/llvm-objdump", "-d", "--no-show-raw-insn", code], check=True, capture_output=True, text=True).stdout
    found, name = {}, None
    for line in text.split("\n"):
        if m := re.match(r"[0-9a-f]+ <(\S+)>:", line):
            name = m.group(1)
            found[name] = []
        elif name and (m := re.match(r"\s+(\S.*?)\s*// ([0-9A-F]+):", line)):
            found[name].append((int(m.group(2), 16), m.group(1)))
    return found


def block_loops(code, records):
    """The innermost ranges that end in a branch back to their beginning, multiply matrices and request K and V of a block, `records` loads of 16 bytes; without a barrier."""
    at = {address: i for i, (address, _) in enumerate(code)}
    ranges = []
    for i, (address, what) in enumerate(code):
        if m := re.match(r"s_c?branch\S*\s+(\d+)", what):
            off = int(m.group(1))
            begin = at.get(address + 4 + 4 * (off - 65536 if off >= 32768 else off))
            if begin is None or begin > i:
                continue
            body = [w for _, w in code[begin:i + 1]]
            if sum("v_mfma" in w for w in body) >= 8 and sum("buffer_load_dwordx4" in w for w in body) >= records and not any("s_barrier" in w for w in body):
                ranges.append((begin, i))
    inner = [r for r in ranges if not any(s != r and r[0] <= s[0] and s[1] <= r[1] for s in ranges)]
    return [[w for _, w in code[a:b + 1]] for a, b in inner]


@pytest.mark.parametrize("source,kernel,loops", [("kv8_attention", "kv8_attn_kernel", 1), ("kv8_apart", "kv8_attn_kernel", 1), ("kv8_shared", "kv8_shared_kernel", 2)])
def test_a_block_waits_for_its_own_loads_alone(source, kernel, loops, tmp_path):
    """Of kv8_shared_kernel the workgroups behind a prefix and, where a prefix's waves are on segments of their own, those on it."""
    found = {k: v for k, v in code_of(source, tmp_path).items() if kernel in k}
    assert found
    for name, code in found.items():
        channels, *_ = (int(x) for x in re.findall(r"Li(\d+)E", name))
        records = 2 * channels // 32
        bodies = block_loops(code, records)
        assert len(bodies) == (1 if "Lb0E" in name else loops), (name, len(bodies))
        for body in bodies:
            waits = [int(m.group(1)) for w in body for m in [re.search(r"vmcnt\((\d+)\)", w)] if m]
            assert waits and min(waits) >= channels // 32, (name, waits)     # V's loads are under way while K is waited for, and the other way round
