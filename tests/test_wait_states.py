"""Wait states that gfx9 leaves to the program, in the built kernels' own code.  The compiler keeps them for instructions it chooses,
not for those of inline assembly: loads into LDS take their address from M0, which has to be written a wait state before them,
and a base in scalar registers that a vector instruction wrote has to be five old."""
import os
import re
import shutil
import subprocess

import pytest

OBJDUMP = shutil.which("llvm-objdump", path="/opt/rocm/llvm/bin" + os.pathsep + os.environ.get("PATH", ""))


def scalars(operand):
    m = re.fullmatch(r"s\[(\d+):(\d+)\]", operand)
    if m:
        return set(range(int(m[1]), int(m[2]) + 1))
    m = re.fullmatch(r"s(\d+)", operand)
    return {int(m[1])} if m else set()


def violations(listing):
    """(number of loads into LDS, those too close behind what they read)."""
    loads, bad, behind, kernel = 0, [], [], ""
    for line in listing.splitlines():
        m = re.match(r"[0-9a-f]+ <(.*)>:", line)
        if m:
            kernel, behind = m[1], []
            continue
        m = re.match(r"\s+([a-z]\S+)\s*([^/]*)", line)
        if not m:
            continue
        op, operands = m[1], [t.split()[0] for t in m[2].split(",") if t.strip()]
        if re.match(r"(global|buffer|scratch)_load_lds_", op):
            loads += 1
            used = set().union(*(scalars(t) for t in operands))
            age = 0
            for earlier, its in reversed(behind):
                if its and its[0] == "m0" and age < 1:
                    bad.append(f"{kernel}: {op} {age} wait states behind {earlier} {its}")
                if earlier.startswith("v_") and its and scalars(its[0]) & used and age < 5:
                    bad.append(f"{kernel}: {op} {age} wait states behind {earlier} {its}")
                age += 1 + (int(its[0]) if earlier == "s_nop" else 0)
                if age >= 5:
                    break
        behind = (behind + [(op, operands)])[-8:]
    return loads, bad


def test_the_check_finds_what_it_looks_for():
    head = "0000 <k>:\n"
    move, load = "\ts_mov_b32 m0, s2      // 0\n", "\tglobal_load_lds_dwordx4 v2, s[4:5]  // 0\n"
    assert violations(head + move + load)[1] and not violations(head + move + "\ts_nop 0  // 0\n" + load)[1]
    base = "\tv_readfirstlane_b32 s5, v1  // 0\n"
    assert violations(head + base + move + "\ts_nop 0  // 0\n" + load)[1]
    assert not violations(head + base + move + "\ts_nop 3  // 0\n" + load)[1]


@pytest.mark.skipif(OBJDUMP is None, reason="no disassembler")
def test_loads_into_lds_keep_their_distance(tmp_path):
    from paper_1305_1422_amd import build
    lib = shutil.copy(build.LIB, tmp_path / "lib.so")
    subprocess.run([OBJDUMP, "--offloading", str(lib)], cwd=tmp_path, check=True, stdout=subprocess.DEVNULL)
    code = sorted(p for p in tmp_path.iterdir() if "amdgcn" in p.name)
    assert code
    loads, bad = 0, []
    for p in code:
        listing = subprocess.run([OBJDUMP, "-d", "--mcpu=gfx950", str(p)], check=True, capture_output=True, text=True).stdout
        some, wrong = violations(listing)
        loads, bad = loads + some, bad + wrong
    assert loads > 0
    assert not bad, f"{len(bad)} of {loads}: {bad[:5]}"
