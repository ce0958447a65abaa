"""The built kernels keep the wait states that gfx950 does not enforce by itself around memory instructions
written in inline assembly, which the compiler does not look into (no GPU).

A scalar write of m0 needs one wait state before a load into LDS that takes its address from m0, and a vector
instruction's write of a scalar register (a lane read, a comparison) five before a memory instruction that reads it.
"""
import glob
import os
import re
import shutil
import subprocess

import pytest

from paper_2606_05875_amd import qcf

OBJDUMP = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "llvm", "bin", "llvm-objdump")
MEMORY = re.compile(r"(global|buffer|flat|scratch)_")


def scalars(operand):
    """Numbers of the scalar registers that an operand names."""
    m = re.fullmatch(r"s\[(\d+):(\d+)\]|s(\d+)", operand)
    if m:
        return set(range(int(m[1]), int(m[2]) + 1)) if m[1] else {int(m[3])}
    return {operand} if operand in ("m0", "vcc") else set()


def short_waits(lines):
    """(memory instructions into LDS, [(function, instruction, what it follows too closely)])."""
    bad, n, fn, before = [], 0, "", []
    for line in lines:
        m = re.match(r"[0-9a-f]+ <(.*)>:", line)
        if m:
            fn, before = m[1], []
            continue
        m = re.match(r"\s+([a-z]\w+)\s*([^/]*)", line)
        if not m:
            continue
        op, args = m[1], [a for a in re.split(r"[,\s]+", m[2]) if a]
        if MEMORY.match(op):
            read = set().union(*map(scalars, args))
            lds = "_lds_" in op or "lds" in args
            n += lds
            states = 0
            for prev, regs in reversed(before):
                if lds and states < 1 and prev.startswith("s_") and regs[:1] == ["m0"]:
                    bad.append((fn, line.strip(), prev))
                if prev.startswith("v_") and set().union(set(), *map(scalars, regs[:2 if "_co_" in prev else 1])) & read:
                    bad.append((fn, line.strip(), prev))
                states += int(regs[0], 0) + 1 if prev == "s_nop" else 1
                if states >= 5:
                    break
        before = before[-7:] + [(op, args)]
    return n, bad


def test_the_scan_finds_short_waits():
    text = ["0000 <f>:", "\ts_mov_b32 m0, s4", "\tglobal_load_lds_dwordx4 v1, s[2:3] // 0", "\ts_mov_b32 m0, s4", "\ts_nop 0",
            "\tbuffer_load_dwordx4 v1, s[8:11], 0 offen lds", "\tv_readlane_b32 s9, v3, 1", "\ts_nop 2",
            "\tglobal_load_dword v1, v0, s[8:9]", "\tv_readlane_b32 s9, v3, 1", "\ts_nop 4", "\tglobal_load_dword v1, v0, s[8:9]"]
    n, bad = short_waits(text)
    assert n == 2 and [b[2] for b in bad] == ["s_mov_b32", "v_readlane_b32"]


@pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="needs llvm-objdump")
def test_wait_states_of_the_built_kernels(tmp_path):
    if not os.path.exists(qcf.lib_path()):
        from paper_2606_05875_amd.build import build
        build(verbose=False)
    shutil.copy(qcf.lib_path(), tmp_path / "lib.so")
    subprocess.run([OBJDUMP, "--offloading", "lib.so"], cwd=tmp_path, check=True, capture_output=True)
    into_lds, bad = 0, []
    for obj in sorted(glob.glob(str(tmp_path / "*gfx950"))):
        r = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", obj], check=True, capture_output=True, text=True)
        n, found = short_waits(r.stdout.splitlines())
        into_lds += n
        bad += found
    assert into_lds > 100  # (the scan reads what the assembly is printed as)
    assert not bad, (len(bad), bad[:5])
