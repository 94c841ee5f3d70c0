"""Wait states around the loads from memory to LDS that are written as asm.

The compiler sees one opaque statement there and inserts none itself.  On
gfx9-family chips such a load must come at least one wait state after the scalar
instruction that writes m0, and any load from memory at least five after a
vector instruction (v_readlane and its like) that writes a scalar register of
its address.  The built library's kernels are read for both; s_nop N counts
N + 1, every other instruction one.
"""

import os
import re
import shutil
import subprocess

import pytest

import paper_2505_22857_amd as ng

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"   # the compiler's own: another may not know the chip
REGISTERS = re.compile(r"\bs(?:(\d+)|\[(\d+):(\d+)\])")


def scalars(text):
    """Numbers of the scalar registers named in an operand."""
    out = set()
    for one, lo, hi in REGISTERS.findall(text):
        out |= set(range(int(lo), int(hi) + 1)) if lo else {int(one)}
    return out


def violations(lines):
    """Loads to LDS of a listing that follow too soon, and how many there are."""
    loads, bad, code = 0, [], []
    for line in lines:
        text = line.split("//")[0].strip()
        if not text or text.endswith(":") or text.startswith(("Disassembly", "libngpu")):
            continue
        code.append(text)
        if not re.match(r"(global|buffer)_load_(lds_|.* lds)", text):
            continue
        loads += 1
        address, state = scalars(text), 0
        for before in reversed(code[-8:-1]):
            name, _, operands = before.partition(" ")
            to = operands.split(",")[0]
            if name == "s_nop":
                state += int(operands.strip(), 0) + 1
                continue
            if name.startswith("s_") and to.strip() == "m0" and state < 1:
                bad.append((before, text))
            if name.startswith("v_") and scalars(to) & address and state < 5:
                bad.append((before, text))
            state += 1
    return loads, bad


def test_the_rule_itself():
    load = "\tglobal_load_lds_dwordx4 v1, s[4:5]   // 000"
    far = ["\ts_nop 4"]
    assert violations(["\ts_mov_b32 m0, s9 // 0", load]) == (1, [("s_mov_b32 m0, s9", load.split("//")[0].strip())])
    assert violations(["\ts_mov_b32 m0, s9 // 0", "\ts_nop 0", load])[1] == []
    assert violations(["\tv_readfirstlane_b32 s5, v0", "\ts_mov_b32 m0, s9", "\ts_nop 2", load])[1] != []
    assert violations(["\tv_readfirstlane_b32 s5, v0", "\ts_mov_b32 m0, s9", "\ts_nop 3", load])[1] == []
    assert violations(["\tv_readlane_b32 s6, v0, 3", "\ts_mov_b32 m0, s9", "\ts_nop 0", load])[1] == []
    assert violations(["\tv_readlane_b32 s4, v0, 3", *far, load]) == (1, [])


def test_loads_to_lds_keep_their_distance(tmp_path):
    if not os.path.exists(OBJDUMP):
        pytest.skip("llvm-objdump is not available")
    ng.load_library()
    lib = shutil.copy(ng.LIB_PATH, tmp_path / "libngpu_lm.so")
    subprocess.run([OBJDUMP, "--offloading", lib], check=True, capture_output=True, cwd=tmp_path)
    objects = [p for p in tmp_path.iterdir() if p.name.endswith("gfx950")]
    assert objects
    loads, bad = 0, []
    for p in objects:
        text = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", str(p)], check=True, capture_output=True,
                              text=True).stdout
        n, b = violations(text.splitlines())
        loads, bad = loads + n, bad + b
    print(f"[case] {loads} loads to LDS", flush=True)
    assert loads > 0
    assert not bad, f"{len(bad)} of {loads}, the first: {bad[0]}"
