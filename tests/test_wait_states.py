"""Wait states that the hardware leaves to the program, in the library's own machine code.

The compiler keeps them between the instructions that it schedules itself, but not towards the ones written in
inline assembly.  Two of them matter to the loads from memory to LDS (CDNA3 ISA, "required user-inserted wait
states", which the compiler also keeps for gfx950): one between a write of M0 and a load to LDS, and five
between a vector instruction that writes a scalar register and a memory instruction that reads it."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2602_06161_amd import build, cover

OBJDUMP = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(build.HIPCC))), "llvm", "bin", "llvm-objdump")

pytestmark = pytest.mark.skipif(not os.path.exists(cover.LIB) or not os.path.exists(OBJDUMP),
                                reason="libcover.so or llvm-objdump is not there")


def _scalars(operand):
    m = re.match(r"s\[(\d+):(\d+)\]$", operand)
    if m:
        return set(range(int(m[1]), int(m[2]) + 1))
    m = re.match(r"s(\d+)$", operand)
    return {int(m[1])} if m else set()


def violations(listing):
    """(rule, kernel, instruction) of every place in a disassembly with too few wait states, and the loads to LDS seen."""
    bad, loads, kernel, past = [], 0, None, []  # past: (mnemonic, what it writes, wait states it stands for)
    for line in listing.splitlines():
        name = re.match(r"^[0-9a-f]+ <(\S+)>:", line)
        if name:
            if not name[1].startswith("L"):
                kernel, past = name[1], []
            continue
        text = line.split("//")[0].strip()
        if not line.startswith(("\t", " ")) or not text:
            continue
        op, _, rest = text.partition(" ")
        args = [a.strip() for a in rest.split(",")]
        if op.startswith(("global_", "buffer_", "scratch_", "flat_")):
            reads = set().union(*(_scalars(a.split()[0]) for a in args if a))
            to_lds = "_lds_" in op or " lds" in rest
            loads += to_lds
            states = 0
            for mnemonic, writes, worth in reversed(past):
                if states >= 5:
                    break
                if to_lds and states < 1 and "m0" in writes:
                    bad.append(("m0", kernel, text))
                if mnemonic.startswith("v_") and writes & reads:
                    bad.append(("scalar of a vector instruction", kernel, text))
                states += worth
        first = args[0].split()[0] if args and args[0] else ""
        writes = {"m0"} if first == "m0" else (_scalars(first) if op.startswith(("v_", "s_")) else set())
        past = (past + [(op, writes, int(first, 0) + 1 if op == "s_nop" else 1)])[-6:]
        if op in ("s_branch", "s_endpgm", "s_setpc_b64"):
            past = []
    return bad, loads


def test_the_rules_themselves():
    head = "0000000000001000 <k>:\n"
    m0, load = "\ts_mov_b32 m0, s4 // 1\n", "\tglobal_load_lds_dwordx4 v1, s[2:3] // 2\n"
    assert violations(head + m0 + load)[0] and violations(head + m0 + "\ts_nop 0 // 3\n" + load) == ([], 1)
    assert violations(head + m0 + "\tv_mov_b32_e32 v0, v1 // 3\n" + load) == ([], 1)
    first = "\tv_readfirstlane_b32 s3, v7 // 4\n"
    for nops in range(6):
        found = violations(head + first + "\ts_nop 0 // 5\n" * nops + "\tglobal_load_dword v1, v0, s[2:3] // 6\n")[0]
        assert bool(found) == (nops < 5)
    assert not violations(head + first + "\ts_nop 4 // 5\n\tglobal_load_dword v1, v0, s[2:3] // 6\n")[0]
    assert not violations(head + first + "\tglobal_load_dword v1, v0, s[4:5] // 6\n")[0]


def test_the_library_keeps_them(tmp_path):
    shutil.copy(cover.LIB, tmp_path / "lib.so")
    subprocess.run([OBJDUMP, "--offloading", "lib.so"], cwd=tmp_path, check=True, capture_output=True)
    objects = sorted(p for p in tmp_path.iterdir() if p.name.endswith("gfx950"))
    assert objects
    found, loads = [], 0
    for obj in objects:
        text = subprocess.run([OBJDUMP, "-d", obj.name], cwd=tmp_path, check=True, capture_output=True, text=True).stdout
        bad, n = violations(text)
        found += bad
        loads += n
    assert loads > 100  # (else the listing was not understood)
    assert not found, f"{len(found)} places, the first: {found[:5]}"
