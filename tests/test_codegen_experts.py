"""Device-code checks of the experts' products (CPU only: hipcc cross-compiles gfx950).

Their direct loads into LDS are inline assembly, inside which the compiler inserts no wait states. On this
architecture a scalar register written by a vector instruction (v_readfirstlane, v_readlane, a comparison)
needs five wait states before a vector memory instruction reads it, and m0 one between its write and a load
that uses it. The generated assembly is scanned for both."""
import os
import re
import subprocess

import pytest

from test_codegen_hazards import CSRC, HIPCC, ROOT

SGPR_TO_VMEM = 5


def sgprs(tok):
    """Scalar registers an operand names."""
    m = re.match(r"s\[(\d+):(\d+)\]$", tok)
    if m:
        return set(range(int(m.group(1)), int(m.group(2)) + 1))
    m = re.match(r"s(\d+)$", tok)
    return {int(m.group(1))} if m else set()


def scan(text):
    """(loads seen, violations) of an assembly listing. Wait states are counted as issued instructions
    (s_nop N as N + 1) along the listing; every label keeps what the instructions above it wrote."""
    loads, bad = 0, []
    recent = []          # (wait states since, registers written by a vector instruction)
    m0_age = 99
    for line in text.splitlines():
        s = line.strip().split(";")[0].strip()
        if not s or s.startswith(".") or s.endswith(":") or s.startswith("//"):
            continue
        parts = s.replace(",", " ").split()
        op, operands = parts[0], parts[1:]
        if re.match(r"(buffer|global)_load\w*", op) and ("lds" in op or "lds" in operands):
            loads += 1
            used = set().union(*[sgprs(t) for t in operands]) if operands else set()
            for age, regs in recent:
                if age < SGPR_TO_VMEM and regs & used:
                    bad.append(("scalar register", s))
            if m0_age < 1:
                bad.append(("m0", s))
        step = int(operands[0]) + 1 if op == "s_nop" else 1
        recent = [(a + step, r) for a, r in recent if a + step < SGPR_TO_VMEM]
        m0_age += step
        if op.startswith("v_") and operands:
            w = sgprs(operands[0])
            if w:
                recent.append((0, w))
        if op in ("s_mov_b32", "s_add_i32", "s_add_u32", "s_lshl_b32") and operands and operands[0] == "m0":
            m0_age = 0
    return loads, bad


def assembly(name):
    out = subprocess.run([HIPCC, "--offload-arch=gfx950", "-O3", "-std=c++17", "-Xclang", "-target-feature", "-Xclang",
                          "-packed-fp32-ops", "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-S",
                          "--offload-device-only", "-o", "-", os.path.join(CSRC, name)], capture_output=True, text=True)
    assert out.returncode == 0, out.stderr[-2000:]
    return out.stdout


def test_scan_flags_planted_violations():
    good = "v_readfirstlane_b32 s4, v1\ns_nop 4\ns_mov_b32 m0, s9\ns_nop 0\nbuffer_load_dwordx4 v1, s[4:7], s8 offen lds\n"
    assert scan(good) == (1, [])
    assert scan(good.replace("s_nop 4", "s_nop 1"))[1]
    assert scan(good.replace("s_nop 0\n", ""))[1]


@pytest.mark.parametrize("name", ["grouped.hip", "fp8.hip"])
def test_direct_loads_keep_their_wait_states(name):
    loads, bad = scan(assembly(name))
    assert loads > 100
    assert not bad, bad[:5]
