"""Wait states of the loads that write LDS, in the machine code that was built
here from csrc (no GPU is needed).  They are written as instructions, so the
compiler does not put apart what CDNA asks to be apart:

    1 wait state   from a scalar write of m0 to the load that takes its LDS address from it
    5 wait states  from a vector instruction's write of a scalar register to a load that reads it

An instruction is one wait state, s_nop n is n + 1."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2608_02168_amd import api

OBJDUMP = next((p for p in ("/opt/rocm/llvm/bin/llvm-objdump", shutil.which("llvm-objdump")) if p and os.path.exists(p)), None)
TARGET = "gfx950"


def scalars(operand):
    """The scalar registers that an operand names."""
    m = re.fullmatch(r"s\[(\d+):(\d+)\]", operand)
    if m:
        return set(range(int(m[1]), int(m[2]) + 1))
    m = re.fullmatch(r"s(\d+)", operand)
    return {int(m[1])} if m else set()


def too_near(before, load):
    """What lies nearer to the load than it may; before: the instructions before it, the nearest first."""
    reads = set().union(*(scalars(x) for x in load[1:]))
    waited = 0
    for op, *args in before:
        if waited >= 5:
            return None
        if waited < 1 and op.startswith("s_") and args and args[0] == "m0":
            return op, args
        # two scalar results at most: the result and the carry
        if op.startswith("v_") and reads & set().union(*(scalars(x) for x in args[:2 if op.startswith(CARRY) else 1])):
            return op, args
        waited += int(args[0], 0) + 1 if op == "s_nop" else 1
    return None


CARRY = ("v_add_co", "v_sub_co", "v_subrev_co", "v_addc_co", "v_subb_co", "v_subbrev_co", "v_div_scale", "v_mad_u64", "v_mad_i64")


def found(lines):
    """(loads, those of them that something lies too near to)"""
    before, loads, bad = [], 0, []
    for line in lines:
        text = line.split("//")[0].split(";")[0].strip()
        if not re.match(r"(s|v|ds|buffer|global|flat|scratch)_", text):
            continue
        now = re.split(r"[ ,]+", text)
        if re.match(r"(buffer|global|scratch)_load", now[0]) and "lds" in now[1:]:
            loads += 1
            near = too_near(before, now)
            if near:
                bad.append((near, text))
        before = [now] + before[:7]
    return loads, bad


def test_what_is_found():
    load = "  buffer_load_dwordx4 v2, s[8:11], 0 offen lds   // 00"
    assert found(["s_mov_b32 m0, s4", load])[1] and not found(["s_mov_b32 m0, s4", "s_nop 0", load])[1]
    assert found(["s_add_i32 m0, s4, 64", load])[1] and not found(["s_mov_b32 s3, m0", load])[1]
    vec = "v_readfirstlane_b32 s10, v3"
    assert found([vec, "s_mov_b32 m0, s4", "s_nop 2", load])[1] and not found([vec, "s_mov_b32 m0, s4", "s_nop 3", load])[1]
    assert not found(["v_readfirstlane_b32 s12, v3", "s_nop 0", load])[1]
    assert found([load, load]) == (2, [])


def test_loads_to_lds_keep_their_distance(tmp_path):
    if not os.path.exists(api.LIB_PATH):
        pytest.skip("libhg.so not built")
    if OBJDUMP is None:
        pytest.skip("llvm-objdump not available")
    lib = tmp_path / "lib.so"
    lib.write_bytes(open(api.LIB_PATH, "rb").read())
    subprocess.run([OBJDUMP, "--offloading", str(lib)], check=True, capture_output=True, cwd=tmp_path)
    objects = [p for p in tmp_path.iterdir() if p.name.endswith(TARGET)]
    assert objects
    loads = 0
    for p in objects:
        code = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", "--no-leading-addr", str(p)], check=True,
                              capture_output=True, text=True).stdout
        n, bad = found(code.splitlines())
        loads += n
        assert not bad, (len(bad), bad[:3])
    assert loads > 0
