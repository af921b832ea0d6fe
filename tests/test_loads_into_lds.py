"""Loads from memory into LDS that are written in inline assembly.  The assembler adds no wait states there, so the code itself has to:
one between a write of m0 and a load into LDS (m0 holds the place in LDS), five between a vector instruction that writes a scalar
register and a load that takes its address from it.  What the compiler has made of the sources is looked through."""
import os
import re
import subprocess

import pytest

from paper_2505_18573_amd import build

LOAD = re.compile(r"(global|buffer|scratch)_load_lds_|_load_\w+ .*\blds$")
SOURCES = [s for s in build.SOURCES if "load_lds" in open(os.path.join(build.CSRC, s)).read()]


def scalars(operand):
    """The numbers of the scalar registers that an operand names."""
    one = re.fullmatch(r"s(\d+)", operand)
    many = re.fullmatch(r"s\[(\d+):(\d+)\]", operand)
    return {int(one[1])} if one else set(range(int(many[1]), int(many[2]) + 1)) if many else set()


def too_near(assembly):
    """Lines of loads into LDS that lie too near behind what they depend on."""
    found = []
    m0_at = -100                                                  # in wait states
    written_at = {}
    now = 0
    for number, line in enumerate(assembly.splitlines(), 1):
        text = line.split(";")[0].split("//")[0].strip()
        if not text or text.startswith(".") or text.endswith(":"):
            continue
        name, _, rest = text.partition(" ")
        operands = [x.strip() for x in rest.split(",")]
        if LOAD.match(text):
            used = set().union(*(scalars(x.split()[0]) for x in operands if x))
            if now - m0_at - 1 < 1 or any(now - written_at.get(r, -100) - 1 < 5 for r in used):
                found.append((number, text))
        if name.startswith("s_") and operands[0] == "m0":
            m0_at = now
        for r in scalars(operands[0]):
            if name.startswith("v_"):
                written_at[r] = now
            elif name.startswith("s_") and not name.startswith("s_cmp"):
                written_at.pop(r, None)
        now += 1 + (int(operands[0], 0) if name == "s_nop" else 0)
    return found


def test_what_is_too_near():
    load = "\tglobal_load_lds_dwordx4 v1, s[4:5]\n"
    assert too_near("\ts_mov_b32 m0, s3\n" + load) == [(2, load.strip())]
    assert too_near("\ts_mov_b32 m0, s3\n\ts_nop 0\n" + load) == [] and too_near("\ts_mov_b32 m0, s3 ; x\n.LBB:\n; y\n\ts_add_u32 s9, s9, 1\n" + load) == []
    near = "\tv_readfirstlane_b32 s5, v0\n\ts_mov_b32 m0, s3\n\ts_nop {}\n" + load
    assert too_near(near.format(2)) == [(4, load.strip())] and too_near(near.format(3)) == []
    assert too_near("\tv_readlane_b32 s5, v0, 3\n\ts_mov_b32 s5, 0\n\ts_mov_b32 m0, s3\n\ts_nop 0\n" + load) == []
    assert too_near("\tv_readfirstlane_b32 s6, v0\n\ts_mov_b32 m0, s3\n\ts_nop 0\n" + load) == []


@pytest.mark.parametrize("source", SOURCES)
def test_loads_wait_for_what_they_depend_on(source, tmp_path):
    out = os.path.join(tmp_path, "device.s")
    flags = [f for f in build.FLAGS if f != "-shared"]
    subprocess.run([build.HIPCC, *flags, "-S", "--offload-device-only", "-o", out, os.path.join(build.CSRC, source)], check=True,
                   stderr=subprocess.DEVNULL)
    assembly = open(out).read()
    assert len(re.findall(r"load_lds_", assembly)) > 0
    assert too_near(assembly) == []
