"""The loads into LDS that are written as inline assembly, in the code that the compiler makes of them: a scalar
operand that a vector instruction writes (v_readlane brings spilled scalars back) may be read by a memory
instruction five wait states later at the earliest, and the compiler does not look into inline assembly."""
import os
import re
import subprocess

import pytest

from paper_2603_23198_amd import build

WAIT = 5


def scalars(operands):
    found = {int(m[1]) for m in re.finditer(r"\bs(\d+)\b", operands)}
    for m in re.finditer(r"\bs\[(\d+):(\d+)\]", operands):
        found |= set(range(int(m[1]), int(m[2]) + 1))
    return found | ({"m0"} if "m0" in operands else set())


def too_early(assembly):
    """(loads, those that read a scalar too early)"""
    loads, bad, before = 0, [], []
    for line in assembly.splitlines():
        code = line.split(";")[0].strip()
        if not code or code.endswith(":") or code.startswith("."):
            continue
        op, _, rest = code.partition(" ")
        if op.startswith("buffer_load") and rest.endswith("lds"):
            loads += 1
            states = 0
            for was, operands in reversed(before):
                if states >= WAIT:
                    break
                if was.startswith("v_") and scalars(operands.split(",")[0]) & (scalars(rest) | {"m0"}):
                    bad.append((was, operands, code))
                states += int(operands) + 1 if was == "s_nop" else 1
        before = before[-2 * WAIT:] + [(op, rest)]
    return loads, bad


def test_the_check_itself():
    load = "buffer_load_dwordx4 v0, s[64:67], s16 offen lds"
    assert too_early("v_readlane_b32 s16, v255, 9\ns_mov_b32 m0, s1\n" + load)[1]
    assert too_early("v_readfirstlane_b32 s65, v3\n" + load)[1]
    assert too_early("v_readlane_b32 s16, v255, 9\ns_nop 4\n" + load) == (1, [])
    assert too_early("v_readlane_b32 s17, v255, 9\n" + load) == (1, [])


@pytest.mark.parametrize("source", ["product8.hip"])
def test_scalars_of_loads_into_lds_are_settled(source, tmp_path):
    out = str(tmp_path / "code.s")
    cmd = [build.hipcc(), *build.FLAGS, "-x", "hip", "-S", "--cuda-device-only", os.path.join(build.CSRC, source), "-o", out]
    subprocess.run(cmd, check=True, capture_output=True)
    with open(out) as f:
        loads, bad = too_early(f.read())
    assert loads > 0 and not bad, bad[:3]
