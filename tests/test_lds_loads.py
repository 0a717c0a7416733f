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


def too_early_on_any_path(assembly):
    """(loads, those that read a scalar too early) along branches too: a write at a loop's end reaches a load at its
    beginning."""
    code, at, jumps = [], {}, {}
    for line in assembly.splitlines():
        text = line.split(";")[0].strip()
        if text.endswith(":"):
            at[text[:-1]] = len(code)
        elif text and not text.startswith("."):
            op, _, rest = text.partition(" ")
            code.append((op, rest))
    for i, (op, rest) in enumerate(code):
        if op.startswith(("s_branch", "s_cbranch")) and rest in at:
            jumps.setdefault(at[rest], []).append(i)

    def before(i):
        falls = i > 0 and code[i - 1][0] not in ("s_branch", "s_endpgm", "s_setpc_b64")
        return ([i - 1] if falls else []) + jumps.get(i, [])

    loads, bad = 0, []
    for i, (op, rest) in enumerate(code):
        if not (op.startswith("buffer_load") and rest.endswith("lds")):
            continue
        loads += 1
        reads, todo, seen = scalars(rest) | {"m0"}, [(j, 0) for j in before(i)], {}
        while todo:
            j, states = todo.pop()
            if states >= WAIT or seen.get(j, WAIT) <= states:
                continue
            seen[j] = states
            was, operands = code[j]
            if was.startswith("v_") and scalars(operands.split(",")[0]) & reads:
                bad.append((was, operands, op, rest))
            todo += [(k, states + (int(operands, 0) + 1 if was == "s_nop" else 1)) for k in before(j)]
    return loads, bad


def test_the_check_along_branches_itself():
    load = "buffer_load_dwordx4 v0, s[64:67], s16 offen lds"
    loop = "top:\n" + load + "\n{}v_readlane_b32 s16, v255, 9\n{}s_cbranch_scc1 top\n"
    assert too_early(loop.format("", ""))[1] == [] and too_early_on_any_path(loop.format("", ""))[1]
    assert too_early_on_any_path(loop.format("", "s_nop 3\n")) == (1, [])
    assert too_early_on_any_path(loop.format("", "s_nop 2\n"))[1]
    assert too_early_on_any_path("v_readlane_b32 s16, v255, 9\ns_branch away\n" + load + "\naway:\ns_endpgm") == (1, [])
    assert too_early_on_any_path("v_readlane_b32 s16, v255, 9\n" + load)[1]


@pytest.mark.parametrize("source", ["product8.hip", "gemm.hip"])
def test_scalars_are_settled_on_every_path(source, tmp_path):
    """gemm.hip's loads have no wait of their own: what the compiler makes of them today leaves the states, and a
    change that spills their scalars shows here."""
    out = str(tmp_path / "code.s")
    cmd = [build.hipcc(), *build.FLAGS, "-x", "hip", "-S", "--cuda-device-only", os.path.join(build.CSRC, source), "-o", out]
    subprocess.run(cmd, check=True, capture_output=True)
    with open(out) as f:
        text = f.read()
    loads, bad = too_early_on_any_path(text)
    assert loads > 0 and not bad, bad[:3]
    assert too_early(text) == (loads, [])


def test_no_other_source_has_such_loads():
    have = set()
    for name in os.listdir(build.CSRC):
        if name.endswith((".hip", ".cpp")):
            with open(os.path.join(build.CSRC, name)) as f:
                if re.search(r"\bload_lds\w*\(", f.read()):
                    have.add(name)
    assert have == {"gemm.hip", "product8.hip"}
