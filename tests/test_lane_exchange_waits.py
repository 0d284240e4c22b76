"""Waits before exchanges between lanes, read from the assembly of the kernels (no GPU
needed).  v_permlane16_swap and v_permlane32_swap may read a register two wait states after
a vector instruction wrote it.  The compiler sees to that for its own instructions, not for
those of asm blocks."""
import os
import re
import subprocess

import pytest

from paper_2211_10725_amd import build

WAITS = 2


def _sources():
    for name in build.SOURCES:
        with open(os.path.join(build.CSRC, name)) as f:
            if "permlane" in f.read():
                yield name


def _registers(operands):
    out = set()
    for m in re.finditer(r"\bv(\d+)\b|\bv\[(\d+):(\d+)\]", operands):
        out |= {int(m[1])} if m[1] else set(range(int(m[2]), int(m[3]) + 1))
    return out


def short_waits(lines):
    """(number of swaps, [(function, wait states, writer)] of those too close to a writer)."""
    function, before, swaps, short = None, [], 0, []
    for line in lines:
        line = line.split(";")[0].strip()
        if re.match(r"_Z\w+:", line):
            function, before = line[:-1], []
        op, _, operands = line.partition(" ")
        if not re.match(r"(v|s|ds|global|flat|buffer|scratch)_", op):
            continue
        operands = operands.strip()
        swap = op.startswith("v_permlane") and "swap" in op
        if swap:
            swaps, waits = swaps + 1, 0
            for name, wrote, states in reversed(before):
                if waits >= WAITS:
                    break
                if wrote & _registers(operands):
                    short.append((function, waits, name))
                    break
                waits += states
        wrote = set()
        if op.startswith("v_"):
            wrote = _registers(operands if swap else operands.split(",")[0])
        before = before[-WAITS:] + [(op, wrote, int(operands) + 1 if op == "s_nop" else 1)]
    return swaps, short


def test_the_scan_of_assembly_itself():
    near = ["_Zf:", "v_add_f32_e32 v3, v1, v2", "v_mov_b32_e32 v9, v8", "v_permlane32_swap_b32_e32 v3, v4"]
    assert short_waits(near) == (1, [("_Zf", 1, "v_add_f32_e32")])
    assert short_waits(near[:2] + ["s_nop 1"] + near[3:]) == (1, [])
    assert short_waits(near[:2] + ["s_nop 0", "ds_read_b32 v7, v6"] + near[3:]) == (1, [])
    assert short_waits(["_Zf:", "v_fmac_f32_dpp v4, v1, v2 row_newbcast:3", near[3]])[1]
    assert short_waits(["_Zf:", "v_pk_mov_b32 v[3:4], v[6:7], v[6:7]", near[3]])[1]
    twice = short_waits(["_Zf:", "v_permlane32_swap_b32_e32 v1, v4", "s_nop 0", near[3]])
    assert twice == (2, [("_Zf", 1, "v_permlane32_swap_b32_e32")])


@pytest.mark.parametrize("source", sorted(_sources()))
def test_exchanges_wait_for_what_they_read(source):
    run = subprocess.run([build.hipcc(), *build.HIP_FLAGS, "--cuda-device-only", "-S",
                          os.path.join(build.CSRC, source), "-o", "-"], capture_output=True, text=True)
    assert run.returncode == 0, run.stderr
    swaps, short = short_waits(run.stdout.splitlines())
    assert swaps > 0 and not short, (swaps, len(short), short[:3])
