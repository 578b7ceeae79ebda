"""Waits around the inline assembly of the products with weights in 4 bits, in the listing of what was compiled (no GPU is touched)."""
import os
import re
import subprocess

from paper_2504_08009_amd import build as b

# An instruction that takes a register from another lane may follow the vector instruction that wrote this register only after two
# others, or a wait of two; the compiler sees to that among its own instructions, but not for those of a statement in assembly.
WAIT = 2
PROBE = """
#include "oz2_w4_matvec.h"
hipError_t one(const W4Call& a) { return launch_tile<OZ2_BF16, 1, 1, false, true>(a); }
hipError_t other(const W4Call& a) { return launch_tile<OZ2_F32, 4, 4, true, false>(a); }
"""


def registers(operand):
    found = re.match(r"v(\d+)$|v\[(\d+):(\d+)\]$", operand)
    if not found:
        return set()
    first, last = (found.group(1),) * 2 if found.group(1) else found.group(2, 3)
    return set(range(int(first), int(last) + 1))


def too_early(assembly):
    """(number of instructions that read other lanes, those of them that come too early behind a register's writer)"""
    count, faults, before = 0, [], []
    for line in assembly.splitlines():
        code = line.split(";")[0].split("//")[0].strip()
        if re.match(r"[\w.]+:", code):
            before = []  # (a jump's target: what comes before it is not known from here on)
        if not code or code.startswith(".") or code.endswith(":"):
            continue
        name, _, rest = code.partition(" ")
        operands = re.split(r",\s*|\s+", rest.strip())
        reads = set()
        if name.startswith("v_permlane"):
            reads = registers(operands[0]) | registers(operands[1])
        elif name.endswith("_dpp"):
            reads = registers(operands[1])
        if reads:
            count += 1
            states = 0
            for writes, waits, writer in reversed(before):
                if states >= WAIT:
                    break
                if writes & reads:
                    faults.append((writer, code))
                    break
                states += waits
        writes = registers(operands[0]) if name.startswith("v_") else set()
        if "swap" in name:
            writes |= registers(operands[1])
        before = before[-7:] + [(writes, int(operands[0], 0) + 1 if name == "s_nop" else 1, code)]
    return count, faults


def test_what_is_counted():
    def faults(*lines):
        return len(too_early("\n".join(lines))[1])

    assert faults("v_mov_b32_e32 v1, v2", "s_nop 1", "v_permlane32_swap_b32_e32 v1, v3") == 0
    assert faults("v_mov_b32_e32 v1, v2", "s_nop 0", "v_permlane32_swap_b32_e32 v1, v3") == 1
    assert faults("v_mov_b32_e32 v3, v2", "s_nop 0", "v_permlane16_swap_b32_e32 v1, v3") == 1
    assert faults("v_mov_b32_e32 v4, v2", "v_permlane16_swap_b32_e32 v1, v3") == 0
    assert faults("v_permlane16_swap_b32_e32 v1, v3", "s_nop 0", "v_permlane32_swap_b32_e32 v3, v5") == 1
    assert faults("v_mov_b32_e32 v4, v2", "v_mov_b32_e32 v6, v2", "s_mov_b32 s0, 0", "v_cndmask_b32_dpp v0, v4, v5, vcc quad_perm:[1,0,3,2]") == 0
    assert faults("v_mov_b32_e32 v4, v2", "s_mov_b32 s0, 0", "v_cndmask_b32_dpp v0, v4, v5, vcc quad_perm:[1,0,3,2]") == 1
    assert faults("v_mov_b32_e32 v5, v2", "v_cndmask_b32_dpp v0, v4, v5, vcc quad_perm:[1,0,3,2]") == 0  # (the second operand is the lane's own)


def test_words_change_lanes_no_earlier_than_they_may(tmp_path):
    source = tmp_path / "probe.hip"
    source.write_text(PROBE)
    run = subprocess.run(["hipcc"] + b.HIP_FLAGS + b.EXTRA_FLAGS["oz2_w4_bf16.hip"] + ["-I", b.CSRC, "--offload-device-only", "-S", str(source), "-o", "-"],
                         stdout=subprocess.PIPE, stderr=subprocess.DEVNULL)
    assert run.returncode == 0
    count, faults = too_early(run.stdout.decode())
    assert count > 24
    assert not faults, "%d of %d: %s" % (len(faults), count, faults[0])
