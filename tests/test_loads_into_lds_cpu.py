"""Loads from memory into LDS that are written in assembly (csrc/tt_product_stream.h), in the device code that the compiler makes of them: it inserts the wait
states that the hardware asks for around its own instructions only, so those around an assembly block's are looked for here."""

import os
import re
import subprocess

import pytest

import __graft_entry__ as entry

CSRC = os.path.join(entry.PKG, "csrc")
SOURCE = """
#include "%s/include/tt_emb.h"
#include "%s/tt_product_stream.h"
#define KERNELS(T, WIDE)                                                                                          \\
    template __global__ void tt::product_stream_kernel<T, T, WIDE>(tt::ProductArgs, tt::EpilogueArgs);            \\
    template __global__ void tt::product_stream_kernel<T, float, WIDE>(tt::ProductArgs, tt::EpilogueArgs);        \\
    template __global__ void tt::pair_stream_kernel<T, T, WIDE>(tt::PairArgs);
KERNELS(tt::%s, true)
KERNELS(tt::%s, false)
"""


def registers(operand):
    """The scalar registers of an operand: s5, s[4:7]."""
    m = re.fullmatch(r"s\[(\d+):(\d+)\]", operand)
    if m:
        return set(range(int(m.group(1)), int(m.group(2)) + 1))
    m = re.fullmatch(r"s(\d+)", operand)
    return {int(m.group(1))} if m else set()


def hazards(lines):
    """Loads into LDS whose M0 was written less than one wait state before, or whose buffer by a vector instruction less than five before.  (Along the text:
    what stands before a label is taken to run before it.)"""
    found, n, before = [], 0, []
    for line in lines:
        line = line.split(";")[0].strip()
        if not line or line.startswith(".") or line.endswith(":"):
            continue
        op, *rest = line.split(None, 1)
        operands = [x.strip() for x in rest[0].split(",")] if rest else []
        if op.startswith("buffer_load") and line.endswith(" lds"):
            n += 1
            states, buffer = 0, registers(operands[1])
            for prior, target in reversed(before[-8:]):
                if prior.startswith("s_nop"):
                    states += int(target)                    # (and one for itself, below)
                if states < 1 and target == "m0":
                    found.append("%s %s; %s" % (prior, target, line))
                if states < 5 and prior.startswith("v_") and registers(target) & buffer:
                    found.append("%s %s; %s" % (prior, target, line))
                states += 1
        before.append((op, operands[0] if operands else ""))
    return n, found


def test_the_check_finds_what_it_looks_for():
    load = "buffer_load_dwordx4 v3, s[16:19], 0 offen lds"
    assert hazards(["s_mov_b32 m0, s20", load])[1] and hazards(["s_mov_b32 m0, s20", "s_nop 0", load]) == (1, [])
    assert hazards(["s_mov_b32 m0, s20", "s_add_i32 s1, s2, s3", load])[1] == []
    assert hazards(["v_readfirstlane_b32 s17, v0", "s_nop 3", load])[1] and hazards(["v_readfirstlane_b32 s17, v0", "s_nop 4", load])[1] == []
    assert hazards(["v_readfirstlane_b32 s20, v0", load])[1] == []


@pytest.mark.parametrize("type", ["bf16_t", "f16_t"])
def test_loads_into_lds_have_their_wait_states(tmp_path, type):
    src, out = tmp_path / "kernels.hip", tmp_path / "kernels.s"
    src.write_text(SOURCE % (entry.ROOT, CSRC, type, type))
    subprocess.check_call([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")] + [f for f in entry.HIPCC_FLAGS if f != "-Wall"] + ["--offload-device-only", "-S", "-o", str(out), str(src)])
    lines = out.read_text().splitlines()
    n, found = hazards(lines)
    assert n >= 100 and not found, (n, found[:3])
    # M0 is these loads' alone: the compiler does not know that the blocks write it
    assert sum(bool(re.search(r"\bm0\b", line.split(";")[0])) for line in lines) == n
