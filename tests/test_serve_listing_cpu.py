"""Reads of matrix instructions' results by inline assembly in the attention of new tokens stand far enough behind them.

The compiler keeps the wait states between a matrix instruction and whoever reads its result, but not for reads inside inline
assembly.  How many it keeps is taken from a small kernel; the reads by hand are looked up in the listing of the library's own
source, along every way that leads forward to them.
"""
import os
import re

from paper_1805_12096_amd import build
from test_accumulator_reads_cpu import listing, needed  # noqa: F401  (a fixture)


def registers(operand):
    m = re.match(r"-?\|?([va])(?:\[(\d+):(\d+)\]|(\d+)\b)", operand)
    if not m:
        return []
    low, high = (m.group(2), m.group(3)) if m.group(2) else (m.group(4), m.group(4))
    return [(m.group(1), r) for r in range(int(low), int(high) + 1)]


def distances(text):
    """(wait states since the matrix instruction that wrote it, kernel, instruction) of every such read by hand."""
    found, age, ways, by_hand, kernel = [], {}, {}, False, None
    for line in text.splitlines():
        line = line.strip()
        if line.startswith(";;#ASM"):
            by_hand = line.startswith(";;#ASMSTART")
        code = line.split(";")[0].strip()
        label = re.match(r"([^\s:]+):$", code)
        if label:
            if label.group(1).startswith("_Z"):
                kernel, age, ways = label.group(1), {}, {}
            for r, a in ways.pop(label.group(1), {}).items():
                age[r] = min(age.get(r, a), a)
            continue
        if not code or code.startswith("."):
            continue
        op = code.split()[0]
        operands = [x.strip() for x in code[len(op):].split(",")]
        if op.startswith(("s_cbranch", "s_branch")):
            there = ways.setdefault(operands[0], {})
            for r, a in age.items():
                there[r] = min(there.get(r, a + 1), a + 1)
            age = {} if op == "s_branch" else {r: a + 1 for r, a in age.items()}
            continue
        if by_hand and op.startswith("v_"):
            found += [(age[r], kernel, code) for x in operands[1:] for r in registers(x) if r in age]
        step = int(operands[0]) + 1 if op == "s_nop" else 1
        age = {r: a + step for r, a in age.items()}
        for r in registers(operands[0]):
            if op.startswith("v_mfma"):
                age[r] = 0
            else:
                age.pop(r, None)
    return found


def test_the_reader_of_listings_follows_branches():
    text = "_Zk:\nv_mfma_f32_32x32x16_bf16 v[0:15], v[20:23], v[24:27], v[0:15]\ns_cbranch_scc0 .L1\ns_nop 7\n.L1:\n;;#ASMSTART\n" \
           "v_max3_f32 v30, v31, v0, v1\n;;#ASMEND\n"
    assert distances(text) == [(1, "_Zk", "v_max3_f32 v30, v31, v0, v1")] * 2


def test_reads_by_hand_keep_the_compilers_distance(needed, tmp_path):  # noqa: F811
    found = distances(listing(os.path.join(build.CSRC, "mq_chunk.hip"), tmp_path / "chunk.s"))
    assert len(found) > 100
    assert not [f for f in found if f[0] < needed]
