"""Reads of matrix instructions' results by inline assembly stand far enough behind them along every way, loops included.

test_serve_listing_cpu.py follows ways that lead forward; here the ages of results go around loops too, until none becomes smaller:
the attention of new tokens reads scores that the pass of its loop before has begun.
"""
import os
import re

from paper_1805_12096_amd import build
from test_accumulator_reads_cpu import listing, needed  # noqa: F401  (a fixture)
from test_serve_listing_cpu import registers

OLD = 40                               # wait states from which on nothing can be too early


def blocks_of(text):
    """{kernel: [(label, [(operation, operands, whether by hand)])]}: pieces that begin at labels and behind branches."""
    kernels, now, by_hand = {}, None, False
    for line in text.splitlines():
        line = line.strip()
        if line.startswith(";;#ASM"):
            by_hand = line.startswith(";;#ASMSTART")
        code = line.split(";")[0].strip()
        label = re.match(r"([^\s:]+):$", code)
        if label and label.group(1).startswith("_Z"):
            now = kernels.setdefault(label.group(1), [])
        if label and now is not None:
            now.append((label.group(1), []))
        if not code or label or code.startswith(".") or now is None:
            continue
        op = code.split()[0]
        now[-1][1].append((op, [x.strip() for x in code[len(op):].split(",")], by_hand))
        if op.startswith(("s_cbranch", "s_branch", "s_endpgm", "s_setpc")):
            now.append((None, []))
    return kernels


def through(block, age, found=None):
    """Ages behind a piece, from those in front of it."""
    age = dict(age)
    for op, operands, by_hand in block:
        if found is not None and by_hand and op.startswith("v_"):
            found += [(age.get(r, OLD), " ".join([op, *operands])) for x in operands[1:] for r in registers(x)]
        step = int(operands[0]) + 1 if op == "s_nop" else 1
        age = {r: a + step for r, a in age.items() if a + step < OLD}
        for r in registers(operands[0]) if op.startswith("v_") else []:
            if op.startswith("v_mfma"):
                age[r] = 0
            else:
                age.pop(r, None)
    return age


def distances(text):
    found = []
    for pieces in blocks_of(text).values():
        at = {label: i for i, (label, _) in enumerate(pieces) if label}
        ahead, todo = [{} for _ in pieces], list(range(len(pieces)))
        while todo:
            i = todo.pop()
            code = pieces[i][1]
            age, last = through(code, ahead[i]), code[-1] if code else ("", [""], False)
            to = [at[last[1][0]]] if last[0].startswith(("s_cbranch", "s_branch")) else []
            if not last[0].startswith(("s_branch", "s_endpgm", "s_setpc")) and i + 1 < len(pieces):
                to.append(i + 1)
            for j in to:
                less = {r: a for r, a in age.items() if a < ahead[j].get(r, OLD)}
                if less:
                    ahead[j].update(less)
                    todo.append(j)
        for (_, code), age in zip(pieces, ahead):
            through(code, age, found)
    return found


def test_ages_go_around_loops():
    text = "_Zk:\nv_mov_b32 v0, 0\n.L1:\ns_nop 1\n;;#ASMSTART\nv_max3_f32 v30, v31, v0, v1\n;;#ASMEND\ns_nop 3\n" \
           "v_mfma_f32_32x32x16_bf16 v[0:15], v[20:23], v[24:27], v[0:15]\nv_mov_b32 v1, v2\ns_cbranch_scc0 .L1\ns_endpgm\n"
    assert sorted(d for d, _ in distances(text)) == [4, OLD, OLD]          # (v31 and v1 are nobody's results)


def test_reads_by_hand_keep_the_compilers_distance_around_loops(needed, tmp_path):  # noqa: F811
    found = distances(listing(os.path.join(build.CSRC, "mq_chunk.hip"), tmp_path / "chunk.s"))
    assert len([d for d, _ in found if d < OLD]) > 100
    short = [f for f in found if f[0] < needed]
    assert not short, short[:5]
