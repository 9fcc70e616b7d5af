"""Reads of accumulation registers that the library writes by hand stand far enough behind the matrix instructions.

The compiler keeps the wait states between a matrix instruction and whoever reads its result, but not for reads inside inline
assembly.  How many it keeps is taken from a small kernel, and the hand-written reads are looked up in the listing of the
library's own source.
"""
import os
import re
import subprocess

import pytest

from paper_1805_12096_amd import build

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
SMALL = """
#include <hip/hip_runtime.h>
typedef float v16f __attribute__((ext_vector_type(16)));
typedef %s p8 __attribute__((ext_vector_type(8)));
extern "C" __global__ void small(const p8* a, float* o) {
  v16f x = {};
  x = __builtin_amdgcn_mfma_f32_32x32x16_%s(a[threadIdx.x], a[threadIdx.x + 64], x, 0, 0, 0);
  o[threadIdx.x] = x[0] * 3.f;
}
"""


def listing(source, out):
    r = subprocess.run([HIPCC, *build.HIPCC_FLAGS, "-S", "--offload-device-only", source, "-o", str(out)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    return open(out).read()


def distances(text):
    """(kernel, place, wait states since the matrix instruction that wrote it) of every accumulation register read by hand."""
    found, written, now, by_hand, kernel = [], {}, 0, False, None
    for line in text.splitlines():
        line = line.strip()
        if line.startswith(";;#ASM"):
            by_hand = line.startswith(";;#ASMSTART")
        code = line.split(";")[0].strip()
        label = re.match(r"([^\s:]+):$", code)
        if label:                                   # (other ways may lead here: only what stands in a line is looked at)
            kernel = label.group(1) if label.group(1).startswith("_Z") else kernel
            written = {}
        if not code or label or code.startswith("."):
            continue
        op = code.split()[0]
        read = re.search(r"\ba(\d+)$", code)
        if by_hand and op.startswith("v_accvgpr_read") and read:
            found.append((kernel, code, now - written[int(read.group(1))] if int(read.group(1)) in written else None))
        now += int(code.split()[1]) + 1 if op == "s_nop" else 1
        to = re.search(r"\ba\[(\d+):(\d+)\]", code.split(",")[0])
        if op.startswith("v_mfma") and to:
            written.update((r, now) for r in range(int(to.group(1)), int(to.group(2)) + 1))
    return found


@pytest.fixture(scope="module")
def needed(tmp_path_factory):
    at, most = tmp_path_factory.mktemp("small"), 0
    for kind, name in (("__bf16", "bf16"), ("_Float16", "f16")):
        source = at / f"{name}.hip"
        source.write_text(SMALL % (kind, name))
        between = re.search(r"v_mfma[^\n]*\n(.*?)v_mul_f32", listing(source, at / f"{name}.s"), re.S).group(1)
        lines = [x.split(";")[0].split() for x in between.splitlines() if x.split(";")[0].strip()]
        most = max(most, sum(int(x[1]) + 1 if x[0] == "s_nop" else 1 for x in lines))
    assert most >= 8
    return most


def test_hand_written_reads_keep_the_compilers_distance(needed, tmp_path):
    found = distances(listing(os.path.join(build.CSRC, "mq_prompt.hip"), tmp_path / "prompt.s"))
    assert len([d for _, _, d in found if d is not None]) > 100
    short = [f for f in found if f[2] is not None and f[2] < needed]
    assert not short, short
