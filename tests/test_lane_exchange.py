"""Lanes that hand each other something through LDS without a workgroup's barrier: a barrier of the wavefront alone orders instructions' issue, not
memory, so in the sources it stands between a release and an acquire fence, or the compiler may move a read in front of another lane's write."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2407_11550_amd", "csrc")


def test_a_wavefronts_barrier_stands_between_fences():
    seen = 0
    for path in sorted(glob.glob(os.path.join(CSRC, "*"))):
        if not path.endswith((".hip", ".h")):
            continue
        with open(path) as f:
            lines = [re.sub(r"\s*//.*", "", line).strip() for line in f]
        for i, line in enumerate(lines):
            if "__builtin_amdgcn_wave_barrier()" not in line:
                continue
            seen += 1
            assert "__builtin_amdgcn_fence(__ATOMIC_RELEASE" in lines[i - 1] and "__builtin_amdgcn_fence(__ATOMIC_ACQUIRE" in lines[i + 1], f"{path}:{i + 1}"
    assert seen
