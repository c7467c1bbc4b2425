"""The attention kernels' loads to LDS write M0 in inline assembly: the compiler
is told so, and the kernels as built use it for nothing else."""

import os
import re

from test_kernel_code_cpu import ROOT, kernels  # noqa: F401


def test_assembly_that_writes_m0_says_so():
    with open(os.path.join(ROOT, "paper_2609_16742_amd", "csrc", "attention.h")) as f:
        blocks = re.findall(r"asm volatile\((.*?)\);", f.read(), re.S)
    writers = [b for b in blocks if re.search(r"\bm0,", b)]
    assert len(writers) == 2
    for b in writers:
        assert '"m0"' in b.rsplit(":", 1)[1], b


def test_m0_is_the_loads_alone(kernels):  # noqa: F811
    seen = 0
    for name, ins in kernels.items():
        if "attend" not in name:
            continue
        for i, s in enumerate(ins):
            if re.search(r"\bm0\b", s):
                seen += 1
                assert s.startswith("s_mov_b32 m0, s"), (name, s)
                assert ins[i + 2].startswith("buffer_load") and ins[i + 2].endswith("lds"), (
                    name, ins[i:i + 3])
    assert seen > 100
