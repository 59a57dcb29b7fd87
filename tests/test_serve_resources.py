"""What the compiler reports for the kernels of the paged cache and the rotary positions (see test_kernel_resources.py): no spills, and
the workgroups per CU that the launches count on.  CPU only; skipped when the library has not been built here."""
import os
import re

import pytest

from paper_2508_04711_amd import build as lib_build

# name, waves per workgroup, workgroups per CU that the division of the work counts on
EXPECTED = [
    (r"paged_few_kernelILb[01]ELi\d+ELi\d+ELb[01]ELi1ELi[02]E", 1, 4),         # a one-wave worker per SIMD
    (r"paged_few_kernelILb[01]ELi\d+ELi\d+ELb[01]ELi8ELi0E", 8, 1),
    (r"paged_many_kernelILi\d+ELi\d+ELb[01]ELi[02]E", 4, 2),
    (r"paged_many_kernelILi(32ELi(32|64|128)|64ELi(32|64)|128ELi32)ELb[01]ELi[02]E", 4, 3),
    (r"paged_plan_kernelILb[01]E", 16, 1),
    (r"paged_reduce_kernelILi(16|128)ELi(32|64|128)E", 4, 8),
    (r"rotary_kernelILb[01]ELb[01]ELb[01]ELb[01]E", 4, 6),
]


@pytest.mark.parametrize("pattern,waves,per_cu", EXPECTED, ids=[e[0] for e in EXPECTED])
def test_kernels_of_the_cache(pattern, waves, per_cu):
    if not os.path.exists(lib_build.RESOURCES):
        pytest.skip("library not built here")
    found = 0
    for line in open(lib_build.RESOURCES):
        name, *pairs = line.split()
        if not re.search(pattern, name):
            continue
        found += 1
        v = dict(p.partition("=")[::2] for p in pairs)
        assert int(v["VGPRs_Spill"]) == 0 and int(v["ScratchSize_[bytes/lane]"]) == 0, line
        assert int(v["Occupancy_[waves/SIMD]"]) * 4 >= waves * per_cu, line
        assert int(v["LDS_Size_[bytes/block]"]) * per_cu <= 160 * 1024, line
    assert found, pattern
