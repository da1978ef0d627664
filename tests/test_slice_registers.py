"""The 8-bit slices with two steps in flight are there so that two workgroups of eight wavefronts share a compute unit, which takes 128
registers a lane and less than half of its LDS: with an epilogue as without."""
import os
import re

import pytest

from paper_2511_17826_amd import build


def test_two_workgroups_fit_a_compute_unit():
    path = os.path.join(build.BUILD, "gemm_slice-hip-amdgcn-amd-amdhsa-gfx950.s")
    if not os.path.exists(path):
        pytest.skip("the library was built elsewhere")
    registers = {}
    for m in re.finditer(r"\.name:\s+\S*gemm_slice_kernelILi(\d)ELb([01])ELi(\d)ELi8ELi(\d)ELb([01])E.*?\.vgpr_count:\s+(\d+)", open(path).read(), re.S):
        registers[tuple(int(x) for x in m.groups()[:5])] = int(m[6])          # (format, scales, groups, steps in flight, epilogue)
    shared = {k: n for k, n in registers.items() if k[0] < 2 and not k[1] and k[2] == 1 and k[3] == 2}
    assert len(shared) == 4 and all(n <= 128 for n in shared.values()), shared
