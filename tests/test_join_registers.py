"""A row of the norms around a block stays in registers over both: no form of the kernel spills, and the forms that hold the most (many
planes of partial sums, rows of more than 32768 columns) give the bits of the sums combined first."""
import os

import pytest
import torch

from paper_2511_17826_amd import binding as tb, build

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


def test_no_form_spills():
    asm = os.path.join(build.BUILD, "rmsnorm_join-hip-amdgcn-amd-amdhsa-gfx950.s")
    if not os.path.exists(asm):
        pytest.skip("the library was built elsewhere")
    build.check_generated_code(asm, "rmsnorm_join_kernel")


@pytest.mark.gpu
@pytest.mark.parametrize("P,M,H,dtype", [(8, 3, 32776, "bf16"), (8, 1, 65536, "fp16"), (8, 2, 40000, "bf16"), (16, 3, 32776, "fp16"), (16, 1, 65536, "bf16"), (16, 2, 40000, "fp16"),
                                         (4, 2, 65536, "bf16"), (16, 2, 32768, "bf16"), (8, 2, 16392, "fp16")])
def test_wide_rows_of_partial_sums(P, M, H, dtype):
    g = torch.Generator().manual_seed(P + M + H)
    parts = torch.randn((P, M, H), generator=g).cuda()
    residual, gate = (torch.randn((M, H), generator=g).to(TYPES[dtype]).cuda() for _ in range(2))
    post, nxt = ((1 + 0.1 * torch.randn(H, generator=g)).to(TYPES[dtype]).cuda() for _ in range(2))
    y = tb.tbik_tree_combine(parts, out_dtype=TYPES[dtype])
    for weight in (post, None):
        got = tb.tbik_rmsnorm_residual_rmsnorm(parts, residual, weight, nxt, 1e-6, residual_scale=0.5, gate=gate)
        want = tb.tbik_rmsnorm_residual_rmsnorm(y, residual, weight, nxt, 1e-6, residual_scale=0.5, gate=gate)
        assert all(torch.equal(a.view(torch.int16), b.view(torch.int16)) for a, b in zip(got, want))
