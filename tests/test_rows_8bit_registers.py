"""A row of the norms to 8 bits stays in registers: no form of the kernel spills, and the forms that hold the most (many planes of partial
sums, rows of up to 65536 columns) give the bits of the numpy steps."""
import os

import pytest
import torch

import eight_bit_reference as ref
from paper_2511_17826_amd import binding as tb, build

EPS = 1e-6
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


def test_no_form_of_the_norm_spills():
    asm = os.path.join(build.BUILD, "rmsnorm_8bit-hip-amdgcn-amd-amdhsa-gfx950.s")
    if not os.path.exists(asm):
        pytest.skip("the library was built elsewhere")
    build.check_generated_code(asm, "rmsnorm_8bit_kernel")


@pytest.mark.gpu
@pytest.mark.parametrize("micro", [False, True])
@pytest.mark.parametrize("P,M,H,dtype", [(16, 2, 20480, "bf16"), (16, 1, 65536, "fp16"), (16, 3, 33792, "bf16"), (16, 2, 16416, "fp16"), (8, 2, 40000, "fp16"),
                                         (4, 2, 40000, "bf16"), (2, 1, 65536, "bf16"), (1, 3, 32800, "fp16"), (16, 5, 8192, "bf16")])
def test_wide_rows_of_partial_sums(P, M, H, dtype, micro):
    fmt = ("e4m3", "e5m2")[(P + M) % 2]
    g = torch.Generator().manual_seed(P + M + H)
    parts = torch.randn((P, M, H), generator=g).cuda()
    r, w = torch.randn((M, H), generator=g).to(TYPES[dtype]).cuda(), (1 + 0.1 * torch.randn(H, generator=g)).to(TYPES[dtype]).cuda()
    want, _ = (tb.tbik_combine_residual_rmsnorm if dtype == "bf16" else tb.tbik_combine_residual_rmsnorm_f16)(parts, r, w, EPS)
    hidden, q, scale = (tb.tbik_combine_residual_rmsnorm_mxfp8 if micro else tb.tbik_combine_residual_rmsnorm_fp8)(parts, r, w, EPS, fmt=fmt)
    assert torch.equal(hidden.view(torch.int16), want.view(torch.int16))
    v = ref.normed32(hidden.float().cpu().numpy(), w.float().cpu().numpy(), EPS)
    want_q, want_s = (ref.micro_scaled if micro else ref.row_scaled)(v, fmt)
    assert (scale.cpu().numpy() == want_s).all() and ref.same_patterns(q.cpu().numpy(), want_q, fmt)


@pytest.mark.gpu
@pytest.mark.parametrize("H", [2048, 4096, 5120, 6144])
def test_rows_around_the_switch_of_forms(H):
    """512 rows take another form of the kernel than 513: a row's bits are the same in both."""
    g = torch.Generator(device="cuda").manual_seed(H)
    x, r = (torch.randn((1100, H), generator=g, device="cuda").bfloat16() for _ in range(2))
    w = torch.randn(H, generator=g, device="cuda").bfloat16()
    for f in (tb.tbik_rmsnorm_fp8, tb.tbik_rmsnorm_mxfp8):
        whole = f(x, w, EPS, residual=r)
        for M in (511, 512, 513, 1024):
            assert all(torch.equal(a, b[:M]) for a, b in zip(f(x[:M], w, EPS, residual=r[:M]), whole)), M
