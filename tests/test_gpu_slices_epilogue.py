"""The slices of small low-bit batches with an epilogue, in every form: one and two groups of rows, steps in flight for a workgroup that has a
compute unit to itself and for two that share one (more than 4096 channels), scaled and plain, with the last channels ragged."""
import pytest
import torch

import test_gpu_gemm_epilogue as ge
from paper_2511_17826_amd import binding as tb

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["fp8 e4m3", "fp8 e5m2", "mx e4m3", "mx e5m2"])
@pytest.mark.parametrize("M,K,N", [(1, 4096, 4136), (7, 4096, 8200), (16, 2048, 6152), (17, 1024, 4136), (32, 2048, 520), (3, 8192, 4096)])
def test_every_form_of_the_slices(kind, M, K, N):
    leaf = 256
    # scaled, more than 16 rows and 4096 channels are quicker in tiles
    assert ge.route_of(kind, M, N, K, leaf, 1) == [(M, "slices", 0, 0) if kind[:2] != "mx" or M <= 16 or N <= 4096 else (M, "tiles", 32, 1)]
    product, partials, with_epilogue = ge.operands(kind, M, K, N, M + K)
    t = product(leaf, 1)
    for out in ("bf16", "fp16", "fp32"):
        scales, bias, residual = ge.parts_of_an_epilogue(M, N, ge.TYPES[out], N)
        call = lambda **kw: with_epilogue(leaf, 1, out_dtype=ge.TYPES[out], **kw)
        assert ge.same(call(), t.to(ge.TYPES[out]))
        assert ge.same(call(bias=bias, residual=residual, **scales), ge.composed(t, ge.TYPES[out], scales, bias, None, residual))
        wide = torch.full((M, N + 9), 3.0, dtype=ge.TYPES[out], device="cuda")
        into = wide[:, 4:4 + N]
        into.copy_(residual)
        call(bias=bias, activation="gelu", residual=into, out=into, **scales)          # in place, at an odd address
        parts = partials(leaf, 1, 4)
        assert ge.same(into.contiguous(), tb.tbik_tree_combine_epilogue(parts, bias=bias, activation="gelu", residual=residual, out_dtype=ge.TYPES[out], **scales))
        assert bool((wide[:, :4] == 3).all()) and bool((wide[:, 4 + N:] == 3).all())
