"""The 8-bit rows at their smallest: no columns."""
import pytest
import torch

from paper_2511_17826_amd import binding as tb

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_an_activation_without_columns_has_the_scale_of_zeros(dtype):
    """A scale per row is 1 for a row of zeros, so also for one that has no element; a caller's scale tensor is not left as it was."""
    gate, up = (torch.zeros((5, 0), dtype=dtype, device="cuda") for _ in range(2))
    given = torch.full((5,), 7.0, device="cuda")
    for kw in ({}, dict(scale=given)):
        q, scale = tb.tbik_silu_mul_fp8(gate, up, **kw)
        assert q.shape == (5, 0) and scale.shape == (5,) and bool((scale == 1).all())
    q, scale = tb.tbik_silu_mul_mxfp8(gate, up)
    assert q.shape == (5, 0) and scale.shape == (5, 0)
    assert [tuple(t.shape) for t in tb.tbik_silu_mul_fp8(gate[:0], up[:0])] == [(0, 0), (0,)]
    with pytest.raises(tb.TbikError):
        tb.tbik_rmsnorm_fp8(gate, torch.zeros(0, dtype=dtype, device="cuda"))            # a mean of nothing
