"""The epilogues' activations far from zero: the bound that tbik.h states, relative with a floor of 2^-100, over the whole of fp32, and what
infinities and NaN become.  eight_bit_reference.act_tolerance derives the relative part."""
import numpy as np
import pytest
import torch

import eight_bit_reference as ref
from paper_2511_17826_amd import binding as tb

pytestmark = pytest.mark.gpu
ACTS = ["relu", "silu", "gelu", "gelu_tanh"]


def through(v, act, out=torch.float32):
    return tb.tbik_tree_combine_epilogue(v.reshape(1, 1, -1).cuda(), activation=act, out_dtype=out).cpu()[0]


@pytest.mark.parametrize("act", ACTS)
def test_tails(act):
    """-88 to -12 (where e^88 is near fp32's largest number and its reciprocal subnormal), past it, and the same on the positive side."""
    tail = torch.cat([torch.linspace(12, 88, 50000), torch.linspace(88, 110, 5000), torch.exp2(torch.linspace(7, 127.9, 5000))])
    for v in (-tail, tail):
        x = v.numpy().astype(np.float64)
        with np.errstate(over="ignore", invalid="ignore"):
            # the definition's limits where x^3 leaves fp64's or the exponent's range: 0 and x
            want = np.where(np.abs(x) > 1e4, np.maximum(x, 0.0), ref.act64(np.clip(x, -1e4, 1e4), act))
            # e^-v enters the positive side as 1 + e^-v = 1: no term in v is left
            tol = ref.act_tolerance(x, act) if v is not tail else ref.act_tolerance(np.zeros_like(x), act)
        err = np.abs(through(v, act).numpy().astype(np.float64) - want)
        bound = np.where(want == 0, 0.0, np.minimum(tol, 1e30) * np.abs(want)) + 2.0 ** -100
        assert np.all(err <= bound), (act, x[err > bound][:5], err[err > bound][:5])


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
def test_infinities_and_nan(act, out):
    inf = float("inf")
    y = through(torch.tensor([inf, -inf, float("nan"), 0.0, -0.0]), act, out).float()
    assert y[0] == inf and torch.isnan(y[2]) and y[3] == 0 and y[4] == 0
    assert y[1] == 0 if act == "relu" else torch.isnan(y[1])
    # an element's infinity stays its own: the product's other columns are as without
    x = torch.ones((2, 64), dtype=torch.bfloat16, device="cuda")
    w = torch.ones((64, 128), dtype=torch.bfloat16, device="cuda")
    bias = torch.zeros(128, device="cuda")
    bias[5] = -inf
    z = tb.tbik_gemm_epilogue(x, w, 64, 1, bias=bias, activation=act, out_dtype=torch.float32).cpu()
    clean = tb.tbik_gemm_epilogue(x, w, 64, 1, activation=act, out_dtype=torch.float32).cpu()
    keep = [i for i in range(128) if i != 5]
    assert torch.equal(z[:, keep], clean[:, keep]) and bool((z[:, 5] == 0).all() if act == "relu" else torch.isnan(z[:, 5]).all())
