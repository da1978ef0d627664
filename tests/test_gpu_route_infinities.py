"""tbik_route_topk on infinite and broken logits, against its definition in 64 bits: +infinity and NaN spread as the formula has it, over the chosen
experts and over all, in one workgroup (up to 64 tokens) and in many, also where the blocks' counts are summed in chunks."""
import numpy as np
import pytest
import torch

from paper_2511_17826_amd import binding as tb
from test_gpu_route import check

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
INF = float("inf")


def logits(T, E, seed):
    l = torch.randn((T, E), generator=torch.Generator().manual_seed(seed))
    l[0, E // 2] = INF                                               # one: not a number over itself, which the sum spreads
    l[1, 1::3] = INF                                                 # several, more than k
    l[2, 0], l[2, E - 1] = INF, -INF
    l[3, 3], l[3, 4] = INF, float("nan")
    l[4, 5] = float("nan")                                           # not chosen, in the sum over all
    l[5] = float("nan")
    l[6] = -INF
    l[7] = -INF
    l[7, 2] = float("nan")                                           # nothing but it: the others come first, without weight
    l[8] = INF
    return l


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T,E", [(9, 20), (64, 128), (65, 64), (200, 130), (300, 512)])
@pytest.mark.parametrize("renormalize", [True, False])
def test_infinite_and_broken_logits(T, E, dtype, renormalize):
    got = check(logits(T, E, T + E).to(dtype).to(DEV), 5, renormalize)
    w = got[1]
    assert np.isnan(w[[0, 1, 2, 3, 5, 8]]).all() and np.isfinite(w[9:]).all()
    assert np.isnan(w[4]).all() != renormalize and (w[6] == 0).all() and (w[7] == 0).all()


def test_tokens_behind_broken_ones_in_chunks_of_blocks():
    """More than 1024 blocks of 32 tokens: the broken rows' choices count like any others."""
    l = torch.randn((33000, 8), generator=torch.Generator().manual_seed(1))
    l[::7, 3] = INF
    l[::11] = float("nan")
    l[::13] = -INF
    check(l.to(DEV), 2)
    experts, weights, offsets, rows, slots = tb.tbik_route_topk(l.to(DEV), 2, renormalize=False)
    first = tb.tbik_route_topk(l.to(DEV), 2)
    assert all(torch.equal(a, b) for a, b in zip((experts, offsets, rows, slots), (first[0], *first[2:])))
