"""tbik_route_topk against its definition, evaluated in 64 bits on the CPU."""
import numpy as np
import pytest
import torch

from paper_2511_17826_amd import binding as tb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def definition(l, k, renormalize):
    """(experts, weights in 64 bits, offsets, rows, slots) of float logits [T, E]."""
    T, E = l.shape
    rank = np.where(np.isnan(l), -np.inf, l.astype(np.float64))
    below = np.isnan(l)                                              # NaN below -infinity
    experts = np.array([sorted(range(E), key=lambda e: (below[t, e], -rank[t, e], e))[:k] for t in range(T)], dtype=np.int64).reshape(T, k)
    with np.errstate(invalid="ignore", over="ignore"):
        chosen = np.take_along_axis(l.astype(np.float64), experts, 1)
        top = chosen[:, :1]
        e = np.exp(chosen - top)
        over = e if renormalize else np.exp(l.astype(np.float64) - top)
        w = np.where(top == -np.inf, 0.0, e / over.sum(1, keepdims=True))
    offsets = np.concatenate([[0], np.cumsum(np.bincount(experts.reshape(-1), minlength=E))])
    slots, fill = np.empty((T, k), np.int64), offsets[:-1].copy()
    rows = np.empty(T * k, np.int64)
    for t in range(T):
        for j in range(k):
            slots[t, j] = fill[experts[t, j]]
            fill[experts[t, j]] += 1
            rows[slots[t, j]] = t
    return experts, w, offsets, rows, slots


def check(logits, k, renormalize=True):
    got = [x.cpu().numpy() for x in tb.tbik_route_topk(logits, k, renormalize)]
    l = logits.float().cpu().numpy()
    want = definition(l, k, renormalize)
    for name, i in (("experts", 0), ("offsets", 2), ("rows", 3), ("slots", 4)):
        assert np.array_equal(got[i], want[i]), name
    # l - l_0 is rounded once (half a step of it moves the exponential by |l - l_0| 2^-24 of its value), the exponential to a step,
    # each addition and the division to half a step; numerator and sum alike.  A logit 104 or more below l_0 has an exponential under 2^-150, which
    # fp32 gives as at most its smallest number, 2^-149, however the difference was rounded: the last term covers it and the spread counts to 104.
    n = k if renormalize else l.shape[1]
    with np.errstate(invalid="ignore"):
        spread = np.where(np.isfinite(l), l, 0.0)
        spread = np.minimum(spread.max(1).astype(np.float64) - spread.min(1), 104.0) if l.size else np.zeros(l.shape[0])
    tol = np.abs(want[1]) * 2.0 ** -24 * (2 * spread[:, None] + 4 + n + 2) + 2.0 ** -126
    bad = ~(np.abs(got[1] - want[1]) <= tol) & ~(np.isnan(got[1]) & np.isnan(want[1]))
    assert not bad.any()
    return got


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (1, 128, 8), (3, 8, 8), (63, 63, 2), (64, 64, 6), (65, 65, 4), (130, 128, 8), (257, 200, 10), (100, 512, 32), (40, 300, 5), (1000, 16, 1)])
def test_choices_weights_and_order(T, E, k, dtype):
    g = torch.Generator().manual_seed(T * 1000 + E + k)
    logits = (2 * torch.randn((T, E), generator=g) + torch.randn(E, generator=g)).to(dtype).to(DEV)
    check(logits, k)
    check(logits, k, renormalize=False)


@pytest.mark.parametrize("T", [5, 200])
def test_ties_go_to_the_lower_expert(T):
    g = torch.Generator().manual_seed(T)
    check(torch.randint(-2, 3, (T, 100), generator=g).float().to(DEV), 7)
    check(torch.zeros((T, 128), device=DEV), 8)
    signs = torch.zeros((T, 70))
    signs[:, ::3] = -0.0                                             # the two zeros are equal
    check(signs.to(DEV), 4)


@pytest.mark.parametrize("T", [6, 70])
def test_masked_and_broken_logits(T):
    g = torch.Generator().manual_seed(T)
    l = torch.randn((T, 66), generator=g)
    l[0] = -float("inf")                                             # nothing left: no weight
    l[1, 3:] = -float("inf")                                         # fewer than k left
    l[2, 5] = float("nan")                                           # never among the k
    l[3] = float("nan")
    l[4] = torch.finfo(torch.float32).min                            # a mask of the type's lowest value
    l[5, 1:64] = torch.finfo(torch.float32).min
    got = check(l.to(DEV), 4)
    assert np.all(got[1][0] == 0) and np.all(got[1][1][3:] == 0) and np.isfinite(got[1][2]).all() and np.isnan(got[1][3]).all()
    l[2, 5] = 0.0
    l[3] = 0.0
    check(l.to(DEV), 4, renormalize=False)


def test_rows_apart_and_no_tokens():
    g = torch.Generator().manual_seed(3)
    wide = torch.randn((90, 50), generator=g).to(DEV)
    check(wide[:, 3:45], 5)                                          # every row at an odd address
    experts, weights, offsets, rows, slots = tb.tbik_route_topk(torch.empty((0, 9), device=DEV), 3)
    assert experts.shape == weights.shape == slots.shape == (0, 3) and rows.numel() == 0
    assert offsets.cpu().tolist() == [0] * 10


def test_a_tokens_choices_do_not_depend_on_the_batch():
    g = torch.Generator().manual_seed(4)
    l = torch.randn((300, 128), generator=g).to(DEV)
    e, w = tb.tbik_route_topk(l, 8)[:2]
    for lo, hi in ((0, 1), (17, 81), (100, 300)):
        e2, w2 = tb.tbik_route_topk(l[lo:hi], 8)[:2]
        assert torch.equal(e2, e[lo:hi]) and torch.equal(w2.view(torch.int32), w[lo:hi].view(torch.int32))


def test_two_graphs_with_workspaces():
    """Captured calls have workspaces of their own: replays of two graphs, eager calls and larger eager calls between them agree."""
    g = torch.Generator().manual_seed(5)
    ls = [torch.randn((T, 96), generator=g).to(DEV) for T in (500, 700)]
    want = [tb.tbik_route_topk(l, 6) for l in ls]
    graphs, outs = [], []
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for l in ls:
            tb.tbik_route_topk(l, 6)
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                outs.append(tb.tbik_route_topk(l, 6))
            graphs.append(graph)
    torch.cuda.current_stream().wait_stream(side)
    for _ in range(3):
        for graph, out in zip(graphs, outs):
            for t in out:
                t.fill_(-1)
            graph.replay()
        tb.tbik_route_topk(torch.randn((5000, 512), device=DEV), 4)
        torch.cuda.synchronize()
        for out, w in zip(outs, want):
            assert all(torch.equal(a, b) for a, b in zip(out, w))


def test_refusals():
    l = torch.randn((4, 8), device=DEV)
    with pytest.raises(tb.TbikError):
        tb.tbik_route_topk(l, 9)
    with pytest.raises(tb.TbikError):
        tb.tbik_route_topk(l, 0)
    with pytest.raises(ValueError):
        tb.tbik_route_topk(l.cpu(), 2)
    with pytest.raises(ValueError):
        tb.tbik_route_topk(l.t(), 2)
    with pytest.raises(TypeError):
        tb.tbik_route_topk(l.double(), 2)
