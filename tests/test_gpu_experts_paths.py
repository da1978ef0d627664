"""The calls of a mixture of experts, of 4-bit weights and of the norms around a block where they take another way: the binding's native half and ctypes,
another stream, workspaces in graphs, rows far apart, very many tokens and rows."""
import pytest
import torch

from paper_2511_17826_amd import binding as tb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
bf, f16, f32, i32, u8 = torch.bfloat16, torch.float16, torch.float32, torch.int32, torch.uint8
K, N = 512, 136


def rnd(shape, dtype=bf, seed=1):
    g = torch.Generator(device=DEV).manual_seed(seed + len(shape) + sum(shape))
    return torch.randn(shape, generator=g, device=DEV).to(dtype)


def whole(shape, hi, dtype=u8, seed=1):
    g = torch.Generator(device=DEV).manual_seed(seed + sum(shape))
    return torch.randint(0, hi, shape, generator=g, device=DEV, dtype=dtype)


ENDS = lambda m: torch.tensor([0, m // 2, m // 2, m], dtype=i32, device=DEV)
W4 = lambda m, t: (rnd((m, K), t), whole((N, K // 2), 256), rnd((N, K // 64), t), 64, 1)
CALLS = {
    "route": lambda m: (tb.tbik_route_topk, (rnd((m, 96), f32), 6), {}),
    "route_all": lambda m: (tb.tbik_route_topk, (rnd((m, 96)), 6, False), {}),
    "grouped": lambda m: (tb.tbik_gemm_grouped, (rnd((m, K)), rnd((3, K, N)), ENDS(m), 64), {}),
    "grouped_f32": lambda m: (tb.tbik_gemm_grouped, (rnd((5, K), f16), rnd((3, K, N), f16), ENDS(m), 64, 1), dict(rows=whole((m,), 5, i32), out_dtype=f32)),
    "swiglu": lambda m: (tb.tbik_gemm_grouped_swiglu, (rnd((5, K)), rnd((3, K, 2 * N)), ENDS(m), 64), dict(rows=whole((m,), 5, i32))),
    "grouped_shards": lambda m: (tb.tbik_gemm_grouped_shard_partials, (rnd((m, K)), rnd((3, K, N)), ENDS(m), 64, 1, 4), {}),
    "sum": lambda m: (tb.tbik_combine_experts, (rnd((9, N)), whole((m, 4), 9, i32), rnd((m, 4), f32)), {}),
    "sum_residual": lambda m: (tb.tbik_combine_experts, (rnd((2, 9, N), f32), whole((m, 4), 9, i32), rnd((m, 4), f32)), dict(residual=rnd((m, N), f16))),
    "sum_f32": lambda m: (tb.tbik_combine_experts, (rnd((9, N)), whole((m, 4), 9, i32), rnd((m, 4), f32)), dict(out_dtype=f32)),
    "w4": lambda m: (tb.tbik_gemm_w4, W4(m, bf), {}),
    "w4_zeros": lambda m: (tb.tbik_gemm_w4, W4(m, f16), dict(zeros=whole((N, K // 64), 16), out_dtype=f32)),
    "w4_shards": lambda m: (tb.tbik_gemm_shard_partials_w4, W4(m, bf) + (2,), dict(zeros=whole((N, K // 64), 16))),
    "join": lambda m: (tb.tbik_rmsnorm_residual_rmsnorm, (rnd((m, N)), rnd((m, N), seed=2), rnd((N,)), rnd((N,), seed=3)), dict(gate=rnd((m, 1)), residual_scale=0.5)),
    "join_shards": lambda m: (tb.tbik_rmsnorm_residual_rmsnorm, (rnd((4, m, N), f32), rnd((m, N), f16), rnd((N,), f16), None, 1e-5), dict(gate=rnd((N,), f16))),
}
HALVES = ("route", "grouped", "experts_sum", "w4", "join")


def equal(a, b):
    a, b = (t if isinstance(t, tuple) else (t,) for t in (a, b))
    assert len(a) == len(b)
    for x, y in zip(a, b):
        assert (x is None) == (y is None)
        if x is not None:
            assert x.dtype == y.dtype and x.shape == y.shape and x.device == y.device and not x.requires_grad
            assert torch.equal(x.view(u8), y.view(u8))


@pytest.mark.parametrize("m", [1, 80])
@pytest.mark.parametrize("name", list(CALLS))
def test_native_and_ctypes_give_the_same_bits(name, m, monkeypatch):
    f, args, kw = CALLS[name](m)
    tb.lib()
    answers = []
    real = tb._native
    spy = lambda g: (lambda *a: answers.append(g(*a)) or answers[-1])
    monkeypatch.setattr(tb, "_native", type("Spy", (), {k: staticmethod(spy(getattr(real, k))) for k in HALVES}))
    native = f(*args, **kw)
    assert len(answers) == 1 and answers[0] is not None           # a common call is answered there
    monkeypatch.setattr(tb, "_native", tb._NotLoaded)
    equal(native, f(*args, **kw))


@pytest.mark.parametrize("name", list(CALLS))
def test_on_the_current_stream(name):
    """Operands that another stream is still writing: the call takes its place in that stream."""
    f, args, kw = CALLS[name](80)
    want = f(*args, **kw)
    fresh = [torch.zeros_like(a) if isinstance(a, torch.Tensor) else a for a in args]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    big = torch.empty(1 << 28, dtype=u8, device=DEV)
    with torch.cuda.stream(side):
        big.fill_(1)                                                 # what the copies wait for
        for to, a in zip(fresh, args):
            if isinstance(a, torch.Tensor):
                to.copy_(a)
        got = f(*fresh, **kw)
    torch.cuda.current_stream().wait_stream(side)
    equal(got, want)
    torch.cuda.synchronize()


def test_graphs_with_workspaces_of_their_own():
    """4-bit products whose K is split: two graphs, a larger eager call between their replays."""
    ops = [(rnd((m, 4096), seed=m), whole((1160, 2048), 256), rnd((1160, 32)).abs(), 256, 1) for m in (40, 24)]
    assert all(tb.lib().tbik_gemm_w4_workspace_bytes(o[0].shape[0], 1160, 4096, 256, 1) > 0 for o in ops)
    want = [tb.tbik_gemm_w4(*o) for o in ops]
    graphs, outs = [], []
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for o in ops:
            tb.tbik_gemm_w4(*o)
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                outs.append(tb.tbik_gemm_w4(*o))
            graphs.append(graph)
    torch.cuda.current_stream().wait_stream(side)
    large = rnd((64, 4096)), whole((4096, 2048), 256), rnd((4096, 32)), 256, 1
    for _ in range(3):
        for graph, out in zip(graphs, outs):
            out.fill_(7)
            graph.replay()
        tb.tbik_gemm_w4(*large)
        torch.cuda.synchronize()
        for out, w in zip(outs, want):
            equal(out, w)


def test_gathered_rows_beyond_four_gigabytes():
    """Rows of X so far apart that their distance passes 32 bits of bytes, with and without an order."""
    far = torch.empty_strided((9, K), (1 << 29, 1), dtype=bf, device=DEV)
    X = rnd((9, K))
    far.copy_(X)
    W = rnd((3, K, N))
    rows = torch.tensor([8, 0, 8, 5, 1, 7], dtype=i32, device=DEV)
    for r, m in ((rows, 6), (None, 9)):
        equal(tb.tbik_gemm_grouped(far, W, ENDS(m), 64, rows=r), tb.tbik_gemm_grouped(X, W, ENDS(m), 64, rows=r))
        equal(tb.tbik_gemm_grouped_shard_partials(far, W, ENDS(m), 64, 1, 2, rows=r), tb.tbik_gemm_grouped_shard_partials(X, W, ENDS(m), 64, 1, 2, rows=r))
    W_gu = rnd((3, K, 2 * N))
    equal(tb.tbik_gemm_grouped_swiglu(far, W_gu, ENDS(6), 64, rows=rows), tb.tbik_gemm_grouped_swiglu(X, W_gu, ENDS(6), 64, rows=rows))
    equal(tb.tbik_gemm_w4(far, *W4(9, bf)[1:]), tb.tbik_gemm_w4(X, *W4(9, bf)[1:]))
    equal(tb.tbik_combine_experts(far, rows.reshape(2, 3), rnd((2, 3), f32)), tb.tbik_combine_experts(X, rows.reshape(2, 3), rnd((2, 3), f32)))


@pytest.mark.parametrize("T,E,k", [(32769, 8, 2), (40007, 128, 8), (70000, 300, 1), (33000, 512, 32), (300000, 64, 4)])
def test_route_of_very_many_tokens(T, E, k):
    """Choices and weights are those of the tokens in batches of 4096; the order is that of a stable sort by expert."""
    l = rnd((T, E), f32) + rnd((E,), f32)
    experts, weights, offsets, rows, slots = tb.tbik_route_topk(l, k)
    for lo in range(0, T, 4096 * 7):
        e, w = tb.tbik_route_topk(l[lo:lo + 4096], k)[:2]
        equal((experts[lo:lo + 4096].clone(), weights[lo:lo + 4096].clone()), (e, w))
    flat = experts.reshape(-1).long()
    order = torch.sort(flat, stable=True).indices
    assert torch.equal(offsets.long(), torch.cat([flat.new_zeros(1), torch.bincount(flat, minlength=E).cumsum(0)]))
    assert torch.equal(rows.long(), order // k)
    assert torch.equal(slots.reshape(-1)[order].long(), torch.arange(T * k, device=DEV))


def test_w4_of_more_rows_than_a_launch():
    """A superleaf of 32 k, which only the general kernel takes, and more rows than one launch of it has."""
    M = 32 * 4096 + 33
    X, Wq, scales = rnd((M, 64)), whole((24, 32), 256), rnd((24, 2))
    want = torch.cat([tb.tbik_gemm_w4(X[lo:lo + 5000], Wq, scales, 32) for lo in range(0, M, 5000)])
    equal(tb.tbik_gemm_w4(X, Wq, scales, 32), want)
    parts = tb.tbik_gemm_shard_partials_w4(X, Wq, scales, 32, 1, 2)
    equal(tb.tbik_tree_combine(parts), want)
