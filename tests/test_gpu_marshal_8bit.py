"""The common calls of the epilogues and 8-bit outputs go through the binding's native half; it gives what the way through ctypes
gives, and leaves to it what is not common."""
import pytest
import torch

from paper_2511_17826_amd import binding as tb

pytestmark = pytest.mark.gpu
bf, f16, f32, u8 = torch.bfloat16, torch.float16, torch.float32, torch.uint8
K, N = 1024, 256


def rnd(shape, dtype=bf):
    g = torch.Generator(device="cuda:0").manual_seed(hash(shape) % 1000)
    return torch.randn(shape, generator=g, device="cuda:0").to(dtype)


def bits(shape, lo=0, hi=120):
    g = torch.Generator(device="cuda:0").manual_seed(len(shape))
    return torch.randint(lo, hi, shape, generator=g, device="cuda:0", dtype=u8)


ENDS = lambda m, out: dict(bias=rnd((N,), f32), activation="gelu", residual=rnd((m, N), out), row_scale=rnd((m,), f32), col_scale=rnd((N,), f32))
CALLS = {
    "gemm": lambda m: (tb.tbik_gemm_epilogue, (rnd((m, K)), rnd((K, N)), 128, 1), ENDS(m, bf)),
    "gemm_f16_f32": lambda m: (tb.tbik_gemm_epilogue, (rnd((m, K), f16), rnd((K, N), f16), 128, 1), dict(ENDS(m, f32), out_dtype=f32)),
    "gemm_bias": lambda m: (tb.tbik_gemm_epilogue, (rnd((m, K)), rnd((K, N)), 128, 1, rnd((N,))), {}),
    "fp8": lambda m: (tb.tbik_gemm_fp8_epilogue, (bits((m, K)), bits((N, K)), 128, 1, "e5m2"), ENDS(m, bf)),
    "fp8_f16": lambda m: (tb.tbik_gemm_fp8_epilogue, (bits((m, K)), bits((N, K)), 128, 1), dict(ENDS(m, f16), out_dtype=f16)),
    "mxfp8": lambda m: (tb.tbik_gemm_mxfp8_epilogue, (bits((m, K)), bits((m, K // 32), 120, 130), bits((N, K)), bits((N, K // 32), 120, 130), 128, 1, "e4m3"), dict(residual=rnd((m, N)))),
    "combine": lambda m: (tb.tbik_tree_combine_epilogue, (rnd((4, m, N), f32),), ENDS(m, bf)),
    "norm_fp8": lambda m: (tb.tbik_rmsnorm_fp8, (rnd((m, K)), rnd((K,)), 1e-6), dict(residual=rnd((m, K)))),
    "norm_mx_alone": lambda m: (tb.tbik_rmsnorm_mxfp8, (rnd((m, K), f16), rnd((K,), f16), 1e-6), dict(fmt="e5m2")),
    "tail_fp8": lambda m: (tb.tbik_combine_residual_rmsnorm_fp8, (rnd((2, m, K), f32), rnd((m, K), f16), rnd((K,), f16), 1e-6), {}),
    "tail_mx": lambda m: (tb.tbik_combine_residual_rmsnorm_mxfp8, (rnd((4, m, K), f32), rnd((m, K)), rnd((K,)), 1e-6), dict(fmt="e5m2")),
    "silu_fp8": lambda m: (tb.tbik_silu_mul_fp8, (rnd((m, 2 * K))[:, :K], rnd((m, 2 * K))[:, K:]), {}),
    "silu_mx": lambda m: (tb.tbik_silu_mul_mxfp8, (rnd((m, K), f16), rnd((m, K), f16)), dict(fmt="e5m2")),
}


@pytest.mark.parametrize("m", [1, 33])
@pytest.mark.parametrize("name", list(CALLS))
def test_native_and_ctypes_give_the_same_bits(name, m, monkeypatch):
    f, args, kw = CALLS[name](m)
    tb.lib()
    answers = []
    real = tb._native
    spy = lambda g: (lambda *a: answers.append(g(*a)) or answers[-1])
    monkeypatch.setattr(tb, "_native", type("Spy", (), {k: staticmethod(spy(getattr(real, k))) for k in ("epilogue", "eight_bits")}))
    native = f(*args, **kw)
    assert len(answers) == 1 and answers[0] is not None           # a common call is answered there
    monkeypatch.setattr(tb, "_native", tb._NotLoaded)
    other = f(*args, **kw)
    native, other = (t if isinstance(t, tuple) else (t,) for t in (native, other))
    assert len(native) == len(other)
    for a, b in zip(native, other):
        assert (a is None) == (b is None)
        if a is not None:
            assert a.dtype == b.dtype and a.shape == b.shape and a.device == b.device and not a.requires_grad
            assert torch.equal(a.view(u8), b.view(u8))


def test_uncommon_arguments_are_left_to_ctypes():
    tb.lib()
    n = tb._native
    g, r = tb._NUMBER["tbik_gemm_epilogue bf16"], tb._NUMBER["tbik_rmsnorm_fp8"]
    x, w = rnd((4, K)), rnd((K, N))
    call = lambda x=x, w=w, leaf=128, out=bf, rs=None, cs=None, bias=None, act=0, res=None, g=g: n.epilogue(g, x, None, w, None, leaf, 1, out, 0, rs, cs, bias, act, res)
    assert call() is not None
    for bad in (dict(x=x.to(f16)), dict(x=x.cpu()), dict(w=w[:-1]), dict(leaf=128.0), dict(out=torch.int32), dict(rs=rnd((5,), f32)), dict(rs=rnd((4,))), dict(cs=rnd((N,), f32).cpu()),
                dict(bias=rnd((2 * N,))[::2]), dict(bias=rnd((N,), torch.float64)), dict(act=None), dict(act="gelu"), dict(res=rnd((4, N), f32)), dict(res=rnd((3, N))), dict(g=r), dict(g=99)):
        assert call(**bad) is None, bad
    weight = rnd((K,))
    norm = lambda x=x, res=None, weight=weight, eps=1e-6, fmt=3: n.eight_bits(r, x, res, weight, eps, fmt)
    assert norm() is not None
    for bad in (dict(x=x.to(f32)), dict(x=x.t().contiguous().t()), dict(x=x.cpu()), dict(res=rnd((4, K), f16)), dict(res=rnd((3, K))), dict(weight=rnd((N,))), dict(weight=rnd((K,), f16)), dict(weight=None),
                dict(eps=0), dict(fmt=None)):
        assert norm(**bad) is None, bad
    assert torch.equal(tb.tbik_rmsnorm_fp8(x, weight, 1)[1], tb.tbik_rmsnorm_fp8(x, weight, 1.0)[1])         # an integer: through ctypes


def test_errors_are_those_of_the_library():
    x, w = rnd((4, K)), rnd((K, N))
    with pytest.raises(tb.TbikError, match="tbik_gemm_epilogue: "):
        tb.tbik_gemm_epilogue(x, w, 100, 1)
    with pytest.raises(tb.TbikError, match="tbik_rmsnorm_mxfp8: "):
        tb.tbik_rmsnorm_mxfp8(rnd((4, 48)), rnd((48,)))               # not whole blocks
    with pytest.raises(tb.TbikError, match="tbik_combine_residual_rmsnorm_fp8: "):
        tb.tbik_combine_residual_rmsnorm_fp8(rnd((3, 4, K), f32), rnd((4, K)), rnd((K,)))
    with pytest.raises(ValueError):
        tb.tbik_silu_mul_fp8(x, x, fmt="e9m9")
    with pytest.raises(ValueError):
        tb.tbik_gemm_epilogue(x, w, 128, 1, activation="swish")


def test_overwritten_workspaces_of_two_streams():
    """Calls on two streams at once, each with a K split: each stream has a workspace of its own."""
    x, w = rnd((8, 16 * K)), rnd((16 * K, N))
    res = [rnd((8, N)), rnd((8, N)) + 1]
    want = [tb.tbik_gemm_epilogue(x, w, 128, 1, residual=r) for r in res]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(20):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(tb.tbik_gemm_epilogue(x, w, 128, 1, residual=res[i]))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(y, want[i]) for y in got[i])


def test_outputs_are_ordinary_tensors():
    """What the native half puts together itself behaves as a tensor that torch made."""
    x = torch.randn(3, 64, device="cuda", dtype=torch.bfloat16)
    w = torch.ones(64, device="cuda", dtype=torch.bfloat16)
    for t in tb.tbik_rmsnorm_fp8(x, w, residual=x):
        torch_s = torch.empty(t.shape, dtype=t.dtype, device="cuda")
        assert t.device == torch_s.device and t.stride() == torch_s.stride() and t.is_contiguous() and t.storage_offset() == 0 and t.is_leaf
        assert torch._C._dispatch_key_set(t) == torch._C._dispatch_key_set(torch_s) and t.untyped_storage().nbytes() == torch_s.untyped_storage().nbytes()
        assert t.untyped_storage().device == torch_s.untyped_storage().device
        want = t.cpu()
        u = t.clone()
        t.record_stream(torch.cuda.current_stream())
        assert torch.equal(t.new_empty(t.shape).copy_(t), u) and torch.equal(t[1:], u[1:]) and repr(t) == repr(u)
        t.resize_(t.numel() * 2)
        assert t.device == u.device and torch.equal(t[:u.numel()].cpu(), want.flatten())
        if t.is_floating_point():
            u.requires_grad_()
            (u * 2).sum().backward()
    with torch.inference_mode():
        y = tb.tbik_rmsnorm_fp8(x, w, residual=x)
    assert all(t.is_inference() for t in y) and not tb.tbik_rmsnorm_fp8(x, w, residual=x)[0].is_inference()
    before = torch.cuda.memory_allocated()
    y = tb.tbik_rmsnorm_fp8(x, w, residual=x)
    assert torch.cuda.memory_allocated() > before - 3 * 512
    del y
    empty = tb.tbik_rmsnorm_fp8(x[:0], w, residual=x[:0])
    assert [tuple(t.shape) for t in empty] == [(0, 64), (0, 64), (0,)]


def test_outputs_under_a_dispatch_mode():
    """Torch is asked for them where a mode listens; the mode sees the allocation."""
    from torch.utils._python_dispatch import TorchDispatchMode

    class Counts(TorchDispatchMode):
        n = 0

        def __torch_dispatch__(self, func, types, args=(), kwargs=None):
            Counts.n += "empty" in str(func)
            return func(*args, **(kwargs or {}))

    x = torch.randn(3, 64, device="cuda", dtype=torch.bfloat16)
    want = tb.tbik_silu_mul_fp8(x, x)
    with Counts():
        got = tb.tbik_silu_mul_fp8(x, x)
    assert Counts.n >= 2 and all(torch.equal(a, b) for a, b in zip(got, want))
