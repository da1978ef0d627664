"""The entry points of the epilogues and of the 8-bit outputs refuse bad arguments before anything is launched (CPU: fake, aligned
device pointers that validation must never let through), and the binding refuses bad tensors."""
import ctypes as C
import os

import pytest
import torch

GOOD, OTHER = 0x1000, 0x200000
F32, BF16, F16, E4M3, E5M2 = 0, 1, 2, 3, 4
OK, NULL, SHAPE, SHARDS, DTYPE, ALIGN, WORKSPACE, UNSUPPORTED = range(8)


@pytest.fixture(scope="module")
def tb():
    from paper_2511_17826_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        from paper_2511_17826_amd import build
        build.build()
    binding.lib()
    return binding


def ends(tb, **kw):
    return C.byref(tb.Epilogue(**kw))


def calls(tb):
    """name -> call(epilogue, **changes) for the four entry points, on arguments that are fine but for the changes."""
    L = tb.lib()
    good = dict(X=GOOD, ldx=512, Xs=GOOD, ldxs=16, W=GOOD, ldw=512, Ws=GOOD, ldws=16, Y=OTHER, ldy=256, yt=BF16, M=4, N=256, K=512, leaf=128, g=1, ws=None, wsb=0, P=4)

    def gemm(e, **kw):
        a = dict(dict(good, xt=BF16), **kw)
        return L.tbik_gemm_epilogue(a["X"], a["ldx"], a["W"], a["ldw"], e, a["Y"], a["ldy"], a["yt"], a["xt"], a["M"], a["N"], a["K"], a["leaf"], a["g"], a["ws"], a["wsb"], None)

    def fp8(e, **kw):
        a = dict(good, **kw)
        return L.tbik_gemm_fp8_epilogue(a["X"], a["ldx"], a["W"], a["ldw"], e, a["Y"], a["ldy"], a["yt"], a.get("xt", E4M3), a["M"], a["N"], a["K"], a["leaf"], a["g"], a["ws"], a["wsb"], None)

    def mx(e, **kw):
        a = dict(good, **kw)
        return L.tbik_gemm_mxfp8_epilogue(a["X"], a["ldx"], a["Xs"], a["ldxs"], a["W"], a["ldw"], a["Ws"], a["ldws"], e, a["Y"], a["ldy"], a["yt"], a.get("xt", E4M3),
                                          a["M"], a["N"], a["K"], a["leaf"], a["g"], a["ws"], a["wsb"], None)

    def combine(e, **kw):
        a = dict(good, **kw)
        return L.tbik_tree_combine_epilogue(a["X"], a["P"], e, a["Y"], a["ldy"], a["yt"], a["M"], a["N"], None)

    return dict(gemm=gemm, fp8=fp8, mx=mx, combine=combine)


@pytest.mark.parametrize("name", ["gemm", "fp8", "mx", "combine"])
def test_epilogue_refusals(tb, name):
    call = calls(tb)[name]
    e = lambda **kw: ends(tb, **kw)
    assert call(e(), M=0) == OK and call(e(), N=0) == OK
    assert call(None) == NULL and call(None, M=0) == NULL
    assert call(e(), Y=None) == NULL and call(e(), X=None) == NULL
    assert call(e(activation=5)) == DTYPE and call(e(activation=-1)) == DTYPE
    assert call(e(bias=GOOD, bias_dtype=3)) == DTYPE and call(e(bias=GOOD, bias_dtype=-1)) == DTYPE
    assert call(e(residual=GOOD, ldr=255)) == SHAPE and call(e(residual=OTHER, ldr=264)) == SHAPE      # too short; in place with other rows
    assert call(e(residual=GOOD + 1, ldr=256)) == ALIGN and call(e(row_scale=GOOD + 2)) == ALIGN and call(e(col_scale=GOOD + 1)) == ALIGN
    assert call(e(bias=GOOD + 1, bias_dtype=BF16)) == ALIGN and call(e(bias=GOOD + 2, bias_dtype=F32)) == ALIGN
    assert call(e(residual=GOOD + 2, ldr=256), yt=F32) == ALIGN
    assert call(e(), ldy=255) == SHAPE and call(e(), yt=E4M3) == DTYPE
    assert call(e(), M=-1) == SHAPE
    if name == "combine":
        assert call(e(), P=3) == SHARDS and call(e(), P=128) == SHARDS and call(e(), X=GOOD + 8) == ALIGN
    else:
        assert call(e(), K=500) == SHAPE and call(e(), X=GOOD + 2) == ALIGN and call(e(), xt=F32) == DTYPE
        assert call(e(), K=4096, leaf=256, ldx=4096, ldw=4096, ldxs=128, ldws=128) in (WORKSPACE,)      # a K split without room for its planes


def test_output_types(tb):
    c = calls(tb)
    e = ends(tb)
    for name in ("fp8", "mx", "combine"):
        assert c[name](e, M=0, yt=F16) == OK and c[name](e, M=0, yt=F32) == OK
    assert c["gemm"](e, M=0, yt=F16) == DTYPE and c["gemm"](e, M=0, yt=F32) == OK
    assert tb.lib().tbik_gemm_fp8(GOOD, 512, GOOD, 512, GOOD, 256, F16, E4M3, 0, 256, 512, 128, 1, None, 0, None) == DTYPE     # as before


def rows_calls(tb):
    L = tb.lib()
    good = dict(x=GOOD, ldx=256, P=2, r=OTHER, ldr=256, w=GOOD, h=OTHER, ldh=256, q=GOOD, ldq=256, s=GOOD, lds=8, t=BF16, qt=E4M3, M=4, H=256)

    def norm(micro, **kw):
        a = dict(good, **kw)
        f = L.tbik_rmsnorm_mxfp8 if micro else L.tbik_rmsnorm_fp8
        return f(a["x"], a["ldx"], a["r"], a["ldr"], a["w"], 1e-6, a["h"], a["ldh"], a["q"], a["ldq"], a["s"], *([a["lds"]] if micro else []), a["t"], a["qt"], a["M"], a["H"], None)

    def tail(micro, **kw):
        a = dict(good, **kw)
        f = L.tbik_combine_residual_rmsnorm_mxfp8 if micro else L.tbik_combine_residual_rmsnorm_fp8
        return f(a["x"], a["P"], a["r"], a["ldr"], a["w"], 1e-6, a["h"], a["ldh"], a["q"], a["ldq"], a["s"], *([a["lds"]] if micro else []), a["t"], a["qt"], a["M"], a["H"], None)

    def silu(micro, **kw):
        a = dict(good, **kw)
        f = L.tbik_silu_mul_mxfp8 if micro else L.tbik_silu_mul_fp8
        return f(a["x"], a["ldx"], a["r"], a["ldr"], a["q"], a["ldq"], a["s"], *([a["lds"]] if micro else []), a["t"], a["qt"], a["M"], a["H"], None)

    return dict(norm=norm, tail=tail, silu=silu)


@pytest.mark.parametrize("micro", [False, True])
@pytest.mark.parametrize("name", ["norm", "tail", "silu"])
def test_8bit_output_refusals(tb, name, micro):
    call = lambda **kw: rows_calls(tb)[name](micro, **kw)
    assert call(M=0) == OK and call(M=-1) == SHAPE
    assert call(t=F32) == DTYPE and call(qt=BF16) == DTYPE
    assert call(x=None) == NULL and call(q=None) == NULL and call(s=None) == NULL and call(r=None) == NULL
    assert call(H=252) == SHAPE and call(H=65544 if not micro else 65568) == SHAPE
    assert call(ldq=248) == SHAPE and call(ldr=248) == SHAPE
    assert call(q=GOOD + 4) == ALIGN and call(ldq=260) == ALIGN and call(x=GOOD + 8) == ALIGN and call(r=OTHER + 8) == ALIGN and call(ldr=260, h=OTHER + 65536) == ALIGN
    if micro:
        assert call(lds=7) == SHAPE and call(H=248) == SHAPE          # whole blocks of 32
    else:
        assert call(s=GOOD + 2) == ALIGN
    if name != "tail":
        assert call(ldx=248) == SHAPE and call(ldx=260) == ALIGN
    if name == "silu":
        assert call(H=0) == OK
        return
    assert call(H=0) == SHAPE and call(w=None) == NULL and call(h=None) == NULL and call(w=GOOD + 8) == ALIGN
    assert call(h=OTHER + 8) == ALIGN and call(ldh=248) == SHAPE and call(ldh=264) == SHAPE      # in place with other rows
    if name == "norm":
        assert call(r=None, h=None, M=0) == OK and call(h=GOOD, ldh=264) == SHAPE
    else:
        assert call(P=3) == SHARDS and call(P=32) == UNSUPPORTED and call(P=0) == SHARDS


def test_the_binding_refuses_other_tensors(tb):
    """On the CPU: what is wrong with the arguments is said before a device pointer is taken."""
    X, W = torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(64, 32, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        tb.tbik_gemm_epilogue(X, W, 64)                                             # not on a GPU
    parts = torch.zeros(2, 4, 32)
    f = lambda **kw: tb._epilogue(4, 32, torch.bfloat16, **dict(dict(row_scale=None, col_scale=None, bias=None, activation=None, residual=None), **kw))
    assert f().activation == 0 and f(activation="gelu").activation == 3
    for bad in (dict(activation="tanh"), dict(bias=torch.zeros(31)), dict(bias=torch.zeros(64)[::2]), dict(row_scale=torch.zeros(32)), dict(col_scale=torch.zeros(4)),
                dict(residual=torch.zeros(4, 32))):
        with pytest.raises(ValueError):
            f(**bad)
    for bad in (dict(bias=torch.zeros(32, dtype=torch.float64)), dict(col_scale=torch.zeros(32, dtype=torch.bfloat16))):
        with pytest.raises(TypeError):
            f(**bad)
    with pytest.raises(ValueError):
        tb.tbik_silu_mul_fp8(X, X)
    with pytest.raises(AssertionError):
        tb.tbik_rmsnorm_fp8(parts, torch.ones(32))
    with pytest.raises(ValueError):
        tb._eight_bit_out(X, 4, 64, False, "e3m4", None, None)
