"""RMSNorm (with the residual's addition, from rows or from shards' partial sums) and the gated activation with 8-bit outputs.

Norms: the fp32 value behind an output is fixed by the contract (TreeSum, IEEE square root and division), so patterns, scales and
the hidden state are compared bit for bit with the steps in numpy, and hidden with the 16-bit calls.  Against the 64-bit
definition: TreeSum of n squares adds at most 8 + log2(n / 8) roundings of relative size u = 2^-24 each to a sum of positive
numbers, half of that reaches r = 1 / sqrt(...), which adds 4 more (division, eps, square root, reciprocal), two products: for
65536 columns (21 / 2 + 6) u < 2^-19 =: D.  Then the row scale is within 2^-19 + 2 u of the exact one, and a value within D, two roundings of the factor and
half a step of the 8-bit format: 2^-4 of the value (E5M2: 2^-3), or half the smallest subnormal step 2^-10 (2^-17) of the scale.
Activation: silu_mul's exponential and reciprocal are the hardware's, so its fp32 value is only known to
(2 |gate| + 8) u (eight_bit_reference.act_tolerance and one more product): a pattern lies between the roundings of the interval's ends.
"""
import numpy as np
import pytest
import torch

import eight_bit_reference as ref
import gpu_util as gu
from paper_2511_17826_amd import binding as tb

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
HALF_STEP = {"e4m3": (2.0 ** -4, 2.0 ** -10), "e5m2": (2.0 ** -3, 2.0 ** -17)}
EPS = 1e-6


def rows(seed, M, H, dtype, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((M, H), generator=g) * scale
    x[:, ::7] *= 8.0
    return x.to(dtype)


def host32(t):
    return t.float().cpu().numpy()


def norm(micro, x, w, residual=None, fmt="e4m3", **kw):
    return (tb.tbik_rmsnorm_mxfp8 if micro else tb.tbik_rmsnorm_fp8)(x, w, EPS, residual=residual, fmt=fmt, **kw)


def check_rows(q, scale, v32, v64, micro, fmt):
    q, scale = q.cpu().numpy(), scale.cpu().numpy()
    want_q, want_s = (ref.micro_scaled if micro else ref.row_scaled)(v32, fmt)
    assert np.array_equal(scale, want_s)
    assert ref.same_patterns(q, want_q, fmt)
    if v64 is None:
        return
    if micro:
        s64 = np.repeat(np.exp2(scale.astype(np.float64) - 127), 32, axis=1)
    else:
        amax = np.abs(v64).max(axis=1)
        exact = np.where(amax > 0, amax / ref.LARGEST[fmt], 1.0)
        assert np.all(np.abs(scale - exact) <= (2.0 ** -19 + 2.0 ** -23) * exact)
        s64 = scale.astype(np.float64)[:, None]
    rel, sub = HALF_STEP[fmt]
    err = np.abs(ref.value_of_8(q, fmt) * s64 - v64)
    assert np.all(err <= np.abs(v64) * (rel + 2.0 ** -18) + sub * s64)


SHAPES = [(1, 32), (1, 4096), (3, 8), (5, 512), (2, 520), (7, 1056), (4, 4104), (33, 5120), (2, 8192), (1, 8224), (3, 16416), (2, 32768), (1, 65536), (2, 40000),
          (1023, 256), (1024, 1032), (1025, 1024), (1030, 96), (1100, 4096), (1027, 5120), (1024, 8192), (1025, 8224)]


@pytest.mark.parametrize("micro", [False, True])
@pytest.mark.parametrize("M,H", SHAPES)
def test_norm_of_rows(M, H, micro):
    if micro and H % 32:
        H = (H + 31) // 32 * 32
    dtype, fmt = ("bf16", "fp16")[(M + H // 8) % 2], ("e4m3", "e5m2")[(M + H // 32) % 2]
    x, r, w = rows(M + H, M, H, TYPES[dtype]), rows(M + H + 1, M, H, TYPES[dtype]), (1 + 0.1 * torch.randn(H)).to(TYPES[dtype])
    dx, dr, dw = x.cuda(), r.cuda(), w.cuda()
    for residual in (None, dr):
        hidden, q, scale = norm(micro, dx, dw, residual, fmt)
        torch.cuda.synchronize()
        h = host32(x) if residual is None else host32((x.float() + r.float()).to(TYPES[dtype]))
        assert (hidden is None) == (residual is None)
        if hidden is not None:
            assert np.array_equal(host32(hidden), h)
        h64 = h.astype(np.float64)
        v64 = h64 / np.sqrt((h64 ** 2).mean(axis=1, keepdims=True) + np.float64(np.float32(EPS))) * host32(w).astype(np.float64)[None, :]
        check_rows(q, scale, ref.normed32(h, host32(w), EPS), v64, micro, fmt)


@pytest.mark.parametrize("micro", [False, True])
@pytest.mark.parametrize("P,M,H", [(1, 3, 4096), (2, 1, 512), (4, 5, 5120), (8, 2, 1056), (16, 1030, 64), (4, 1025, 4096), (2, 2, 20480)])
def test_norm_of_partial_sums(P, M, H, micro):
    """hidden is tbik_combine_residual_rmsnorm's, the 8-bit output that of the numpy steps on it."""
    dtype, fmt = ("bf16", "fp16")[P % 3 % 2], ("e4m3", "e5m2")[M % 2]
    g = torch.Generator().manual_seed(P + M + H)
    parts = torch.randn((P, M, H), generator=g).cuda()
    r, w = rows(H, M, H, TYPES[dtype]).cuda(), (1 + 0.1 * torch.randn(H, generator=g)).to(TYPES[dtype]).cuda()
    want, _ = (tb.tbik_combine_residual_rmsnorm if dtype == "bf16" else tb.tbik_combine_residual_rmsnorm_f16)(parts, r, w, EPS)
    f = tb.tbik_combine_residual_rmsnorm_mxfp8 if micro else tb.tbik_combine_residual_rmsnorm_fp8
    hidden, q, scale = f(parts, r, w, EPS, fmt=fmt)
    assert torch.equal(hidden.view(torch.int16), want.view(torch.int16))
    check_rows(q, scale, ref.normed32(host32(hidden), host32(w), EPS), None, micro, fmt)
    y = tb.tbik_tree_combine(parts, out_dtype=TYPES[dtype])                     # the same through the sum of the shards
    h2, q2, s2 = norm(micro, y, w, r, fmt)
    assert torch.equal(h2.view(torch.int16), hidden.view(torch.int16)) and torch.equal(q2, q) and torch.equal(s2, scale)


@pytest.mark.parametrize("micro", [False, True])
def test_strides_in_place_and_batches(micro):
    """Rows far apart, hidden in place of x or of the residual, unused columns left alone, a row alone = the row in a batch."""
    M, H = 1029, 1024
    x, r, w = rows(1, M, H, torch.bfloat16).cuda(), rows(2, M, H, torch.bfloat16).cuda(), torch.ones(H, dtype=torch.bfloat16).cuda()
    hidden, q, scale = norm(micro, x, w, r)
    xs, rs = torch.full((M, H + 24), 7.0, dtype=torch.bfloat16, device="cuda"), torch.full((M, H + 8), 5.0, dtype=torch.bfloat16, device="cuda")
    qs = torch.full((M, H + 16), 9, dtype=torch.uint8, device="cuda")
    ss = torch.full((M, H // 32 + 3), 9, dtype=torch.uint8, device="cuda")
    xs[:, 8:8 + H], rs[:, :H] = x, r
    for into in (xs[:, 8:8 + H], rs[:, :H]):
        kw = dict(hidden=into, out=qs[:, :H])
        if micro:
            kw["scale"] = ss[:, 1:1 + H // 32]
        xs[:, 8:8 + H], rs[:, :H] = x, r
        h2, q2, s2 = norm(micro, xs[:, 8:8 + H], w, rs[:, :H], **kw)
        assert h2.data_ptr() == into.data_ptr() and torch.equal(h2, hidden) and torch.equal(q2, q) and torch.equal(s2, scale)
        assert bool((xs[:, :8] == 7).all()) and bool((xs[:, 8 + H:] == 7).all()) and bool((rs[:, H:] == 5).all()) and bool((qs[:, H:] == 9).all())
        if micro:
            assert bool((ss[:, 0] == 9).all()) and bool((ss[:, 1 + H // 32:] == 9).all())
    for rows_ in ([17], [0, 5, 1028], list(range(100, 900))):                   # other launches, same bits
        h3, q3, s3 = norm(micro, x[rows_].contiguous(), w, r[rows_].contiguous())
        assert torch.equal(h3, hidden[rows_]) and torch.equal(q3, q[rows_]) and torch.equal(s3, scale[rows_])
    assert norm(micro, x[:0], w, r[:0])[1].shape == (0, H)


@pytest.mark.parametrize("micro", [False, True])
@pytest.mark.parametrize("M", [3, 1024])
def test_rows_further_apart_than_32_bits(micro, M):
    """The last row lies more than 2^31 elements behind the first."""
    H = 256
    ld = ((2 ** 31 + 2 ** 20) // (M - 1) + 7) // 8 * 8
    x = torch.empty((M - 1) * ld + H, dtype=torch.bfloat16, device="cuda").as_strided((M, H), (ld, 1))
    x.copy_(rows(3, M, H, torch.bfloat16))
    w = torch.ones(H, dtype=torch.bfloat16, device="cuda")
    q8 = torch.empty((M - 1) * ld + H, dtype=torch.uint8, device="cuda").as_strided((M, H), (ld, 1))
    want = norm(micro, x.contiguous(), w)
    got = norm(micro, x, w, out=q8)
    assert torch.equal(got[1], want[1]) and torch.equal(got[2], want[2])


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
def test_special_rows(fmt):
    """Zeros, one element, subnormal weights, ties of the 8-bit rounding, NaN and infinity in one row: the others are as without."""
    H = 64
    x = rows(5, 8, H, torch.bfloat16)
    x[1] = 0
    x[2] = 0
    x[2, 33] = 3.0
    x[4, 5] = float("nan")
    x[5, 40] = float("inf")
    w = torch.ones(H, dtype=torch.bfloat16)
    w[::3] = 2.0 ** -130                                       # a bf16 subnormal
    for micro in (False, True):
        _, q, s = norm(micro, x.cuda(), w.cuda(), fmt=fmt)
        v = ref.normed32(host32(x), host32(w), EPS)
        check_rows(q, s, v, None, micro, fmt)
        clean = [0, 1, 2, 3, 6, 7]
        _, q2, s2 = norm(micro, x[clean].cuda(), w.cuda(), fmt=fmt)
        assert torch.equal(q2, q[clean]) and torch.equal(s2, s[clean])
    # values that fall between two patterns: x of constant magnitude 1 gives r = 1 (eps = 0), the weight picks the values
    x1 = torch.ones((1, 512), dtype=torch.bfloat16)
    w1 = torch.from_numpy((np.arange(512) / 2.0).astype(np.float32)).to(torch.bfloat16)
    _, q, s = tb.tbik_rmsnorm_mxfp8(x1.cuda(), w1.cuda(), 0.0, fmt=fmt)
    check_rows(q, s, host32(w1)[None, :], None, True, fmt)


@pytest.mark.parametrize("micro", [False, True])
@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("M,I,pad", [(1, 32, 0), (3, 4096, 0), (77, 12288, 0), (5, 4128, 8), (2, 16416, 0), (300, 1024, 24), (1, 65536, 0), (2, 16384, 8)])
def test_silu_mul(dtype, fmt, micro, M, I, pad):
    g = torch.Generator().manual_seed(M + I)
    buf = (torch.randn((M, 2 * I + pad), generator=g) * 3).to(TYPES[dtype])
    buf[0, 0], buf[0, I] = -30.0, 2.0
    dbuf = buf.cuda()
    gate, up = dbuf[:, :I], dbuf[:, I:2 * I]
    q, scale = (tb.tbik_silu_mul_mxfp8 if micro else tb.tbik_silu_mul_fp8)(gate, up, fmt=fmt)
    q, scale = q.cpu().numpy(), scale.cpu().numpy()
    g64, u64 = buf[:, :I].double().numpy(), buf[:, I:2 * I].double().numpy()
    v64 = ref.act64(g64, "silu") * u64
    tol = (2 * np.abs(g64) + 8) * 2.0 ** -24
    amax = np.abs(v64).max(axis=1)
    if micro:
        blocks = np.abs(v64).reshape(M, I // 32, 32).max(axis=2)
        up_to = lambda a: np.ceil(np.log2(a)) - ref.EMAX[fmt] + 127
        worst = tol.max()
        assert np.all((scale >= up_to(blocks * (1 - worst))) & (scale <= up_to(blocks * (1 + worst))))
        s64 = np.repeat(np.exp2(scale.astype(np.float64) - 127), 32, axis=1)
        factor_tol = 2.0 ** -24                                 # fp32 ends of the interval below
    else:
        assert np.all(np.abs(scale - amax / ref.LARGEST[fmt]) <= (tol.max() + 2.0 ** -24) * amax / ref.LARGEST[fmt])
        s64 = scale.astype(np.float64)[:, None]
        factor_tol = 3 * 2.0 ** -24                             # the reciprocal, the product; fp32 ends of the interval below
    lo, hi = np.abs(v64) / s64 * (1 - tol - factor_tol), np.abs(v64) / s64 * (1 + tol + factor_tol)
    got = np.abs(ref.value_of_8(q, fmt))
    r8 = lambda a: ref.value_of_8(torch.from_numpy(np.minimum(a, ref.LARGEST[fmt])).float().to(ref.TORCH8[fmt]).view(torch.uint8).numpy(), fmt)
    assert np.all((got >= r8(lo)) & (got <= r8(hi)))
    signs = got > 0
    assert np.array_equal(np.signbit(ref.value_of_8(q, fmt))[signs], np.signbit(v64)[signs])
    assert np.array_equal(q[:1], (tb.tbik_silu_mul_mxfp8 if micro else tb.tbik_silu_mul_fp8)(gate[:1], up[:1], fmt=fmt)[0].cpu().numpy())


def test_silu_mul_of_infinities():
    """Exact cases: gates past 32 are their own activation; an infinity and a NaN stay in their element (and their row's scale)."""
    gate = torch.full((3, 64), 64.0, dtype=torch.bfloat16)
    up = (torch.arange(192).reshape(3, 64) % 13 - 6).to(torch.bfloat16)
    gate[1, 3], up[1, 3] = float("inf"), 1.0
    up[2, 40] = float("nan")
    v = (gate.float() * up.float()).numpy()
    for fmt in ("e4m3", "e5m2"):
        for micro in (False, True):
            q, s = (tb.tbik_silu_mul_mxfp8 if micro else tb.tbik_silu_mul_fp8)(gate.cuda(), up.cuda(), fmt=fmt)
            check_rows(q, s, v, None, micro, fmt)


def test_another_stream():
    """The calls take the current stream: after a producer on it, before a consumer on it, with no synchronisation between."""
    s = torch.cuda.Stream()
    x, w = rows(9, 64, 4096, torch.bfloat16).cuda(), torch.ones(4096, dtype=torch.bfloat16, device="cuda")
    want = norm(True, x + x, w)
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        y = x + x
        got = norm(True, y, w)
        copy = got[1].clone()
    s.synchronize()
    assert torch.equal(copy, want[1]) and torch.equal(got[2], want[2])


@pytest.mark.parametrize("name", ["norm", "tail", "silu"])
def test_more_rows_than_threads_of_a_grid(name):
    """2^32 threads are a grid's limit: 17 million rows of 256 of them, 68 million of 64.  The last rows against a call of their own, and
    the rows around every 2^21."""
    M, H = (17 if name == "silu" else 68) * 10 ** 6 + 5, 8
    x = torch.randint(-30000, 16000, (M, H), dtype=torch.int16, device="cuda").view(torch.bfloat16) if name != "tail" else torch.rand((2, M, H), device="cuda")
    w = torch.full((H,), 0.75, dtype=torch.bfloat16, device="cuda")
    calls = {"norm": lambda t: tb.tbik_rmsnorm_fp8(t, w), "tail": lambda t: tb.tbik_combine_residual_rmsnorm_fp8(t, torch.ones_like(t[0], dtype=torch.bfloat16), w),
             "silu": lambda t: tb.tbik_silu_mul_fp8(t, t)}
    q, scale = calls[name](x)[-2:]
    for m in (0, 1 << 21, 5 << 21, 8 << 21, M):
        rows = slice(max(m - 70, 0), min(m + 70, M))
        part = x[rows] if name != "tail" else x[:, rows].contiguous()
        q1, s1 = calls[name](part)[-2:]
        assert torch.equal(q[rows], q1) and torch.equal(scale[rows].view(torch.int32), s1.view(torch.int32)), m
