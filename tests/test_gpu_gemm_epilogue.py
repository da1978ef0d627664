"""Matrix products with an epilogue: scales, bias, activation, residual, one rounding.

The contract makes most of it a bit comparison: an epilogue without an activation is the fp32 output of the product without one
(tbik_gemm and its forms, tested on their own), then torch's fp32 products and sums in the stated order and one rounding; with
one, the same around the activation's fp32 value, which a call with fp32 output gives.  Only that value has a tolerance, derived in
eight_bit_reference.act_tolerance, plus 2^-100 where exponentials leave the normal range.  Every kernel an output can end in is
reached (the shapes assert which), and every one must give the bits of tbik_tree_combine_epilogue on the shards' partial sums.
"""
import numpy as np
import pytest
import torch

import eight_bit_reference as ref
from paper_2511_17826_amd import binding as tb

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
ACTS = [None, "relu", "silu", "gelu", "gelu_tanh"]


def bits(t):
    return t.contiguous().view(torch.int32 if t.dtype == torch.float32 else torch.int16)


def same(a, b):
    return a.dtype == b.dtype and a.shape == b.shape and torch.equal(bits(a), bits(b))


def operands(kind, M, K, N, seed):
    """(product(leaf, g, **kw) with fp32 output, partials(leaf, g, P), with_epilogue(leaf, g, **kw)) of random operands."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    X, W = torch.randn((M, K), generator=g, device="cuda"), torch.randn((K, N), generator=g, device="cuda") * 0.05
    if kind in ("bf16", "fp16"):
        X, W = X.to(TYPES[kind]), W.to(TYPES[kind])
        f, p = (tb.tbik_gemm, tb.tbik_gemm_shard_partials) if kind == "bf16" else (tb.tbik_gemm_f16, tb.tbik_gemm_shard_partials_f16)
        return (lambda leaf, k_first: f(X, W, leaf, k_first, out_dtype=torch.float32), lambda leaf, k_first, P: p(X, W, leaf, k_first, P),
                lambda leaf, k_first, **kw: tb.tbik_gemm_epilogue(X, W, leaf, k_first, **kw))
    fmt = kind[-4:]
    q = lambda t: t.to(ref.TORCH8[fmt]).view(torch.uint8)
    X8, W8 = q(X), q((W * 16).t().contiguous())
    if kind.startswith("fp8"):
        return (lambda leaf, k_first: tb.tbik_gemm_fp8(X8, W8, leaf, k_first, fmt, out_dtype=torch.float32),
                lambda leaf, k_first, P: tb.tbik_gemm_shard_partials_fp8(X8, W8, leaf, k_first, P, fmt),
                lambda leaf, k_first, **kw: tb.tbik_gemm_fp8_epilogue(X8, W8, leaf, k_first, fmt, **kw))
    Xs = torch.randint(124, 131, (M, K // 32), generator=g, device="cuda", dtype=torch.uint8)
    Ws = torch.randint(121, 127, (N, K // 32), generator=g, device="cuda", dtype=torch.uint8)
    return (lambda leaf, k_first: tb.tbik_gemm_mxfp8(X8, Xs, W8, Ws, leaf, k_first, fmt, out_dtype=torch.float32),
            lambda leaf, k_first, P: tb.tbik_gemm_shard_partials_mxfp8(X8, Xs, W8, Ws, leaf, k_first, P, fmt),
            lambda leaf, k_first, **kw: tb.tbik_gemm_mxfp8_epilogue(X8, Xs, W8, Ws, leaf, k_first, fmt, **kw))


def parts_of_an_epilogue(M, N, out, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")
    return dict(row_scale=r(M).abs() + 0.1, col_scale=r(N).abs() + 0.1), r(N), (2 * r(M, N)).to(out)


def composed(t, out, scales, bias, act32, residual):
    """The stated steps in torch, one fp32 operation each.  act32: the activation's fp32 value, or None."""
    if scales:
        t = t * scales["row_scale"][:, None] * scales["col_scale"][None, :]
    if bias is not None:
        t = t + bias.float()
    if act32 is not None:
        t = act32
    if residual is not None:
        t = t + residual.float()
    return t.to(out)


# (kind, M, K, N, leaf, k_first, route): the last is what tbik_gemm_route must say, or None where it cannot (strides, forced variants)
SHAPES = [
    ("bf16", 1, 4096, 512, 256, 1, [(1, "tiles", 32, 16)]),                    # a K split
    ("fp16", 40, 512, 33024, 512, 1, [(40, "tiles", 64, 1)]),
    ("bf16", 20, 512, 32896, 512, 1, [(20, "tiles", 32, 1)]),
    ("fp16", 80, 512, 32776, 256, 1, [(80, "tiles", 96, 1)]),                  # the last columns not a whole tile
    ("bf16", 600, 256, 8192, 128, 1, [(600, "tiles", 128, 1)]),                # the last row tile ragged
    ("fp16", 1024, 256, 4096, 64, 1, [(1024, "tiles", 128, 1)]),
    ("bf16", 1100, 4096, 4096, 256, 1, [(1024, "tiles", 128, 1), (76, "tiles", 64, 4)]),      # two pieces, the second split
    ("bf16", 33, 256, 104, 16, 1, [(33, "reference", 0, 0)]),
    ("fp8 e4m3", 5, 4096, 512, 256, 1, [(5, "slices", 0, 0)]),
    ("fp8 e5m2", 31, 2048, 520, 256, 1, [(31, "slices", 0, 0)]),
    ("fp8 e4m3", 600, 256, 8192, 128, 1, [(600, "tiles", 128, 1)]),
    ("fp8 e5m2", 1030, 4096, 4096, 256, 1, [(1024, "tiles", 128, 1), (6, "slices", 0, 0)]),
    ("fp8 e4m3", 100, 4096, 4096, 256, 1, [(100, "tiles", 32, 1)]),
    ("fp8 e4m3", 50, 192, 72, 64, 3, [(50, "reference", 0, 0)]),
    ("fp8 e5m2", 200, 4096, 640, 256, 1, None),
    ("mx e4m3", 7, 4096, 512, 256, 1, [(7, "slices", 0, 0)]),
    ("mx e5m2", 600, 256, 8192, 128, 1, [(600, "tiles", 128, 1)]),
    ("mx e4m3", 300, 4096, 1000, 256, 1, None),
    ("mx e4m3", 50, 192, 72, 64, 3, [(50, "reference", 0, 0)]),
    # More tiles than compute units with one to four stages each, and rows or scales that end inside 16 bytes: the epilogue's operands
    # lie several tiles ahead in the ring of every tile height.
    ("bf16", 603, 64, 8192, 64, 1, [(603, "tiles", 128, 1)]),
    ("fp16", 3, 64, 32896, 64, 1, [(3, "tiles", 32, 1)]),
    ("bf16", 4095, 128, 4096, 128, 1, [(4095, "tiles", 128, 1)]),
    ("fp8 e4m3", 603, 128, 8192, 128, 1, [(603, "tiles", 128, 1)]),
    ("fp8 e5m2", 3, 256, 16640, 128, 1, [(3, "tiles", 32, 1)]),
    ("fp8 e4m3", 50, 512, 33024, 128, 1, [(50, "tiles", 64, 1)]),
    ("mx e4m3", 1031, 128, 8192, 128, 1, [(1031, "tiles", 128, 1)]),
    ("mx e4m3", 2, 256, 16640, 128, 1, [(2, "tiles", 32, 1)]),
    ("mx e5m2", 50, 512, 33024, 128, 1, [(50, "tiles", 64, 1)]),
]


def route_of(kind, M, N, K, leaf, g):
    return tb.gemm_route({"fp8 ": "fp8", "mx e": "mxfp8"}.get(kind[:4], kind), M, N, K, leaf, g)


@pytest.mark.parametrize("kind,M,K,N,leaf,g,route", SHAPES)
def test_the_epilogue_is_the_stated_steps(kind, M, K, N, leaf, g, route):
    got_route = route_of(kind, M, N, K, leaf, g)
    print(kind, M, K, N, got_route)
    if route is not None:
        assert got_route == route
    product, partials, with_epilogue = operands(kind, M, K, N, M + N)
    t = product(leaf, g)
    outs = [kind, "fp32"] if kind in ("bf16", "fp16") else ["bf16", "fp32", "fp16"]
    for i, out in enumerate(outs):
        scales, bias32, residual = parts_of_an_epilogue(M, N, TYPES[out], M + i)
        bias = bias32.to(TYPES[("bf16", "fp32", "fp16")[(M + i) % 3]])
        call = lambda **kw: with_epilogue(leaf, g, out_dtype=TYPES[out], **kw)
        assert same(call(), composed(t, TYPES[out], None, None, None, None))
        assert same(call(bias=bias), composed(t, TYPES[out], None, bias, None, None))
        assert same(call(residual=residual), composed(t, TYPES[out], None, None, None, residual))
        assert same(call(bias=bias, residual=residual, **scales), composed(t, TYPES[out], scales, bias, None, residual))
        into = residual.clone()
        assert call(bias=bias, residual=into, out=into, **scales) is into and same(into, composed(t, TYPES[out], scales, bias, None, residual))
        act = ACTS[1 + (M + i) % 4]
        act32 = with_epilogue(leaf, g, out_dtype=torch.float32, bias=bias, activation=act, **scales)
        assert same(call(bias=bias, activation=act, residual=residual, **scales), composed(t, TYPES[out], scales, bias, act32, residual))
        assert same(call(bias=bias, activation=act, **scales), composed(t, TYPES[out], scales, bias, act32, None))
        P = min(K // (leaf * g), 4)
        parts = partials(leaf, g, P)
        assert same(tb.tbik_tree_combine_epilogue(parts, bias=bias, activation=act, residual=residual, out_dtype=TYPES[out], **scales),
                    call(bias=bias, activation=act, residual=residual, **scales))


@pytest.mark.parametrize("act", ACTS[1:])
def test_activations_against_64_bits(act):
    """Through the combine of one plane, whose input is the activation's argument: every binade from 2^-40 to 12, both signs."""
    v = torch.cat([torch.linspace(-12, 12, 40000), torch.exp2(torch.linspace(-40, 3.58, 6000)), -torch.exp2(torch.linspace(-40, 3.58, 6000)),
                   torch.tensor([0.0, -0.0, 30.0, -30.0, 100.0, -100.0, 1e30, -1e30])])
    y = tb.tbik_tree_combine_epilogue(v.reshape(1, 1, -1).cuda(), activation=act, out_dtype=torch.float32).cpu().numpy()[0].astype(np.float64)
    x = v.numpy().astype(np.float64)
    want = ref.act64(x, act)
    wide = np.abs(x) > 12                                         # saturated: the argument, or zero
    assert np.all(np.abs(y - want)[~wide] <= (ref.act_tolerance(x, act) * np.abs(want) + 2.0 ** -100)[~wide])
    assert np.all(np.abs(y - want)[wide] <= 2.0 ** -22 * np.abs(x * (x > 0))[wide] + 2.0 ** -30)
    special = torch.tensor([float("nan"), float("inf")]).reshape(1, 1, 2).cuda()
    s = tb.tbik_tree_combine_epilogue(special, activation=act, out_dtype=torch.float32).cpu()
    assert torch.isnan(s[0, 0]) and s[0, 1] == float("inf")


@pytest.mark.parametrize("kind", ["bf16", "fp16", "fp8 e4m3", "mx e4m3"])
def test_against_64_bits(kind):
    """The whole operator against its definition: products of K = 1024 terms, within 2 (256 + 8) u of the sum of magnitudes (the stated
    order's bound; 8-bit operands lose up to 2^-13 of the largest product of eight in each of K / 8 groups), activation, one rounding."""
    M, K, N, leaf = 150, 1024, 264, 256
    g = torch.Generator(device="cuda").manual_seed(11)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")
    dt = TYPES.get(kind, torch.bfloat16)
    bias, residual, rs, cs = r(N), r(M, N).to(dt), r(M).abs() + 0.5, r(N).abs() + 0.5
    kw = dict(bias=bias, activation="gelu", residual=residual, row_scale=rs, col_scale=cs)
    if kind in ("bf16", "fp16"):
        X, W = r(M, K).to(dt), (0.05 * r(K, N)).to(dt)
        y = tb.tbik_gemm_epilogue(X, W, leaf, 1, **kw)
        x64, w64, loss = X.double(), W.double(), 2.0 ** -20
    else:
        X, Wt = (t.to(torch.float8_e4m3fn) for t in (r(M, K), r(N, K)))
        x64, w64, loss = X.double(), Wt.double().t(), 2.0 ** -12
        rs = rs * 0.05
        kw["row_scale"] = rs
        if kind == "fp8 e4m3":
            y = tb.tbik_gemm_fp8_epilogue(X, Wt, leaf, 1, **kw)
        else:
            Xs = torch.randint(125, 129, (M, K // 32), generator=g, device="cuda", dtype=torch.uint8)
            Ws = torch.randint(125, 129, (N, K // 32), generator=g, device="cuda", dtype=torch.uint8)
            y = tb.tbik_gemm_mxfp8_epilogue(X.view(torch.uint8), Xs, Wt.view(torch.uint8), Ws, leaf, 1, **kw)
            spread = lambda t: torch.exp2(t.double() - 127).repeat_interleave(32, dim=1)
            x64, w64 = x64 * spread(Xs), (Wt.double() * spread(Ws)).t()
    scale = rs.double()[:, None] * cs.double()
    w64 = w64.contiguous()
    v = (x64 @ w64) * scale + bias.double()
    off = (x64.abs() @ w64.abs()) * scale * (2 * 264 * 2.0 ** -24 + loss) + v.abs() * 2.0 ** -22
    want = (v.cpu().numpy() * __import__("scipy.special", fromlist=["ndtr"]).ndtr(v.cpu().numpy())) + residual.double().cpu().numpy()
    half = 2.0 ** (-8 if dt == torch.bfloat16 else -11)
    # |gelu'| <= 1.13; the activation's own error at |v| <= 12; half a step of the output
    bound = 1.13 * off.cpu().numpy() + 2.0 ** -16 * np.abs(v.cpu().numpy()) + half * np.abs(want) * 1.001 + 2.0 ** -20
    assert np.all(np.abs(y.double().cpu().numpy() - want) <= bound)


@pytest.mark.parametrize("variant", [tb.VARIANT_REFERENCE, tb.VARIANT_T128, tb.VARIANT_T64, tb.VARIANT_T32])
def test_every_16_bit_kernel(variant):
    M, K, N, leaf = 200, 2048, 328, 128
    product, _, with_epilogue = operands("bf16", M, K, N, 3)
    t = product(leaf, 1)
    scales, bias, residual = parts_of_an_epilogue(M, N, torch.bfloat16, 4)
    want = with_epilogue(leaf, 1, bias=bias, activation="gelu", residual=residual, **scales)
    want32 = with_epilogue(leaf, 1, bias=bias, out_dtype=torch.float32, **scales)
    assert same(want32, composed(t, torch.float32, scales, bias, None, None))
    tb.tbik_set_gemm_variant(variant)
    ws = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")
    assert same(with_epilogue(leaf, 1, bias=bias, activation="gelu", residual=residual, workspace=ws, **scales), want)
    assert same(with_epilogue(leaf, 1, bias=bias, out_dtype=torch.float32, workspace=ws, **scales), want32)


@pytest.mark.parametrize("kind", ["bf16", "fp8 e4m3", "mx e4m3"])
@pytest.mark.parametrize("M,N,K,leaf", [(300, 1024, 256, 128), (1, 512, 4096, 256), (9, 136, 1024, 256)])
def test_strides_and_unaligned_parts(kind, M, N, K, leaf):
    """Output and residual inside wider buffers, at odd addresses; bias and scales that start anywhere; nothing else is written."""
    _, _, with_epilogue = operands(kind, M, K, N, 8)
    scales, bias, residual = parts_of_an_epilogue(M, N, torch.bfloat16, 9)
    want = with_epilogue(leaf, 1, bias=bias.bfloat16(), activation="silu", residual=residual, **scales)
    for pad, at in ((8, 8), (3, 1), (5, 0), (24, 16)):
        buf = torch.full((M, N + 2 * pad), 3.0, dtype=torch.bfloat16, device="cuda")
        res = torch.full((M, N + 2 * pad + 1), 2.0, dtype=torch.bfloat16, device="cuda")
        res[:, at:at + N] = residual
        b = torch.zeros(N + 9, dtype=torch.bfloat16, device="cuda")[at % 8 + 1:][:N]
        b.copy_(bias)
        sc = {k: torch.zeros(len(v) + 4, device="cuda")[1:1 + len(v)].copy_(v) for k, v in scales.items()}
        out = buf[:, at:at + N]
        with_epilogue(leaf, 1, bias=b, activation="silu", residual=res[:, at:at + N], out=out, **sc)
        assert same(out, want)
        assert bool((buf[:, :at] == 3).all()) and bool((buf[:, at + N:] == 3).all())
        buf[:, at:at + N] = residual                                # in place in the wider buffer
        with_epilogue(leaf, 1, bias=b, activation="silu", residual=out, out=out, **sc)
        assert same(out, want) and bool((buf[:, :at] == 3).all()) and bool((buf[:, at + N:] == 3).all())


@pytest.mark.parametrize("ld", [2 ** 24 + 8, 2 ** 26])
def test_rows_of_output_and_residual_far_apart(ld):
    """Offsets past 32 bits, below and above the distance up to which a tile is stored 16 bytes at a time."""
    M, N, K, leaf = 150 if ld < 2 ** 25 else 40, 4096, 128, 128
    X, W = torch.randn(M, K, device="cuda").bfloat16(), torch.randn(K, N, device="cuda").bfloat16()
    res = torch.randn(M, N, device="cuda").bfloat16()
    want = tb.tbik_gemm_epilogue(X, W, leaf, 1, activation="relu", residual=res)
    far = torch.empty((M - 1) * ld + N, dtype=torch.bfloat16, device="cuda").as_strided((M, N), (ld, 1))
    far.copy_(res)
    tb.tbik_gemm_epilogue(X, W, leaf, 1, activation="relu", residual=far, out=far)
    assert same(far, want)
    far.copy_(res)
    parts = tb.tbik_gemm_shard_partials(X, W, leaf, 1, 1)
    tb.tbik_tree_combine_epilogue(parts, activation="relu", residual=far, out=far)
    assert same(far, want)


@pytest.mark.parametrize("kind", ["bf16", "fp8 e4m3", "mx e4m3"])
def test_residual_of_many_distant_rows_in_place(kind):
    """Offsets past 32 bits from one tile to another where a tile's residual is loaded ahead of its product; columns around it untouched."""
    M, N, K, leaf, ld = 1100, 8192, 256, 128, 2 ** 22 - 8
    product, _, call = operands(kind, M, K, N, 5)
    bias, res = torch.randn(N, device="cuda"), torch.randn(M, N, device="cuda").bfloat16()
    want = composed(product(leaf, 1), torch.bfloat16, None, bias, None, res)
    buf = torch.empty((M - 1) * ld + N + 16, dtype=torch.bfloat16, device="cuda")
    far, around = buf.as_strided((M, N), (ld, 1)), [buf.as_strided((M, 8), (ld, 1), N)]
    for b in around:
        b.fill_(3)
    far.copy_(res)
    call(leaf, 1, bias=bias, residual=far, out=far)
    assert same(far, want) and all(bool((b == 3).all()) for b in around)


@pytest.mark.parametrize("P", [1, 2, 4, 8, 16, 32, 64])
@pytest.mark.parametrize("M,N", [(3, 64), (5, 37), (1, 1), (130, 1028)])
def test_combine_with_an_epilogue(P, M, N):
    g = torch.Generator(device="cuda").manual_seed(P + M + N)
    parts = torch.randn((P, M, N), generator=g, device="cuda")
    t = tb.tbik_tree_combine(parts, out_dtype=torch.float32)
    for out in ("bf16", "fp16", "fp32"):
        scales, bias, residual = parts_of_an_epilogue(M, N, TYPES[out], P)
        assert same(tb.tbik_tree_combine_epilogue(parts, out_dtype=TYPES[out], bias=bias, residual=residual, **scales), composed(t, TYPES[out], scales, bias, None, residual))
        assert same(tb.tbik_tree_combine_epilogue(parts, out_dtype=TYPES[out]), t.to(TYPES[out]))
    assert tb.tbik_tree_combine_epilogue(parts[:, :0].contiguous(), bias=torch.zeros(N, device="cuda")).shape == (0, N)


def test_rows_do_not_depend_on_the_batch():
    """A row alone, in a batch that splits K, in one that does not: the same bits; NaN in a row stays in it."""
    K, N, leaf = 4096, 4096, 256
    g = torch.Generator(device="cuda").manual_seed(2)
    X, W = torch.randn((700, K), generator=g, device="cuda").bfloat16(), (0.02 * torch.randn((K, N), generator=g, device="cuda")).bfloat16()
    bias, res = torch.randn(N, generator=g, device="cuda"), torch.randn((700, N), generator=g, device="cuda").bfloat16()
    full = tb.tbik_gemm_epilogue(X, W, leaf, 1, bias=bias, activation="gelu", residual=res)
    for rows in ([5], [699, 0, 3], list(range(64, 164))):
        assert same(tb.tbik_gemm_epilogue(X[rows].contiguous(), W, leaf, 1, bias=bias, activation="gelu", residual=res[rows].contiguous()), full[rows])
    X[7, 100] = float("nan")
    res[9, 8] = float("inf")
    y = tb.tbik_gemm_epilogue(X, W, leaf, 1, bias=bias, activation="gelu", residual=res)
    keep = [i for i in range(700) if i not in (7, 9)]
    assert bool(torch.isnan(y[7]).all()) and float(y[9, 8]) == float("inf") and same(y[keep], full[keep])


def test_refusals_on_the_gpu():
    X, W = torch.zeros((8, 256), dtype=torch.bfloat16, device="cuda"), torch.zeros((256, 64), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError):
        tb.tbik_gemm_epilogue(X, W, 128, 1, residual=torch.zeros((8, 64), device="cuda"))            # not of the output's type
    with pytest.raises(ValueError):
        tb.tbik_gemm_epilogue(X, W, 128, 1, bias=torch.zeros(64))                                     # on the CPU
    with pytest.raises(tb.TbikError):
        tb.tbik_gemm_epilogue(X, W, 128, 1, out_dtype=torch.float16)
    need = tb.gemm_16bit_workspace_bytes(8, 64, 256, 128, 1)
    assert need > 0
    with pytest.raises(tb.TbikError):
        tb.tbik_gemm_epilogue(X, W, 128, 1, workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))
    assert tb.tbik_gemm_epilogue(X[:0], W, 128, 1).shape == (0, 64)
