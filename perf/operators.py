"""Performance cases of the operators around the 8-bit products of a decoder layer, and of the products' epilogues.

Three operators, as a layer uses them one after the other: RMSNorm with the residual's addition whose output is 8-bit with
scales (from 16-bit rows, or from the fp32 partial sums of a tensor-parallel layer); the gated activation with an 8-bit output;
matrix products whose epilogue applies the operands' scales, a bias, an activation and a residual (on 16-bit, 8-bit and
microscaled operands, and on the partial sums of the shards).

Shapes are those of the layers that the tests and the benchmark use: an 8B-class layer (hidden 4096, MLP 12288 or 14336, leaf
256) and a 32B-class layer (hidden 5120, MLP 25600, leaf 128).  Batches go from one token to a prefill and are ragged, as
batches of requests are.  8-bit outputs are compared as the numbers their patterns stand for (torch's float8 types).
"""
import math

import torch

own = False
DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
FP8 = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
LARGEST = {"e4m3": 448.0, "e5m2": 57344.0}
TOP = {"e4m3": 8, "e5m2": 15}                     # exponent of the largest binade
STEP = {"e4m3": (3, -6), "e5m2": (2, -14)}        # fraction bits, exponent of the smallest normal number
EPS = 1e-6

# (K, N, leaf, k_first) of the layers' products
GEMMS_16 = [(4096, 4096, 256, 1), (12288, 4096, 256, 3), (14336, 4096, 256, 7), (4096, 6144, 256, 1), (4096, 12288, 256, 1),
            (5120, 5120, 128, 5), (5120, 7168, 128, 5), (25600, 5120, 128, 25)]
GEMMS_8 = [(4096, 4096, 256, 1), (12288, 4096, 256, 3), (4096, 6144, 256, 1), (4096, 12288, 256, 1), (14336, 4096, 256, 7)]


def listed():
    return [
        # The norm before a block of one decoded token: latency of the smallest call.
        dict(name="norm_mx_one_token", kind="norm", scheme="mx", fmt="e4m3", dtype="bf16", M=1, H=4096, residual=True),
        # The norm of a long prefill with a scale per row, 32B-class hidden size.
        dict(name="norm_fp8_prefill", kind="norm", scheme="fp8", fmt="e4m3", dtype="bf16", M=8191, H=5120, residual=True),
        # What follows a row-parallel layer of a tensor-parallel group of four: shards' sums, residual, norm, 8 bits.
        dict(name="tail_mx_tp4", kind="tail", scheme="mx", fmt="e5m2", dtype="fp16", P=4, M=1003, H=4096),
        # The MLP's activation of a decode batch of odd size, a scale per row.
        dict(name="silu_fp8_decode", kind="silu", scheme="fp8", fmt="e4m3", dtype="bf16", M=77, I=12288),
        # The MLP's activation of a prefill, microscaled.
        dict(name="silu_mx_prefill", kind="silu", scheme="mx", fmt="e4m3", dtype="bf16", M=4096, I=14336),
        # o_proj of one token onto the residual stream.
        dict(name="gemm_one_token", kind="gemm", dtype="bf16", M=1, K=4096, N=4096, leaf=256, k_first=1, bias="same", act="none", residual=True),
        # down_proj of a ragged mid-size batch onto the residual stream.
        dict(name="gemm_down_residual", kind="gemm", dtype="fp16", M=500, K=12288, N=4096, leaf=256, k_first=3, bias="none", act="none", residual=True),
        # The first product of an MLP without a gate: bias and GELU of a prefill.
        dict(name="gemm_gelu_prefill", kind="gemm", dtype="bf16", M=4096, K=4096, N=12288, leaf=256, k_first=1, bias="same", act="gelu", residual=False),
        # A decode batch on an 8-bit weight: scales of the rows and of the channels, bias, residual.
        dict(name="gemm_fp8_decode", kind="gemm_fp8", fmt="e4m3", dtype="bf16", M=16, K=12288, N=4096, leaf=256, k_first=3, bias="none", act="none", residual=True),
        # The qkv projection of a prefill on 8-bit operands: scales and bias.
        dict(name="gemm_fp8_prefill", kind="gemm_fp8", fmt="e4m3", dtype="bf16", M=4000, K=4096, N=6144, leaf=256, k_first=1, bias="fp32", act="none", residual=False),
        # down_proj of a ragged prefill on microscaled operands, onto the residual stream.
        dict(name="gemm_mx_prefill", kind="gemm_mx", fmt="e4m3", dtype="bf16", M=1500, K=12288, N=4096, leaf=256, k_first=3, bias="same", act="none", residual=True),
        # The shards' partial sums of a column block with a bias and an activation, then the residual.
        dict(name="combine_tp4", kind="combine", dtype="bf16", P=4, M=1000, N=4096, bias="same", act="silu", residual=True),
    ]


def _log_int(rng, lo, hi):
    """An integer spread over the logarithm of [lo, hi]; odd values as likely as even ones."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def _draw_once(rng):
    kind = rng.choice(["norm", "norm", "tail", "silu", "gemm", "gemm", "gemm_fp8", "gemm_fp8", "gemm_mx", "combine"])
    dt, fmt, scheme = rng.choice(["bf16", "bf16", "fp16"]), rng.choice(["e4m3", "e4m3", "e5m2"]), rng.choice(["fp8", "mx"])
    width = lambda: rng.choice([4096, 5120, 5120, 32 * _log_int(rng, 4, 512)])
    if kind == "norm":
        return dict(kind=kind, scheme=scheme, fmt=fmt, dtype=dt, M=_log_int(rng, 1, 8192), H=width(), residual=rng.random() < 0.7)
    if kind == "tail":
        return dict(kind=kind, scheme=scheme, fmt=fmt, dtype=dt, P=rng.choice([1, 2, 4, 8]), M=_log_int(rng, 1, 2048), H=width())
    if kind == "silu":
        return dict(kind=kind, scheme=scheme, fmt=fmt, dtype=dt, M=_log_int(rng, 1, 4096),
                    I=rng.choice([12288, 14336, 25600, 32 * _log_int(rng, 8, 800)]))
    ends = dict(bias=rng.choice(["none", "same", "fp32"]), act=rng.choice(["none", "none", "relu", "silu", "gelu", "gelu_tanh"]),
                residual=rng.random() < 0.6)
    if kind == "combine":
        return dict(kind=kind, dtype=dt, P=rng.choice([1, 2, 4, 8]), M=_log_int(rng, 1, 2048), N=rng.choice([4096, 5120, _log_int(rng, 64, 8192)]), **ends)
    if kind == "gemm":
        K, N, leaf, kf = rng.choice(GEMMS_16)
        return dict(kind=kind, dtype=dt, M=_log_int(rng, 1, 4096), K=K, N=N, leaf=leaf, k_first=kf, **ends)
    K, N, leaf, kf = rng.choice(GEMMS_8)
    return dict(kind=kind, fmt=fmt, dtype="bf16", M=_log_int(rng, 1, 4096), K=K, N=N, leaf=leaf, k_first=kf, **ends)


def _cost(case):
    w = work(case)
    return max(w["bytes"] / 5e12, w["flops"] / 1e15)


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        case = _draw_once(rng)
        if _cost(case) <= most:
            return case


def work(case):
    """What a pass cannot do without: each input read once, each output written once; the products' operations."""
    k, M = case["kind"], case["M"]
    scales = lambda n: M * n / 32 if case["scheme"] == "mx" else M * 4
    if k == "norm":
        n = case["H"]
        return {"bytes": M * n * (2 + (4 if case["residual"] else 0) + 1) + 2 * n + scales(n), "flops": 0}
    if k == "tail":
        n = case["H"]
        return {"bytes": M * n * (4 * case["P"] + 4 + 1) + 2 * n + scales(n), "flops": 0}
    if k == "silu":
        return {"bytes": M * case["I"] * 5 + scales(case["I"]), "flops": 0}
    N = case["N"]
    ends = M * N * (4 if case["residual"] else 2) + N * {"none": 0, "same": 2, "fp32": 4}[case["bias"]]
    if k == "combine":
        return {"bytes": 4 * case["P"] * M * N + ends, "flops": 0}
    K = case["K"]
    if k == "gemm":
        operands = 2 * (M * K + K * N)
    else:
        operands = (M + N) * K + ((M + N) * K / 32 if k == "gemm_mx" else 4 * (M + N))
    return {"bytes": operands + ends, "flops": 2 * M * N * K}


# ---- inputs ----

def _rows(g, M, n, dtype):
    """Rows of a residual stream: N(0, 1) with a few channels that are far larger, as trained models have them."""
    x = torch.randn((M, n), generator=g, device=DEV)
    x[:, :: max(1, n // 5)] *= 12.0
    return x.to(dtype)


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    k, M, dt = case["kind"], case["M"], TYPES[case["dtype"]]
    s = dict(case=case)
    randn = lambda *shape: torch.randn(shape, generator=g, device=DEV)
    if k in ("norm", "tail"):
        H = case["H"]
        s["weight"] = (1 + 0.1 * randn(H)).to(dt)
        if k == "norm":
            s["x"] = _rows(g, M, H, dt)
        else:
            s["partials"] = randn(case["P"], M, H) * 0.6
        s["residual"] = _rows(g, M, H, dt) if k == "tail" or case["residual"] else None
        return s
    if k == "silu":
        s["gate_up"] = torch.cat([2 * randn(M, case["I"]), randn(M, case["I"])], dim=1).to(dt)      # the merged projection's output
        return s
    N = case["N"]
    s["bias"] = None if case["bias"] == "none" else (0.5 * randn(N)).to(dt if case["bias"] == "same" else torch.float32)
    s["residual"] = _rows(g, M, N, dt) if case["residual"] else None
    if k == "combine":
        s["partials"] = randn(case["P"], M, N) * 0.6
        return s
    K = case["K"]
    if k == "gemm":
        s["X"], s["W"] = randn(M, K).to(dt), (0.02 * randn(K, N)).to(dt)
    elif k == "gemm_fp8":                                          # a scale per token and per output channel
        s["X"], s["row_scale"] = _row_scaled(_rows(g, M, K, torch.float32), case["fmt"])
        s["Wt"], s["col_scale"] = _row_scaled(0.02 * randn(N, K), case["fmt"])
        s["X"], s["Wt"] = s["X"].view(torch.uint8), s["Wt"].view(torch.uint8)
    else:
        s["X"], s["Xs"] = (t.view(torch.uint8) for t in _micro_scaled(_rows(g, M, K, torch.float32), case["fmt"]))
        s["Wt"], s["Ws"] = (t.view(torch.uint8) for t in _micro_scaled(0.02 * randn(N, K), case["fmt"]))
    return s


# ---- the operators in plain form ----

def _row_scaled(y, fmt):
    """8-bit values and one fp32 scale per row that brings its largest magnitude to the format's largest number."""
    amax = y.abs().amax(dim=1)
    scale = torch.where(amax > 0, (amax / LARGEST[fmt]).clamp(min=2.0 ** -126), torch.ones_like(amax))
    return (y * (1.0 / scale)[:, None]).to(FP8[fmt]), scale


def _micro_scaled(y, fmt):
    """8-bit values and a power of two per 32 consecutive ones that brings the largest of them into the format's top binade."""
    blocks = y.reshape(y.shape[0], -1, 32)
    amax = blocks.abs().amax(dim=2)
    fraction, exponent = torch.frexp(amax)                         # amax = fraction 2^exponent, fraction in [1/2, 1)
    ceil_log2 = exponent - (fraction == 0.5).to(exponent.dtype)
    byte = torch.where(amax > 0, ceil_log2 - TOP[fmt] + 127, torch.full_like(exponent, 127)).clamp(1, 254)
    q = (blocks * torch.exp2((127 - byte).float())[:, :, None]).to(FP8[fmt])
    return q.reshape(y.shape), byte.to(torch.uint8).view(torch.float8_e8m0fnu)


def _eight_bits(y, case):
    return (_row_scaled if case["scheme"] == "fp8" else _micro_scaled)(y, case["fmt"])


def _plain_norm(s, case):
    dt = TYPES[case["dtype"]]
    x = s["x"].float() if case["kind"] == "norm" else s["partials"].sum(dim=0).to(dt).float()
    hidden = None
    if s["residual"] is not None:
        hidden = (x + s["residual"].float()).to(dt)
        x = hidden.float()
    r = 1.0 / torch.sqrt(x.square().mean(dim=1, keepdim=True) + EPS)
    q, scale = _eight_bits(x * r * s["weight"].float(), case)
    return hidden, q, scale


def _plain_silu(s, case):
    gate, up = s["gate_up"].float().chunk(2, dim=1)
    return _eight_bits(gate / (1.0 + torch.exp(-gate)) * up, case)


def _plain_ends(y, s, case):
    if "row_scale" in s:
        y = y * s["row_scale"][:, None] * s["col_scale"]
    if s["bias"] is not None:
        y = y + s["bias"].float()
    act = case["act"]
    if act == "relu":
        y = y.clamp(min=0)
    elif act == "silu":
        y = y / (1.0 + torch.exp(-y))
    elif act == "gelu":
        y = 0.5 * y * torch.erfc(y * -math.sqrt(0.5))
    elif act == "gelu_tanh":
        y = 0.5 * y * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (y + 0.044715 * y * y * y)))
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return y.to(TYPES[case["dtype"]])


def _spread(scales, K):
    return scales.view(torch.float8_e8m0fnu).float().repeat_interleave(32, dim=1)[:, :K]


def _plain_gemm(s, case):
    k = case["kind"]
    if k == "gemm":
        y = s["X"].float() @ s["W"].float()
    elif k == "combine":
        y = s["partials"].sum(dim=0)
    else:
        X, Wt = s["X"].view(FP8[case["fmt"]]).float(), s["Wt"].view(FP8[case["fmt"]]).float()
        if k == "gemm_mx":
            X, Wt = X * _spread(s["Xs"], case["K"]), Wt * _spread(s["Ws"], case["K"])
        y = X @ Wt.t()
    return _plain_ends(y, s, case)


# ---- the framework's calls ----

def _own(s, case):
    from paper_2511_17826_amd import binding as tb
    k = case["kind"]
    if k in ("norm", "tail", "silu"):
        fp8, fmt = case["scheme"] == "fp8", case["fmt"]
        if k == "norm":
            hidden, q, scale = (tb.tbik_rmsnorm_fp8 if fp8 else tb.tbik_rmsnorm_mxfp8)(s["x"], s["weight"], EPS, residual=s["residual"], fmt=fmt)
        elif k == "tail":
            hidden, q, scale = (tb.tbik_combine_residual_rmsnorm_fp8 if fp8 else tb.tbik_combine_residual_rmsnorm_mxfp8)(
                s["partials"], s["residual"], s["weight"], EPS, fmt=fmt)
        else:
            I = case["I"]
            q, scale = (tb.tbik_silu_mul_fp8 if fp8 else tb.tbik_silu_mul_mxfp8)(s["gate_up"][:, :I], s["gate_up"][:, I:], fmt=fmt)
        q = q.view(FP8[fmt])
        scale = scale if fp8 else scale.view(torch.float8_e8m0fnu)
        return (q, scale) if k == "silu" else (hidden, q, scale)
    ends = dict(bias=s["bias"], activation=None if case["act"] == "none" else case["act"], residual=s["residual"])
    if k == "gemm":
        return tb.tbik_gemm_epilogue(s["X"], s["W"], case["leaf"], case["k_first"], **ends)
    if k == "combine":
        return tb.tbik_tree_combine_epilogue(s["partials"], out_dtype=TYPES[case["dtype"]], **ends)
    if k == "gemm_fp8":
        return tb.tbik_gemm_fp8_epilogue(s["X"], s["Wt"], case["leaf"], case["k_first"], case["fmt"], row_scale=s["row_scale"],
                                         col_scale=s["col_scale"], **ends)
    return tb.tbik_gemm_mxfp8_epilogue(s["X"], s["Xs"], s["Wt"], s["Ws"], case["leaf"], case["k_first"], case["fmt"], **ends)


def run(state):
    s, case = state, state["case"]
    if own:
        return _own(s, case)
    if case["kind"] in ("norm", "tail"):
        return _plain_norm(s, case)
    if case["kind"] == "silu":
        return _plain_silu(s, case)
    return _plain_gemm(s, case)


# ---- the operators' definitions in 64 bits ----

def _on_grid(v, fraction_bits, lowest):
    """The nearest number with this many fraction bits and exponents from `lowest` on, ties to even."""
    exponent = torch.frexp(v).exponent - 1
    step = torch.exp2((exponent.clamp(min=lowest) - fraction_bits).double())
    return torch.round(v / step) * step


def _exact_16(v, dtype):
    return _on_grid(v, 7, -126) if dtype == "bf16" else _on_grid(v, 10, -14)


def _exact_eight_bits(v, case):
    fmt = case["fmt"]
    if case["scheme"] == "fp8":
        top = v.abs().max(dim=1, keepdim=True).values
        scale = torch.where(top > 0, top / LARGEST[fmt], torch.ones_like(top))
        return _on_grid(v / scale, *STEP[fmt]), scale[:, 0]
    blocks = v.reshape(v.shape[0], v.shape[1] // 32, 32)
    top = blocks.abs().max(dim=2, keepdim=True).values
    scale = torch.exp2(torch.ceil(torch.log2(torch.where(top > 0, top, torch.full_like(top, 2.0 ** TOP[fmt])))) - TOP[fmt])
    return _on_grid(blocks / scale, *STEP[fmt]).reshape(v.shape), scale[:, :, 0]


def _exact_act(v, act):
    if act == "relu":
        return torch.where(v > 0, v, torch.zeros_like(v))
    if act == "silu":
        return v * torch.special.expit(v)
    if act == "gelu":
        return v * torch.special.ndtr(v)
    if act == "gelu_tanh":
        return v * torch.special.expit(2 * math.sqrt(2 / math.pi) * (v + 0.044715 * v ** 3))
    return v


def exact(case, seed):
    s = prepare(case, seed)
    k = case["kind"]
    if k in ("norm", "tail"):
        v = s["x"].double() if k == "norm" else _exact_16(s["partials"].double().sum(dim=0), case["dtype"])
        hidden = None
        if s["residual"] is not None:
            v = hidden = _exact_16(v + s["residual"].double(), case["dtype"])
        n = v * s["weight"].double() / torch.sqrt((v * v).sum(dim=1, keepdim=True) / case["H"] + EPS)
        return (hidden,) + _exact_eight_bits(n, case)
    if k == "silu":
        gate, up = s["gate_up"][:, :case["I"]].double(), s["gate_up"][:, case["I"]:].double()
        return _exact_eight_bits(_exact_act(gate, "silu") * up, case)
    if k == "combine":
        v = s["partials"].double().sum(dim=0)
    elif k == "gemm":
        v = torch.mm(s["X"].double(), s["W"].double())
    else:
        a, b = s["X"].view(FP8[case["fmt"]]).double(), s["Wt"].view(FP8[case["fmt"]]).double()
        if k == "gemm_fp8":
            a, b = a * s["row_scale"].double()[:, None], b * s["col_scale"].double()[:, None]
        else:
            power = lambda t: torch.exp2(t.double() - 127)[:, :, None]
            a = (a.reshape(a.shape[0], -1, 32) * power(s["Xs"])).reshape(a.shape)
            b = (b.reshape(b.shape[0], -1, 32) * power(s["Ws"])).reshape(b.shape)
        v = torch.mm(a, b.t().contiguous())
    if s["bias"] is not None:
        v = v + s["bias"].double()
    v = _exact_act(v, case["act"])
    return v if s["residual"] is None else v + s["residual"].double()
