"""Plain references of the 8-bit outputs and the epilogues for the tests: the fp32 steps one by one in numpy where the contract
fixes them (bit comparisons), the definitions in 64 bits beside it."""
import numpy as np
import torch

TORCH8 = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
LARGEST = {"e4m3": 448.0, "e5m2": 57344.0}
EMAX = {"e4m3": 8, "e5m2": 15}
f32 = np.float32


def tree_sum_of_squares(h):
    """TreeSum of App. C on the squares of fp32 rows [M, H]: in-order leaves of 8, padded with +0 to a power of two."""
    M, H = h.shape
    sq = (h * h).astype(f32).reshape(M, H // 8, 8)
    leaf = np.zeros((M, H // 8), f32)
    for e in range(8):
        leaf = (leaf + sq[:, :, e]).astype(f32)
    n = 1
    while n < H // 8:
        n *= 2
    v = np.zeros((M, n), f32)
    v[:, :H // 8] = leaf
    while v.shape[1] > 1:
        v = (v[:, 0::2] + v[:, 1::2]).astype(f32)
    return v[:, 0]


def normed32(h, w, eps):
    """The fp32 value that the RMSNorm of rows h (fp32 values of 16-bit numbers) rounds."""
    with np.errstate(all="ignore"):
        ss = tree_sum_of_squares(h)
        r = (f32(1) / np.sqrt((ss / f32(h.shape[1]) + f32(eps)).astype(f32)).astype(f32)).astype(f32)
        return ((h * r[:, None]).astype(f32) * w[None, :]).astype(f32)


def to_8(v, fmt):
    """fp32 -> patterns, to nearest even (no value here is past the format's largest number)."""
    return torch.from_numpy(np.ascontiguousarray(v, dtype=f32)).to(TORCH8[fmt]).view(torch.uint8).numpy()


def value_of_8(q, fmt):
    return torch.from_numpy(np.ascontiguousarray(q)).view(TORCH8[fmt]).double().numpy()


def row_scaled(v, fmt):
    """(patterns, scales) with a scale per row of fp32 rows, each operation rounded to fp32 as stated."""
    with np.errstate(all="ignore"):
        amax = np.nanmax(np.where(np.isnan(v), 0, np.abs(v)), axis=1).astype(f32)
        scale = np.where(amax > 0, np.maximum((amax / f32(LARGEST[fmt])).astype(f32), f32(2.0 ** -126)), f32(1)).astype(f32)
        factor = (f32(1) / scale).astype(f32)
        return to_8((v * factor[:, None]).astype(f32), fmt), scale


def micro_scaled(v, fmt):
    """(patterns, scale bytes) with a power of two per 32 columns of fp32 rows."""
    M, n = v.shape
    b = v.reshape(M, n // 32, 32)
    amax = np.where(np.isnan(b), 0, np.abs(b)).max(axis=2).astype(np.float64)
    frac, ex = np.frexp(amax)                               # amax = frac 2^ex, frac in [1/2, 1)
    ceil_log2 = np.where(np.isinf(amax), 128, ex - (frac == 0.5))
    byte = np.where(amax > 0, np.maximum(ceil_log2 - EMAX[fmt] + 127, 1), 127).astype(np.int64)
    with np.errstate(all="ignore"):
        q = to_8((b * np.exp2(127.0 - byte)[:, :, None].astype(f32)).astype(f32).reshape(M, n), fmt)
    return q, byte.astype(np.uint8)


def same_patterns(got, want, fmt):
    """Equal patterns; a NaN is any NaN."""
    g, w = value_of_8(got, fmt), value_of_8(want, fmt)
    return np.array_equal(np.isnan(g), np.isnan(w)) and np.array_equal(got[~np.isnan(g)], want[~np.isnan(g)])


def act64(v, act):
    import scipy.special as sp
    v = np.asarray(v, dtype=np.float64)
    if act == "relu":
        return np.where(v < 0, 0.0, v)
    if act == "silu":
        return v * sp.expit(v)
    if act == "gelu":
        return v * sp.ndtr(v)
    if act == "gelu_tanh":
        return v * sp.expit(2 * np.sqrt(2 / np.pi) * (v + 0.044715 * v ** 3))
    return v


def act_tolerance(v, act):
    """Relative error of the fp32 activations against the definition, in steps of u = 2^-24.  Common: 1 + e, the reciprocal and the
    exponential (an ulp = 2 u each), the last product: 1 + 2 + 2 + 1 = 6 u; e's part counts in full only where e >> 1 (v < 0).
      silu       exponent v log2(e): constant and product, u each, an absolute error of |v| 2 u in the exponent of e^-v
      gelu_tanh  exponent -2 U, U = sqrt(2/pi)(v + 0.044715 v^3): v^2, the fused step (two constants), the product, the constant
                 and the last product, six roundings: |2 U| 6 u
      gelu       tail = t q(t) e^(-v^2/2): exponent's v^2, constant, product: (v^2 / 2) 3 u; q(t) 3.3e-7 = 5.6 u; t 3 u (its argument
                 included); two products 2 u, exponential 2 u, 1 - tail u, last product u: 15 u"""
    v = np.abs(np.asarray(v, dtype=np.float64))
    u = 2.0 ** -24
    if act == "silu":
        return (6 + 2 * v) * u
    if act == "gelu_tanh":
        return (6 + 12 * np.sqrt(2 / np.pi) * (v + 0.044715 * v ** 3)) * u
    if act == "gelu":
        return (15 + 1.5 * v * v) * u
    return np.zeros_like(v)
