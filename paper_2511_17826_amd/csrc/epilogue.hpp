// The epilogue of the matrix products (tbik_epilogue), shared by every kernel that ends one: on the fp32 value t = T(...) of
// an output element, in this order and each step one fp32 operation,
//   t * row_scale[m] * col_scale[n]  + bias[n]  -> activation  + residual[m][n]  -> one rounding to the output's type.
// What is absent is skipped.  Position-wise, and the one definition for all kernels, so an element's bits do not depend on
// the kernel, the tile, the K split or the launch that computes it.
#pragma once

#include "tbik_device.hpp"
#include "tbik_internal.hpp"

namespace tbik {

// v / (1 + e^-v) as silu_mul() forms it: hardware exponential and reciprocal, about one fp32 ulp each.
__device__ __forceinline__ float silu_of(float v) { return v * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(v * -1.4426950408889634f)); }

// v Phi(v), Phi the normal distribution function.  Its tail, Phi(-a) = erfc(a / sqrt 2) / 2, decides both sides (v < 0: the tail
// itself; else one minus it), so it is formed without a cancellation: erfc(z) = e^(-z^2) erfcx(z), and erfcx(z) = t q(t) with
// t = 1 / (1 + 0.375 z), q the polynomial of degree 8 whose largest relative error over z in [0, 10.2] is smallest, fitted for this
// kernel (3.2e-8 with its coefficients in fp32; t q(t) formed from v in fp32, with a correctly rounded reciprocal, 3.6e-7); beyond,
// e^(-z^2) is zero in fp32.  The coefficients hold the half.
__device__ __forceinline__ float gelu_of(float v) {
    const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(__builtin_fabsf(v), 0.26516504294495535f, 1.0f));      // 0.375 / sqrt 2
    float q = 0.03065868280827999f;
    q = __builtin_fmaf(q, t, -0.14314346015453339f);
    q = __builtin_fmaf(q, t, 0.21515342593193054f);
    q = __builtin_fmaf(q, t, -0.11354447156190872f);
    q = __builtin_fmaf(q, t, 0.13608127832412720f);
    q = __builtin_fmaf(q, t, 0.06107687950134277f);
    q = __builtin_fmaf(q, t, 0.10257558524608612f);
    q = __builtin_fmaf(q, t, 0.10533598810434341f);
    q = __builtin_fmaf(q, t, 0.10580608993768692f);
    const float tail = q * t * __builtin_amdgcn_exp2f(v * v * -0.72134752044448170f);
    return v * (v < 0.0f ? tail : 1.0f - tail);
}

// v (1 + tanh u) / 2 with u = sqrt(2 / pi) (v + 0.044715 v^3), as v / (1 + e^(-2 u)).
__device__ __forceinline__ float gelu_tanh_of(float v) {
    const float u = v * __builtin_fmaf(v * v, 0.035677408136300125f, 0.79788456080286541f);
    return v * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(u * -2.8853900817779268f));
}

template <int ACT>
__device__ __forceinline__ float activation_of(float v) {
    if constexpr (ACT == TBIK_ACT_RELU) return v < 0.0f ? 0.0f : v;            // NaN stays
    else if constexpr (ACT == TBIK_ACT_SILU) return silu_of(v);
    else if constexpr (ACT == TBIK_ACT_GELU) return gelu_of(v);
    else return gelu_tanh_of(v);
}

__device__ __forceinline__ float widened(const void *p, int64_t i, int dtype) {
    if (dtype == TBIK_F32) return reinterpret_cast<const float *>(p)[i];
    const uint16_t h = reinterpret_cast<const uint16_t *>(p)[i];
    return dtype == TBIK_F16 ? (float)__builtin_bit_cast(_Float16, h) : bf16_bits_to_f32(h);
}
__device__ __forceinline__ uint32_t pack_16x2(float lo, float hi, bool f16) { return f16 ? pack_f16x2(lo, hi) : pack_bf16x2(lo, hi); }

// The steps on COUNT elements of one row, consecutive columns; what is absent is skipped for all of them at once (uniform branches).
// A step's fp32 values are made values of their own: no merging of a last operation with the rounding to 16 bits (see silu_mul).
template <int COUNT>
__device__ __forceinline__ void values_of_their_own(float (&v)[COUNT]) {
#pragma unroll
    for (int i = 0; i < COUNT; ++i) asm("" : "+v"(v[i]));
}
// of ROWS rows; the flags say which parts there are, at run time or as constants
template <int ROWS, int COUNT, class Flag1, class Flag2, class Flag3>
__device__ __forceinline__ void scale_and_bias(Flag1 row_scale, Flag2 col_scale, Flag3 bias, float (&v)[ROWS][COUNT], const float (&rs)[ROWS], const float (&cs)[COUNT], const float (&b)[COUNT]) {
    if (row_scale) {
#pragma unroll
        for (int r = 0; r < ROWS; ++r)
#pragma unroll
            for (int i = 0; i < COUNT; ++i) v[r][i] = v[r][i] * rs[r];
    }
    if (col_scale) {
#pragma unroll
        for (int r = 0; r < ROWS; ++r)
#pragma unroll
            for (int i = 0; i < COUNT; ++i) v[r][i] = v[r][i] * cs[i];
    }
    if (bias) {
#pragma unroll
        for (int r = 0; r < ROWS; ++r)
#pragma unroll
            for (int i = 0; i < COUNT; ++i) v[r][i] = v[r][i] + b[i];
    }
#pragma unroll
    for (int r = 0; r < ROWS; ++r) values_of_their_own(v[r]);
}
template <int ROWS, int COUNT>
__device__ __forceinline__ void scale_and_bias(const EpilogueParams &e, float (&v)[ROWS][COUNT], const float (&rs)[ROWS], const float (&cs)[COUNT], const float (&b)[COUNT]) {
    scale_and_bias(e.row_scale != nullptr, e.col_scale != nullptr, e.bias != nullptr, v, rs, cs, b);
}
template <int ACT, int ROWS, int COUNT>
__device__ __forceinline__ void activate_as(float (&v)[ROWS][COUNT]) {
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
#pragma unroll
        for (int i = 0; i < COUNT; ++i) v[r][i] = activation_of<ACT>(v[r][i]);
        values_of_their_own(v[r]);
    }
}
template <int ROWS, int COUNT>
__device__ __forceinline__ void activate(int act, float (&v)[ROWS][COUNT]) {
    switch (act) {                         // uniform
        case TBIK_ACT_RELU: activate_as<TBIK_ACT_RELU>(v); break;
        case TBIK_ACT_SILU: activate_as<TBIK_ACT_SILU>(v); break;
        case TBIK_ACT_GELU: activate_as<TBIK_ACT_GELU>(v); break;
        case TBIK_ACT_GELU_TANH: activate_as<TBIK_ACT_GELU_TANH>(v); break;
        default: break;
    }
}
template <int COUNT>
__device__ __forceinline__ void add_residual(float (&v)[COUNT], const float (&r)[COUNT]) {
#pragma unroll
    for (int i = 0; i < COUNT; ++i) v[i] = v[i] + r[i];
    values_of_their_own(v);
}

// One element: its operands as they lie in memory, so that a kernel can have them on their way long before it needs them, and the
// element through the epilogue, stored.
struct ElementOperands {
    float rs, cs;
    uint32_t bias, residual;
};
__device__ __forceinline__ uint32_t raw_element(const void *p, int64_t i, int dtype) {
    return dtype == TBIK_F32 ? reinterpret_cast<const uint32_t *>(p)[i] : reinterpret_cast<const uint16_t *>(p)[i];
}
__device__ __forceinline__ float value_of_raw(uint32_t raw, int dtype) {
    return dtype == TBIK_F32 ? __uint_as_float(raw) : dtype == TBIK_F16 ? (float)__builtin_bit_cast(_Float16, (uint16_t)raw) : bf16_bits_to_f32(raw);
}
__device__ __forceinline__ ElementOperands element_operands(const EpilogueParams &e, int64_t row, int64_t col) {
    ElementOperands o = {0.0f, 0.0f, 0u, 0u};
    if (e.row_scale) o.rs = e.row_scale[row];
    if (e.col_scale) o.cs = e.col_scale[col];
    if (e.bias) o.bias = raw_element(e.bias, col, e.bias_dtype);
    if (e.residual) o.residual = raw_element(e.residual, row * e.ldr + col, e.y_dtype);
    return o;
}
__device__ __forceinline__ void finish_and_store(const EpilogueParams &e, float t, const ElementOperands &o, void *Y, int64_t ldy, int64_t row, int64_t col) {
    float v[1][1] = {{t}};
    const float cs[1] = {o.cs}, b[1] = {value_of_raw(o.bias, e.bias_dtype)}, r[1] = {value_of_raw(o.residual, e.y_dtype)}, rs[1] = {o.rs};
    scale_and_bias(e, v, rs, cs, b);
    activate(e.act, v);
    if (e.residual) add_residual(v[0], r);
    if (e.y_dtype == TBIK_F32) reinterpret_cast<float *>(Y)[row * ldy + col] = v[0][0];
    else reinterpret_cast<uint16_t *>(Y)[row * ldy + col] = (uint16_t)pack_16x2(v[0][0], 0.0f, e.y_dtype == TBIK_F16);
}
__device__ __forceinline__ void finish_and_store(const EpilogueParams &e, float t, void *Y, int64_t ldy, int64_t row, int64_t col) {
    finish_and_store(e, t, element_operands(e, row, col), Y, ldy, row, col);
}

}  // namespace tbik
