// 8-bit outputs with scales, as the 8-bit and microscaling products take their operands: how a kernel that holds fp32 values of a
// row turns them into patterns.  Every element takes one rounding, from fp32 to nearest even.
//   a scale per row (tbik_gemm_fp8_epilogue's row_scale):  scale = max |v| / largest, fp32, at least 2^-126, 1 for a row of
//       zeros;  q = r8(v * (1 / scale)), both divisions rounded once.  |q| stays within the format: v / scale is at most `largest`
//       but for three fp32 roundings, far less than half a step there.
//   microscaling (tbik_gemm_mxfp8's operands):  per 32 consecutive elements the power of two that brings their largest magnitude
//       into (2^(emax - 1), 2^emax] (emax: 8 for E4M3, 15 for E5M2; 2^0 for zeros), as the byte exponent + 127, at least 1;  q = r8(v / scale),
//       the division exact but below 2^-126.  Nothing saturates.
// NaN does not count for a maximum and becomes a NaN pattern; an infinity makes its scale infinite (a scale per row) or as
// large as the largest finite number asks for (microscaling) and becomes NaN (E4M3) or infinity (E5M2; NaN with a scale per row).
#pragma once

#include "tbik_device.hpp"
#include "tbik_internal.hpp"

namespace tbik {

// Eight values to eight bytes (v_cvt_pk_fp8_f32 / v_cvt_pk_bf8_f32: round to nearest even).
__device__ __forceinline__ uint2 to_8_bits(const float (&f)[8], float factor, bool e5m2) {
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = f[i] * factor;
    int lo = 0, hi = 0;
    if (e5m2) {
        lo = __builtin_amdgcn_cvt_pk_bf8_f32(v[0], v[1], lo, false);
        lo = __builtin_amdgcn_cvt_pk_bf8_f32(v[2], v[3], lo, true);
        hi = __builtin_amdgcn_cvt_pk_bf8_f32(v[4], v[5], hi, false);
        hi = __builtin_amdgcn_cvt_pk_bf8_f32(v[6], v[7], hi, true);
    } else {
        lo = __builtin_amdgcn_cvt_pk_fp8_f32(v[0], v[1], lo, false);
        lo = __builtin_amdgcn_cvt_pk_fp8_f32(v[2], v[3], lo, true);
        hi = __builtin_amdgcn_cvt_pk_fp8_f32(v[4], v[5], hi, false);
        hi = __builtin_amdgcn_cvt_pk_fp8_f32(v[6], v[7], hi, true);
    }
    return make_uint2((unsigned)lo, (unsigned)hi);
}

__device__ __forceinline__ float largest_magnitude(const float (&f)[8]) {
    float m = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = fmaxf(m, __builtin_fabsf(f[i]));
    return m;
}

// A scale per row.
__device__ __forceinline__ float row_scale_of(float amax, bool e5m2) {
    return amax > 0.0f ? fmaxf(amax / (e5m2 ? 57344.0f : 448.0f), 0x1p-126f) : 1.0f;
}

// Microscaling: a block of 32 lies in the eight elements of four consecutive lanes (4 i .. 4 i + 3); all of them are active.
__device__ __forceinline__ float block_max(float m) {
    m = fmaxf(m, from_lane_in_row<0xB1>(m));
    return fmaxf(m, from_lane_in_row<0x4E>(m));
}
__device__ __forceinline__ int block_scale_byte(float amax, bool e5m2) {
    const unsigned bits = __float_as_uint(amax);
    const int ceil_exponent = (int)(bits >> 23) + ((bits & 0x7fffffu) != 0);      // + 127; subnormal numbers end below 1
    return amax > 0.0f ? max(ceil_exponent - (e5m2 ? 15 : 8), 1) : 127;
}
// 2^(127 - byte), for bytes up to 253 (the largest is 255 - 8).
__device__ __forceinline__ float block_factor(int byte) { return __uint_as_float((unsigned)(254 - byte) << 23); }

}  // namespace tbik
