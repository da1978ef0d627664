// Tree-Based MatMul of 16-bit rows on a 4-bit weight with a scale per group of consecutive k and channel (decode batches).
//
//   Y[m,n] = T over superleaves of  sum over groups g of the superleaf, ascending:  acc = fma(scale[n,g], S_g, acc), acc from +0
//   S_g    = sum over k of the group of  x[m,k] (q[n,k] - zero[n,g])     chained matrix instructions from +0
// q - zero is a whole number of -15 .. 15 and exact in either 16-bit format, so the weight is never rounded: the scale multiplies a
// group's fp32 sum, once per group, row and channel.
//
// What bounds it is the weight's bytes (half a byte an element) and, of more rows, the batch's, which every workgroup reads.  A workgroup
// takes 32 channels, up to 32 rows and all of a shard's K in one launch: its wavefronts take consecutive superleaves each, whole and in order
// (Sec. 4.2, App. D.1), and the upper levels of the tree run over their sums in LDS (App. C).  An instruction multiplies 16 k of 32
// channels; which 16 of a unit of 64 (or 32, for groups that no 64 divides) it takes is chosen so that a lane's elements of the
// whole unit are 16 (8) consecutive bytes: half a lane's 32 channels at the unit's first half, the other at its second.  Operands go
// from memory to registers, DEPTH units ahead; an element becomes a float with one conversion of the hardware (v_cvt_off_f32_i4, the 4-bit two's
// complement number over 16, which the scale takes back exactly) and two of them a pair of 16-bit values with one more.
#include <type_traits>

#include "tbik_device.hpp"
#include "tbik_internal.hpp"

namespace tbik {

namespace {

struct W4Params {
    const uint16_t *X;
    const uint8_t *W;
    const uint16_t *scales;
    const uint8_t *zeros;
    float *partials;
    void *Y;
    int64_t ldx, ldw, lds, ldz, ldy;
    int M, N;
    int y_f32;
    int group, superleaf;
    int leaves_per_wave, active_waves, leaves_per_shard;
};

typedef uint32_t w4_u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t w4_u32x2 __attribute__((ext_vector_type(2)));

// Eight elements of one dword, element i in bits 4 i .. 4 i + 3, as 16-bit floats of (q - 8) / 16, or (q - zero) / 16.
template <bool F16, bool ZEROS>
__device__ __forceinline__ bf16x8 widened_levels(uint32_t w, float zero) {
    const uint32_t even = w ^ 0x88888888u, odd = even >> 4;          // 4-bit two's complement of q - 8; the conversion reads four bits
    float v[8];
#pragma unroll
    for (int b = 0; b < 4; ++b) {
        v[2 * b] = __builtin_amdgcn_cvt_off_f32_i4(even >> (8 * b));
        v[2 * b + 1] = __builtin_amdgcn_cvt_off_f32_i4(odd >> (8 * b));
    }
    if constexpr (ZEROS) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = v[i] - zero;
    }
    union { uint32_t u[4]; bf16x8 v; } out;
#pragma unroll
    for (int b = 0; b < 4; ++b) {
        if constexpr (F16) out.u[b] = pack_f16x2(v[2 * b], v[2 * b + 1]);
        else out.u[b] = __builtin_amdgcn_perm(__float_as_uint(v[2 * b + 1]), __float_as_uint(v[2 * b]), 0x07060302u);      // exact: the upper halves
    }
    return out.v;
}

template <bool F16>
__device__ __forceinline__ float widened_16(uint16_t h) { return F16 ? (float)__builtin_bit_cast(_Float16, h) : bf16_bits_to_f32(h); }

constexpr int W4_WAVES = 8;

// UNIT: k of a lane pair's unit, 64 or 32.
template <int UNIT, bool F16, bool ZEROS>
__global__ __launch_bounds__(64 * W4_WAVES, 2) void gemm_w4_kernel(const W4Params p) {
    constexpr int STEPS = UNIT / 16, DEPTH = UNIT == 64 ? 4 : 8;
    using Words = std::conditional_t<UNIT == 64, w4_u32x4, w4_u32x2>;
    __shared__ float red[W4_WAVES * 1024];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int li = lane & 31, lg = lane >> 5;
    const int n0 = blockIdx.x * 32, m0 = blockIdx.y * 32;
    const int first_leaf = blockIdx.z * p.leaves_per_shard + wave * p.leaves_per_wave;
    f32x16 acc;
    if (wave < p.active_waves) {
        const int channel = min(n0 + li, p.N - 1);
        const int64_t k0 = (int64_t)first_leaf * p.superleaf;
        const uint8_t *w_at = p.W + channel * p.ldw + k0 / 2 + lg * (UNIT / 4);
        const uint16_t *s_at = p.scales + channel * p.lds + k0 / p.group;
        const uint8_t *z_at = ZEROS ? p.zeros + channel * p.ldz + k0 / p.group : nullptr;
        // Rows behind the last one read it once more; they are not stored.
        const uint16_t *x_at = p.X + (int64_t)min(m0 + li, p.M - 1) * p.ldx + k0 + lg * (UNIT / 2);
        const int units = p.leaves_per_wave * (p.superleaf / UNIT), units_per_group = p.group / UNIT, groups_per_leaf = p.superleaf / p.group;
        Words w[DEPTH];
        uint4 x[DEPTH][STEPS];
        auto fetch = [&](int d) __attribute__((always_inline)) {
            w[d] = *reinterpret_cast<const Words *>(w_at);
#pragma unroll
            for (int i = 0; i < STEPS; ++i) x[d][i] = *reinterpret_cast<const uint4 *>(x_at + 8 * i);
            w_at += UNIT / 2;
            x_at += UNIT;
        };
#pragma unroll
        for (int d = 0; d < DEPTH; ++d)
            if (d < units) fetch(d);
        f32x16 stash[4], sum;
        int left_in_group = units_per_group, left_in_leaf = groups_per_leaf, leaf = 0;
        float scale = widened_16<F16>(*s_at) * 16.0f, zero = 0.0f;                  // of the group that is being summed
        if constexpr (ZEROS) zero = (float)(int)((*z_at & 15) - 8) * 0.0625f;
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[r] = sum[r] = 0.0f;
        for (int u0 = 0; u0 < units; u0 += DEPTH) {
#pragma unroll
            for (int d = 0; d < DEPTH; ++d) {
                if (u0 + d >= units) continue;
#pragma unroll
                for (int i = 0; i < STEPS; ++i)
                    sum = mfma_32x32x16<F16>(__builtin_bit_cast(bf16x8, x[d][i]), widened_levels<F16, ZEROS>(w[d][i], zero), sum);
                if (u0 + d + DEPTH < units) fetch(d);
                if (--left_in_group == 0) {
                    left_in_group = units_per_group;
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        acc[r] = __builtin_fmaf(scale, sum[r], acc[r]);
                        sum[r] = 0.0f;
                    }
                    if (u0 + d + 1 < units) {
                        scale = widened_16<F16>(*++s_at) * 16.0f;
                        if constexpr (ZEROS) zero = (float)(int)((*++z_at & 15) - 8) * 0.0625f;
                    }
                    if (--left_in_leaf == 0) {                                      // a superleaf ends: the carry-over step of the tree
                        left_in_leaf = groups_per_leaf;
                        const int t = __builtin_ctz(~leaf);
#pragma unroll
                        for (int l = 0; l < 4; ++l)
                            if (l < t) {
#pragma unroll
                                for (int r = 0; r < 16; ++r) acc[r] = stash[l][r] + acc[r];
                            }
                        if (++leaf < p.leaves_per_wave) {
#pragma unroll
                            for (int l = 0; l < 4; ++l)
                                if (l == t) stash[l] = acc;
#pragma unroll
                            for (int r = 0; r < 16; ++r) acc[r] = 0.0f;
                        }
                    }
                }
            }
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) red[wave * 1024 + (8 * (r >> 2) + 4 * lg + (r & 3)) * 32 + li] = acc[r];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 1024 / (64 * W4_WAVES); ++i) {
        const int at = i * 64 * W4_WAVES + threadIdx.x, row = m0 + at / 32, col = n0 + at % 32;
        if (row >= p.M || col >= p.N) continue;
        float v[W4_WAVES];
#pragma unroll
        for (int w = 0; w < W4_WAVES; ++w) v[w] = red[w < p.active_waves ? w * 1024 + at : at];
#pragma unroll
        for (int s = 1; s < W4_WAVES; s *= 2)
#pragma unroll
            for (int r = 0; r < W4_WAVES; r += 2 * s)
                if (r + s < p.active_waves) v[r] = v[r] + v[r + s];
        if (p.partials) p.partials[((int64_t)blockIdx.z * p.M + row) * p.N + col] = v[0];
        else if (p.y_f32) reinterpret_cast<float *>(p.Y)[(int64_t)row * p.ldy + col] = v[0];
        else reinterpret_cast<uint16_t *>(p.Y)[(int64_t)row * p.ldy + col] = (uint16_t)f32_to_16_bits<F16>(v[0]);
    }
}

}  // namespace

hipError_t launch_gemm_w4(const W4Args &a, hipStream_t s) {
    if (a.M <= 0 || a.N <= 0) return hipSuccess;
    W4Params p;
    p.X = a.X; p.W = reinterpret_cast<const uint8_t *>(a.W); p.scales = a.scales; p.zeros = a.zeros;
    p.partials = a.partials; p.Y = a.Y;
    p.ldx = a.ldx; p.ldw = a.ldw; p.lds = a.lds; p.ldz = a.ldz; p.ldy = a.ldy;
    p.M = a.M; p.N = a.N;
    p.y_f32 = a.y_dtype == TBIK_F32;
    p.group = a.group; p.superleaf = a.superleaf;
    p.leaves_per_shard = a.ns / a.P;
    p.leaves_per_wave = p.leaves_per_shard > W4_WAVES ? p.leaves_per_shard / W4_WAVES : 1;
    p.active_waves = p.leaves_per_shard > W4_WAVES ? W4_WAVES : p.leaves_per_shard;
    if (p.leaves_per_wave > 16) return hipErrorInvalidValue;
    auto launch = [&](auto kernel) {
        for (int64_t m0 = 0; m0 < a.M; m0 += 32 * 4096) {              // 4096 row tiles a launch
            W4Params q = p;
            q.M = (int)(a.M - m0 < 32 * 4096 ? a.M - m0 : 32 * 4096);
            q.X += m0 * a.ldx;
            if (q.Y) q.Y = static_cast<char *>(q.Y) + m0 * a.ldy * (p.y_f32 ? 4 : 2);
            hipLaunchKernelGGL(kernel, dim3((unsigned)((a.N + 31) / 32), (unsigned)((q.M + 31) / 32), (unsigned)a.P), dim3(64 * W4_WAVES), 0, s, q);
        }
    };
    const bool f16 = a.x_dtype == TBIK_F16, zeros = a.zeros != nullptr;
    if (a.group % 64 == 0) {
        if (zeros) launch(f16 ? gemm_w4_kernel<64, true, true> : gemm_w4_kernel<64, false, true>);
        else launch(f16 ? gemm_w4_kernel<64, true, false> : gemm_w4_kernel<64, false, false>);
    } else {
        if (zeros) launch(f16 ? gemm_w4_kernel<32, true, true> : gemm_w4_kernel<32, false, true>);
        else launch(f16 ? gemm_w4_kernel<32, true, false> : gemm_w4_kernel<32, false, false>);
    }
    return hipGetLastError();
}

}  // namespace tbik
