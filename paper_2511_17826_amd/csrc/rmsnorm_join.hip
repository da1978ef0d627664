// What joins one block of a decoder layer to the next, where a norm follows the block as well as preceding it:
//   n      = RMSNorm(y; post_weight)                          fp32, not rounded (y itself without that weight)
//   hidden = r16( residual_scale * residual + gate * n )      each product and the sum one fp32 operation, one rounding
//   normed = RMSNorm(hidden; next_weight)                     exactly tbik_rmsnorm of hidden
// y is the block's 16-bit output, or r16(T(partials)) of P shards' partial sums as in tbik_combine_residual_rmsnorm.
//
// One workgroup owns one row, whatever M is.  Leaf c of a row's tree is the in-order fp32 sum of the squares of elements 8c .. 8c+7; a
// segment is 64 leaves, one wavefront's lanes; a wavefront owns every WAVES-th segment, whose sums meet in LDS, and each wavefront
// evaluates the upper levels of the tree over all segments for itself: the bits do not depend on the number of wavefronts, and
// are those of the norms on their own.  y, residual and gate are read once and the row stays in registers over both norms.
//
// Bound by HBM: y, residual (and a gate per element) read once, hidden and normed written once.
#include "tbik_device.hpp"
#include "tbik_internal.hpp"

namespace tbik {

namespace {

struct JoinParams {
    const uint16_t *y;             // [M, ldy], P == 0
    int64_t ldy;
    const float *partials;         // [P, M, H], rows ldy apart, planes `plane` apart
    int64_t plane;
    const uint16_t *residual;
    int64_t ldr;
    const uint16_t *post, *next;   // [H] or nullptr
    const uint16_t *gate;          // element (m, i) at m * gate_row + i * gate_column, or nullptr
    int64_t gate_row;
    int gate_column;               // 0 or 1
    uint16_t *hidden, *normed;
    int64_t ldh, ldn;
    float residual_scale, eps;
    int H, segments;
};

// T over the row's segments (+0 behind the last), from LDS: the lanes are the lower six levels.
template <bool MANY>
__device__ __forceinline__ float segments_tree(const float *sums, int segments, int lane) {
    const float low = wave_tree_sum(lane < segments ? sums[lane] : 0.0f);
    if constexpr (!MANY) return low;
    return low + wave_tree_sum(lane + 64 < segments ? sums[lane + 64] : 0.0f);
}

// PER_WAVE: segments of a wavefront.  P: 0 for 16-bit rows.
template <int P, int WAVES, int PER_WAVE, bool F16>
__global__ __launch_bounds__(64 * WAVES) void rmsnorm_join_kernel(const JoinParams p) {
    __shared__ float sums[2][WAVES * PER_WAVE];
    constexpr bool MANY = WAVES * PER_WAVE > 64;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t row = blockIdx.x;
    const int chunks = p.H >> 3;
    uint4 y[PER_WAVE], r[PER_WAVE];
#pragma unroll
    for (int i = 0; i < PER_WAVE; ++i) {
        const int c = (i * WAVES + wave) * 64 + lane;
        y[i] = r[i] = make_uint4(0, 0, 0, 0);
        if (c < chunks) {
            r[i] = *reinterpret_cast<const uint4 *>(p.residual + row * p.ldr + c * 8);
            if constexpr (P == 0) y[i] = *reinterpret_cast<const uint4 *>(p.y + row * p.ldy + c * 8);
            else {
                const float *src = p.partials + row * p.ldy + c * 8;
                // Sixteen planes of eight columns are 128 registers, all that a thread of 1024 has, and eight segments of y and of the residual are 64: eight
                // planes at a time, four beside eight segments, a half or a quarter of the tree each.  (Eight beside eight segments spill: 256 rows of 65536
                // columns, 16 planes 239 us, so 213, 8 planes 137 and 123; one row of 40000, 16 planes 36.6 and 35.2, 8 planes 21.5 and 22.3.)
                constexpr int AT_ONCE = P > 4 && PER_WAVE >= 8 ? 4 : P > 8 ? 8 : P, PARTS = P / AT_ONCE;
                float v[8], third[8];
#pragma unroll
                for (int part = 0; part < PARTS; ++part) {
                    f32x4 lo[AT_ONCE], hi[AT_ONCE];
#pragma unroll
                    for (int q = 0; q < AT_ONCE; ++q) {
                        lo[q] = *reinterpret_cast<const f32x4 *>(src + (part * AT_ONCE + q) * p.plane);
                        hi[q] = *reinterpret_cast<const f32x4 *>(src + (part * AT_ONCE + q) * p.plane + 4);
                    }
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        float u[AT_ONCE];
#pragma unroll
                        for (int q = 0; q < AT_ONCE; ++q) u[q] = e < 4 ? lo[q][e & 3] : hi[q][e & 3];
                        const float t = tree_of<AT_ONCE>(u);
                        if (part == 0) v[e] = t;
                        else if (PARTS == 4 && part == 2) third[e] = t;
                        else v[e] = v[e] + (part == 3 ? third[e] + t : t);
                    }
                }
                y[i] = make_uint4(pack_16x2<F16>(v[0], v[1]), pack_16x2<F16>(v[2], v[3]), pack_16x2<F16>(v[4], v[5]), pack_16x2<F16>(v[6], v[7]));
            }
        }
    }
    float scale = 0.0f;
    if (p.post) {                                      // uniform
#pragma unroll
        for (int i = 0; i < PER_WAVE; ++i) {
            float f[8], leaf = 0.0f;
            unpack8<F16>(y[i], f);
#pragma unroll
            for (int e = 0; e < 8; ++e) leaf = leaf + f[e] * f[e];
            leaf = wave_tree_sum(leaf);
            if (lane == 0) sums[0][i * WAVES + wave] = leaf;
        }
        __syncthreads();
        scale = 1.0f / sqrtf(segments_tree<MANY>(sums[0], p.segments, lane) / (float)p.H + p.eps);
    }
    // A gate per row is one value; per channel or element, eight.
    float row_gate = 1.0f;
    if (p.gate && p.gate_column == 0) {
        const uint16_t h = p.gate[row * p.gate_row];
        row_gate = F16 ? (float)__builtin_bit_cast(_Float16, h) : bf16_bits_to_f32(h);
    }
#pragma unroll
    for (int i = 0; i < PER_WAVE; ++i) {
        const int c = (i * WAVES + wave) * 64 + lane;
        if (c < chunks) {
            float f[8], x[8];
            unpack8<F16>(y[i], f);
            unpack8<F16>(r[i], x);
            if (p.post) {
                float w[8];
                unpack8<F16>(*reinterpret_cast<const uint4 *>(p.post + c * 8), w);
#pragma unroll
                for (int e = 0; e < 8; ++e) f[e] = (f[e] * scale) * w[e];
            }
            if (p.gate) {
                if (p.gate_column) {
                    float g[8];
                    unpack8<F16>(*reinterpret_cast<const uint4 *>(p.gate + row * p.gate_row + c * 8), g);
#pragma unroll
                    for (int e = 0; e < 8; ++e) f[e] = g[e] * f[e];
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) f[e] = row_gate * f[e];
                }
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                f[e] = x[e] * p.residual_scale + f[e];
                asm("" : "+v"(f[e]));                  // a value of its own: no merging with the rounding (see silu_mul)
            }
            y[i] = make_uint4(pack_16x2<F16>(f[0], f[1]), pack_16x2<F16>(f[2], f[3]), pack_16x2<F16>(f[4], f[5]), pack_16x2<F16>(f[6], f[7]));
            *reinterpret_cast<uint4 *>(p.hidden + row * p.ldh + c * 8) = y[i];
        }
    }
    if (!p.next) return;                               // uniform
#pragma unroll
    for (int i = 0; i < PER_WAVE; ++i) {
        float f[8], leaf = 0.0f;
        unpack8<F16>(y[i], f);                         // behind the row's end all +0: its leaf is +0
#pragma unroll
        for (int e = 0; e < 8; ++e) leaf = leaf + f[e] * f[e];
        leaf = wave_tree_sum(leaf);
        if (lane == 0) sums[1][i * WAVES + wave] = leaf;
    }
    __syncthreads();
    scale = 1.0f / sqrtf(segments_tree<MANY>(sums[1], p.segments, lane) / (float)p.H + p.eps);
#pragma unroll
    for (int i = 0; i < PER_WAVE; ++i) {
        const int c = (i * WAVES + wave) * 64 + lane;
        if (c < chunks) {
            float f[8], w[8];
            unpack8<F16>(y[i], f);
            unpack8<F16>(*reinterpret_cast<const uint4 *>(p.next + c * 8), w);
            float o[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                o[e] = (f[e] * scale) * w[e];
                asm("" : "+v"(o[e]));
            }
            *reinterpret_cast<uint4 *>(p.normed + row * p.ldn + c * 8) =
                make_uint4(pack_16x2<F16>(o[0], o[1]), pack_16x2<F16>(o[2], o[3]), pack_16x2<F16>(o[4], o[5]), pack_16x2<F16>(o[6], o[7]));
        }
    }
}

template <int P, int WAVES, int PER_WAVE, bool F16>
hipError_t launch_join(const JoinParams &p, int M, hipStream_t s) {
    hipLaunchKernelGGL((rmsnorm_join_kernel<P, WAVES, PER_WAVE, F16>), dim3((unsigned)M), dim3(64 * WAVES), 0, s, p);
    return hipGetLastError();
}
// One segment a wavefront while a row has up to ten, which is the quickest for few rows; two in eight wavefronts up to sixteen, which is that for many rows; beyond, sixteen
// wavefronts.  us, bf16, wavefronts x segments of each; rows 64 / 8191:
//   1024 columns  4 x 1 2.71 / 18.6, 8 x 1 2.69 / 25.7, 2 x 1 2.67 / 16.8       2048   4 x 1 2.90 / 27.3, 8 x 1 2.82 / 28.9, 2 x 2 3.53 / 27.7
//   4096          8 x 1 3.56 / 47.6, 8 x 2 3.99 / 49.0, 4 x 2 4.39 / 50.6       5120  10 x 1 3.91 / 67.4, 8 x 2 4.31 / 61.7, 16 x 1 3.88 / 68.8
//   6144          8 x 2 4.39 / 72.3, 12 x 1 3.96 / 78.6, 16 x 1 3.90 / 79.1     8192   8 x 2 4.77 / 98.7, 16 x 1 4.31 / 101.5, 4 x 4 6.21 / 104.3
//   16384        16 x 2 6.88 / 191, 8 x 4 7.54 / 196                           32768  16 x 4 11.1 / 404, 8 x 8 14.1 / 406
template <int P, bool F16>
hipError_t launch_join_rows(const JoinParams &p, int M, hipStream_t s) {
    if (p.segments <= 4) return launch_join<P, 4, 1, F16>(p, M, s);
    if (p.segments <= 8) return launch_join<P, 8, 1, F16>(p, M, s);
    if (p.segments <= 10) return launch_join<P, 10, 1, F16>(p, M, s);
    if (p.segments <= 16) return launch_join<P, 8, 2, F16>(p, M, s);
    if (p.segments <= 32) return launch_join<P, 16, 2, F16>(p, M, s);
    if (p.segments <= 64) return launch_join<P, 16, 4, F16>(p, M, s);
    return launch_join<P, 16, 8, F16>(p, M, s);
}
template <bool F16>
hipError_t launch_join_of(const JoinParams &p, int P, int M, hipStream_t s) {
    switch (P) {
        case 0: return launch_join_rows<0, F16>(p, M, s);
        case 1: return launch_join_rows<1, F16>(p, M, s);
        case 2: return launch_join_rows<2, F16>(p, M, s);
        case 4: return launch_join_rows<4, F16>(p, M, s);
        case 8: return launch_join_rows<8, F16>(p, M, s);
        case 16: return launch_join_rows<16, F16>(p, M, s);
        default: return hipErrorInvalidValue;
    }
}

}  // namespace

hipError_t launch_rmsnorm_join(const JoinArgs &a, hipStream_t s) {
    JoinParams p{a.y, a.ldy, a.partials, (int64_t)a.M * a.H, a.residual, a.ldr, a.post, a.next, a.gate, a.gate_row, a.gate_column,
                 a.hidden, a.normed, a.ldh, a.ldn, a.residual_scale, a.eps, a.H, (a.H / 8 + 63) / 64};
    if (a.P) p.ldy = a.H;
    for (int64_t m0 = 0; m0 < a.M; m0 += kRowsOfALaunch) {
        JoinParams q = p;
        if (a.P) q.partials += m0 * a.H;
        else q.y += m0 * p.ldy;
        q.residual += m0 * p.ldr;
        if (p.gate) q.gate += m0 * p.gate_row;
        q.hidden += m0 * p.ldh;
        if (p.normed) q.normed += m0 * p.ldn;
        const int m = (int)(a.M - m0 < kRowsOfALaunch ? a.M - m0 : kRowsOfALaunch);
        const hipError_t e = a.dtype == TBIK_F16 ? launch_join_of<true>(q, a.P, m, s) : launch_join_of<false>(q, a.P, m, s);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace tbik
