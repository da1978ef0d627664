// RMSNorm with the residual's addition and an 8-bit output with scales, the operand of the 8-bit and microscaling products:
//   h = x, or r16(x + residual), or r16(r16(T(partials)) + residual)     stored as the residual stream where there is a residual
//   n_i = (h_i r) w_i,   r = 1 / sqrt(TreeSum(h^2) / H + eps)            the fp32 value that tbik_rmsnorm rounds, same order
//   q, scales = 8 bits of n                                            eight_bit_rows.hpp
// HBM-bound: per element 2 bytes of x (4 P of partials), 2 + 2 of residual and h, 1 written.  A row stays in registers as 16-bit
// values between the sum of squares and the output, so it is read once.
#include <algorithm>

#include "eight_bit_rows.hpp"

namespace tbik {

namespace {

constexpr int MAX_SEGMENTS = 128;       // of 64 leaves of 8 elements: 65536 columns

// WAVES wavefronts per row (WAVES == 1: four rows per workgroup), CPL chunks of 8 elements per lane; segment s of the row's
// tree (64 consecutive leaves) belongs to wavefront s % WAVES.  P: planes of partial sums, 0: x is 16-bit.
template <bool F16, int P, int WAVES, int CPL>
__global__ __launch_bounds__(WAVES == 1 ? 256 : 64 * WAVES) void rmsnorm_8bit_kernel(const Rms8Args a, int nseg2) {
    constexpr int ROWS = WAVES == 1 ? 4 : 1;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t row = (int64_t)blockIdx.x * ROWS + (WAVES == 1 ? wave : 0);
    if (row >= a.M) return;             // WAVES == 1: whole wavefronts; else never
    const int w = WAVES == 1 ? 0 : wave;
    const int nchunks = a.H >> 3;
    const uint4 *const weight = reinterpret_cast<const uint4 *>(a.weight);
    __shared__ float sums[WAVES == 1 ? 1 : MAX_SEGMENTS];
    __shared__ float maxima[WAVES];

    uint4 h[CPL];
#pragma unroll
    for (int s = 0; s < CPL; ++s) {
        const int c = (s * WAVES + w) * 64 + lane;
        h[s] = make_uint4(0, 0, 0, 0);
        if (c < nchunks) {
            if constexpr (P == 0) {
                h[s] = *reinterpret_cast<const uint4 *>(a.x + row * a.ldx + c * 8);
            } else {
                const float *src = a.partials + row * a.H + c * 8;
                float y[8];
                // Eight columns of 16 planes are 128 registers, all that a thread of 1024 has: eight planes at a time there, half of the tree
                // each (256 x 32768 with all 16, three registers spilled, 134 -> 114 us; 16 x 65536, 47 spilled, 82 -> 56; with four
                // columns of all 16 at a time, half a cache line per load, 155 and 72).
                constexpr int AT_ONCE = P > 8 && WAVES == 16 && CPL > 2 ? 8 : P;
#pragma unroll
                for (int first = 0; first < P; first += AT_ONCE) {
                    f32x4 in[2][AT_ONCE];
#pragma unroll
                    for (int p = 0; p < AT_ONCE; ++p) {
                        in[0][p] = *reinterpret_cast<const f32x4 *>(src + (first + p) * a.plane);
                        in[1][p] = *reinterpret_cast<const f32x4 *>(src + (first + p) * a.plane + 4);
                    }
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        float v[AT_ONCE];
#pragma unroll
                        for (int p = 0; p < AT_ONCE; ++p) v[p] = in[e >> 2][p][e & 3];
                        const float t = tree_of<AT_ONCE>(v);
                        y[e] = first == 0 ? t : y[e] + t;
                    }
                    if (AT_ONCE < P) __builtin_amdgcn_sched_barrier(0);
                }
                h[s] = make_uint4(pack_16x2<F16>(y[0], y[1]), pack_16x2<F16>(y[2], y[3]), pack_16x2<F16>(y[4], y[5]), pack_16x2<F16>(y[6], y[7]));
            }
            if (a.residual) {
                float f[8], r[8];
                unpack8<F16>(h[s], f);
                unpack8<F16>(*reinterpret_cast<const uint4 *>(a.residual + row * a.ldr + c * 8), r);
#pragma unroll
                for (int e = 0; e < 8; ++e) f[e] = f[e] + r[e];
                h[s] = make_uint4(pack_16x2<F16>(f[0], f[1]), pack_16x2<F16>(f[2], f[3]), pack_16x2<F16>(f[4], f[5]), pack_16x2<F16>(f[6], f[7]));
                *reinterpret_cast<uint4 *>(a.hidden + row * a.ldh + c * 8) = h[s];
            }
        }
    }
    TreeStash<8> st;
    float ss = 0.0f;
#pragma unroll
    for (int s = 0; s < CPL; ++s) {
        float f[8], leaf = 0.0f;
        unpack8<F16>(h[s], f);              // a chunk past the row is all +0: its leaf is +0
#pragma unroll
        for (int e = 0; e < 8; ++e) leaf = leaf + f[e] * f[e];
        const float sum = wave_tree_sum(leaf);
        if constexpr (WAVES == 1) {
            if (s < nseg2) ss = st.push(sum, (unsigned)s);
        } else if (lane == 0) {
            sums[s * WAVES + w] = sum;
        }
    }
    if constexpr (WAVES == 1) {
        for (int s = CPL; s < nseg2; ++s) ss = st.push(0.0f, (unsigned)s);       // padding segments: T of +0 leaves
    } else {
        __syncthreads();
        // T over the segments, padded with +0 to 64 (or 128): adding +0 changes nothing
        ss = wave_tree_sum(lane < WAVES * CPL ? sums[lane] : 0.0f);
        if (WAVES * CPL > 64) ss = ss + wave_tree_sum(sums[64 + lane]);
    }
    const float r = 1.0f / sqrtf(ss / (float)a.H + a.eps);
    auto normed = [&](int s, int c, float (&n)[8]) __attribute__((always_inline)) {
        float f[8], g[8];
        unpack8<F16>(h[s], f);
        unpack8<F16>(weight[c], g);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float t = f[e] * r;
            n[e] = t * g[e];
        }
    };
    uint8_t *const q = a.out.q + row * a.out.ldq;
    if (a.out.micro) {
        uint8_t *const scales = reinterpret_cast<uint8_t *>(a.out.scales) + row * a.out.lds;
#pragma unroll
        for (int s = 0; s < CPL; ++s) {
            const int c = (s * WAVES + w) * 64 + lane;
            if (c < nchunks) {              // whole blocks of four lanes: H % 32 == 0
                float n[8];
                normed(s, c, n);
                const int byte = block_scale_byte(block_max(largest_magnitude(n)), a.out.e5m2);
                *reinterpret_cast<uint2 *>(q + c * 8) = to_8_bits(n, block_factor(byte), a.out.e5m2);
                if ((lane & 3) == 0) scales[c >> 2] = (uint8_t)byte;
            }
        }
    } else {
        constexpr int KEPT = CPL <= 4 ? CPL : 1;               // few values are kept between the maximum and the output, many formed again
        float amax = 0.0f, n[KEPT][8];
#pragma unroll
        for (int s = 0; s < CPL; ++s) {
            const int c = (s * WAVES + w) * 64 + lane;
            if (c < nchunks) {
                normed(s, c, n[s % KEPT]);
                amax = fmaxf(amax, largest_magnitude(n[s % KEPT]));
            }
        }
        amax = wave_max(amax);
        if constexpr (WAVES > 1) {
            if (lane == 0) maxima[w] = amax;
            __syncthreads();
#pragma unroll
            for (int i = 0; i < WAVES; ++i) amax = fmaxf(amax, maxima[i]);
        }
        const float scale = row_scale_of(amax, a.out.e5m2), factor = 1.0f / scale;
#pragma unroll
        for (int s = 0; s < CPL; ++s) {
            const int c = (s * WAVES + w) * 64 + lane;
            if (c < nchunks) {
                if constexpr (KEPT < CPL) normed(s, c, n[0]);
                *reinterpret_cast<uint2 *>(q + c * 8) = to_8_bits(n[s % KEPT], factor, a.out.e5m2);
            }
        }
        if (w == 0 && lane == 0) reinterpret_cast<float *>(a.out.scales)[row] = scale;
    }
}

template <bool F16, int P>
hipError_t launch_p(const Rms8Args &a, hipStream_t s) {
    const int nchunks = a.H / 8, segments = (nchunks + 63) / 64;
    int n2 = 1;
    while (n2 < nchunks) n2 *= 2;
    const int nseg2 = n2 < 64 ? 1 : n2 / 64;
    auto rows_of_a_wavefront = [&](auto k) { hipLaunchKernelGGL(k, dim3((a.M + 3) / 4), dim3(256), 0, s, a, nseg2); };
    auto rows_of = [&](auto k, int waves) { hipLaunchKernelGGL(k, dim3(a.M), dim3(64 * waves), 0, s, a, nseg2); };
    // Few chunks per lane: a row is one pass of load, sum, output, and what hides its latencies is the number of wavefronts.  Up to
    // 1024 columns a wavefront takes a row alone; many 16-bit rows of up to 6144 take four, which leaves fewer of them at the barriers
    // than eight; partial sums are P times the loads and take eight.  us, wavefronts x chunks, bf16 with residual:
    //   1 x 4096          8x1 2.7   4x2 3.2   1x8 6.5          512 x 4096     8x1 4.5   4x2 4.7   1x8 9.3
    //   8192 x 4096       8x1 43.2  4x2 40.0  1x8 49.0         8191 x 5120    8x2 54.3  4x3 50.6  1x10 67.0      4096 x 1024  4x1 8.9  1x2 7.7
    //   1003 x 4096, P 4  8x1 14.1  4x2 14.7  1x8 17.7         1024 x 16384   16x2 20.9 8x4 22.9                 2048 x 512   4x1 3.8  1x2 3.2
    // Where four begin to pay is near two rows per compute unit (six sets of operands in turn):
    //   rows of 4096      256  8x1 3.7   4x2 4.1     512  5.7  5.6     640  6.9  6.5     896   8.2  7.6     2048  13.2  12.6
    //   rows of 5120      256  8x2 4.7   4x3 5.4     512  6.5  6.5     640  7.8  7.4     896   9.3  8.7     2048  16.9  15.8
    // (8191 x 5120: 5.8 TB/s of the bytes that have to move, a copy of 1 GiB reaches 5.1.)
    if constexpr (P == 0) {
        if (a.M > 512 && segments > 2 && segments <= 12) {
            if (segments <= 8) rows_of(rmsnorm_8bit_kernel<F16, P, 4, 2>, 4);
            else rows_of(rmsnorm_8bit_kernel<F16, P, 4, 3>, 4);
            return hipGetLastError();
        }
    }
    if (segments <= 2) rows_of_a_wavefront(rmsnorm_8bit_kernel<F16, P, 1, 2>);
    else if (segments <= 8) rows_of(rmsnorm_8bit_kernel<F16, P, 8, 1>, 8);
    else if (segments <= 16) rows_of(rmsnorm_8bit_kernel<F16, P, 8, 2>, 8);
    else if (segments <= 32) rows_of(rmsnorm_8bit_kernel<F16, P, 16, 2>, 16);
    else if (segments <= 64) rows_of(rmsnorm_8bit_kernel<F16, P, 16, 4>, 16);
    else rows_of(rmsnorm_8bit_kernel<F16, P, 16, 8>, 16);
    return hipGetLastError();
}

template <bool F16>
hipError_t launch_of(const Rms8Args &a, hipStream_t s) {
    switch (a.P) {
        case 0: return launch_p<F16, 0>(a, s);
        case 1: return launch_p<F16, 1>(a, s);
        case 2: return launch_p<F16, 2>(a, s);
        case 4: return launch_p<F16, 4>(a, s);
        case 8: return launch_p<F16, 8>(a, s);
        case 16: return launch_p<F16, 16>(a, s);
        default: return hipErrorInvalidValue;
    }
}

}  // namespace

hipError_t launch_rmsnorm_8bit(const Rms8Args &all, int dtype, hipStream_t s) {
    for (int64_t m = 0; m < all.M; m += kRowsOfALaunch) {
        Rms8Args a = all;
        a.M = (int)std::min<int64_t>(kRowsOfALaunch, all.M - m);
        if (a.x) a.x += m * a.ldx;
        if (a.partials) a.partials += m * a.H;
        if (a.residual) {
            a.residual += m * a.ldr;
            a.hidden += m * a.ldh;
        }
        a.out = all.out.from_row(m);
        const hipError_t e = dtype == TBIK_F16 ? launch_of<true>(a, s) : launch_of<false>(a, s);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace tbik
