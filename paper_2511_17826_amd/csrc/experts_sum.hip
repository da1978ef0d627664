// The weighted sum of a token's experts, the residual added: out[t] = sum_j weights[t, j] y[slots[t, j]] (+ residual[t]).
//
// Element by element the sum is one chain of fused multiply-adds in fp32 from +0, j ascending, whatever the batch.  y is the 16-bit
// output of the experts' second product or the fp32 partial sums of P shards of it (then y = T(partials), the top of the tree, as
// tbik_tree_combine forms it, and the result does not depend on P).  A choice whose slot is no row of y adds nothing.
//
// Bound by HBM: k rows read and one written per token, the reads gathered but whole rows.  A thread holds 8 consecutive columns and
// has the rows of up to 8 choices on their way before it adds the first (fp32 sums of P shards: 8 / P choices); slots and weights are
// the workgroup's (one token), in scalar registers.
#include <algorithm>

#include "tbik_device.hpp"
#include "tbik_internal.hpp"

namespace tbik {

namespace {

struct SumParams {
    const void *y;                 // 16-bit [R, ldy], or fp32 [P, R, H] dense
    int64_t ldy, plane;
    const int32_t *slots;          // [T, k]
    const float *weights;          // [T, k]
    const void *residual;          // [T, ldr] of the output's type, or nullptr
    int64_t ldr;
    void *out;                     // [T, ldo]
    int64_t ldo;
    int R, H, k;
};

typedef unsigned int sum_u32x4 __attribute__((ext_vector_type(4)));

// y of 8 consecutive columns as it lies in memory, and widened.
template <int P>
struct Piece {
    f32x4 lo[P], hi[P];
    __device__ __forceinline__ void load(const SumParams &p, int64_t row, int col) {
        const float *src = reinterpret_cast<const float *>(p.y) + row * p.ldy + col;
#pragma unroll
        for (int q = 0; q < P; ++q) {
            lo[q] = *reinterpret_cast<const f32x4 *>(src + q * p.plane);
            hi[q] = *reinterpret_cast<const f32x4 *>(src + q * p.plane + 4);
        }
    }
    template <bool F16>
    __device__ __forceinline__ void widen(float (&v)[8]) const {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float u[P];
#pragma unroll
            for (int q = 0; q < P; ++q) u[q] = e < 4 ? lo[q][e & 3] : hi[q][e & 3];
            v[e] = tree_of<P>(u);
        }
    }
};
template <>
struct Piece<0> {
    uint4 raw;
    __device__ __forceinline__ void load(const SumParams &p, int64_t row, int col) {
        raw = *reinterpret_cast<const uint4 *>(reinterpret_cast<const uint16_t *>(p.y) + row * p.ldy + col);
    }
    template <bool F16>
    __device__ __forceinline__ void widen(float (&v)[8]) const { unpack8<F16>(raw, v); }
};

// P: 0 for 16-bit rows.  F16: of the rows and a 16-bit output.  WIDE: fp32 output.
template <int P, bool F16, bool WIDE>
__global__ __launch_bounds__(256) void experts_sum_kernel(const SumParams p) {
    const int64_t t = blockIdx.y;
    if ((blockIdx.x * 256u + threadIdx.x) * 8u >= (unsigned)p.H) return;       // up to 2^31 + 2047: not an int
    const int col = (blockIdx.x * 256 + threadIdx.x) * 8;
    // us with 1 / 2 / 4 / 8 choices ahead, 8 chosen of 4096 columns: 16-bit rows, one token 3.65 / 3.47 / 3.30 / 3.25, 77 tokens 5.93 / 5.82 / 5.64 / 5.53; P = 1, 77 tokens
    // 6.37 / 5.54 / 5.06 / 4.89; P = 2, one token 5.33 / 4.90 / 4.77 / 4.72, 1000 52.2 / 52.2 / 52.6 / 54.0; P = 4, one 6.70 / 6.39 / 6.15 / 6.05, 1000 98.3 / 98.4 /
    // 98.3 / 101.5; P = 8, 77 21.7 / 18.3 / 18.7 / -, 300 of 2 chosen 19.0 / 18.8 / 21.4 / -; P = 16, 77 35.7 / 33.1 / - / -, 300 of 2 chosen 32.9 / 35.8 / - / -.
    constexpr int AHEAD = P <= 1 ? 8 : P == 2 ? 4 : P == 4 ? 2 : 1;
    const int32_t *const slots = p.slots + t * p.k;
    const float *const weights = p.weights + t * p.k;
    float r[8];
    if (p.residual) {                                  // on its way with the first rows
        if constexpr (WIDE) {
            const float *src = reinterpret_cast<const float *>(p.residual) + t * p.ldr + col;
            const f32x4 a = *reinterpret_cast<const f32x4 *>(src), b = *reinterpret_cast<const f32x4 *>(src + 4);
#pragma unroll
            for (int e = 0; e < 8; ++e) r[e] = e < 4 ? a[e & 3] : b[e & 3];
        } else {
            unpack8<F16>(*reinterpret_cast<const uint4 *>(reinterpret_cast<const uint16_t *>(p.residual) + t * p.ldr + col), r);
        }
    }
    float acc[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
    for (int j0 = 0; j0 < p.k; j0 += AHEAD) {
        Piece<P> piece[AHEAD];
        int slot[AHEAD];
        float w[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            slot[i] = j0 + i < p.k ? slots[j0 + i] : -1;
            w[i] = j0 + i < p.k ? weights[j0 + i] : 0.0f;
        }
#pragma unroll
        for (int i = 0; i < AHEAD; ++i)
            if ((unsigned)slot[i] < (unsigned)p.R) piece[i].load(p, slot[i], col);
#pragma unroll
        for (int i = 0; i < AHEAD; ++i)
            if ((unsigned)slot[i] < (unsigned)p.R) {
                float v[8];
                piece[i].template widen<F16>(v);
#pragma unroll
                for (int e = 0; e < 8; ++e) acc[e] = __builtin_fmaf(w[i], v[e], acc[e]);
            }
    }
    if (p.residual) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            acc[e] = acc[e] + r[e];
            asm("" : "+v"(acc[e]));                    // a value of its own: no merging with the rounding (see silu_mul)
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) asm("" : "+v"(acc[e]));
    }
    if constexpr (WIDE) {
        float *dst = reinterpret_cast<float *>(p.out) + t * p.ldo + col;
        *reinterpret_cast<f32x4 *>(dst) = f32x4{acc[0], acc[1], acc[2], acc[3]};
        *reinterpret_cast<f32x4 *>(dst + 4) = f32x4{acc[4], acc[5], acc[6], acc[7]};
    } else {
        *reinterpret_cast<uint4 *>(reinterpret_cast<uint16_t *>(p.out) + t * p.ldo + col) =
            make_uint4(pack_16x2<F16>(acc[0], acc[1]), pack_16x2<F16>(acc[2], acc[3]), pack_16x2<F16>(acc[4], acc[5]), pack_16x2<F16>(acc[6], acc[7]));
    }
}

// Rows that cannot be read 16 bytes at a time: an element per thread, the same arithmetic.
template <bool F16>
__device__ __forceinline__ float element_16(const void *p, int64_t i) {
    const uint16_t h = reinterpret_cast<const uint16_t *>(p)[i];
    return F16 ? (float)__builtin_bit_cast(_Float16, h) : bf16_bits_to_f32(h);
}
template <int P, bool F16, bool WIDE>
__global__ __launch_bounds__(256) void experts_sum_element_kernel(const SumParams p) {
    const int64_t t = blockIdx.y;
    if (blockIdx.x * 256u + threadIdx.x >= (unsigned)p.H) return;
    const int col = blockIdx.x * 256 + threadIdx.x;
    float acc = 0.0f;
    for (int j = 0; j < p.k; ++j) {
        const int slot = p.slots[t * p.k + j];
        if ((unsigned)slot >= (unsigned)p.R) continue;
        float y;
        if constexpr (P == 0) {
            y = element_16<F16>(p.y, slot * p.ldy + col);
        } else {
            float u[P > 0 ? P : 1];
#pragma unroll
            for (int q = 0; q < P; ++q) u[q] = reinterpret_cast<const float *>(p.y)[slot * p.ldy + col + q * p.plane];
            y = tree_of<P>(u);
        }
        acc = __builtin_fmaf(p.weights[t * p.k + j], y, acc);
    }
    if (p.residual) acc = acc + (WIDE ? reinterpret_cast<const float *>(p.residual)[t * p.ldr + col] : element_16<F16>(p.residual, t * p.ldr + col));
    asm("" : "+v"(acc));
    if constexpr (WIDE) reinterpret_cast<float *>(p.out)[t * p.ldo + col] = acc;
    else reinterpret_cast<uint16_t *>(p.out)[t * p.ldo + col] = (uint16_t)f32_to_16_bits<F16>(acc);
}

template <int P, bool F16, bool WIDE>
void launch_sum(const SumParams &p, int T, bool vector, hipStream_t s) {
    const int64_t blocks = ((int64_t)p.H + (vector ? 2047 : 255)) / (vector ? 2048 : 256);
    // A grid has fewer than 2^32 threads: 16384 tokens a launch, fewer of rows of more than 2^18 columns (2^21 of eight a thread).
    const int64_t most = std::max<int64_t>(1, std::min<int64_t>(16384, (1 << 24) / blocks - 1));
    for (int64_t t0 = 0; t0 < T; t0 += most) {
        SumParams q = p;
        const int tokens = (int)std::min(T - t0, most);
        q.slots += t0 * p.k;
        q.weights += t0 * p.k;
        if (q.residual) q.residual = static_cast<const char *>(q.residual) + t0 * p.ldr * (WIDE ? 4 : 2);
        q.out = static_cast<char *>(q.out) + t0 * p.ldo * (WIDE ? 4 : 2);
        const dim3 grid((unsigned)blocks, (unsigned)tokens);
        if (vector) hipLaunchKernelGGL((experts_sum_kernel<P, F16, WIDE>), grid, dim3(256), 0, s, q);
        else hipLaunchKernelGGL((experts_sum_element_kernel<P, F16, WIDE>), grid, dim3(256), 0, s, q);
    }
}
template <bool F16, bool WIDE>
hipError_t launch_sum_of(const SumParams &p, int P, int T, bool vector, hipStream_t s) {
    switch (P) {
        case 0: launch_sum<0, F16, WIDE>(p, T, vector, s); break;
        case 1: launch_sum<1, F16, WIDE>(p, T, vector, s); break;
        case 2: launch_sum<2, F16, WIDE>(p, T, vector, s); break;
        case 4: launch_sum<4, F16, WIDE>(p, T, vector, s); break;
        case 8: launch_sum<8, F16, WIDE>(p, T, vector, s); break;
        case 16: launch_sum<16, F16, WIDE>(p, T, vector, s); break;
        default: return hipErrorInvalidValue;
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_experts_sum(const ExpertsSumArgs &a, hipStream_t s) {
    if (a.T <= 0 || a.H <= 0) return hipSuccess;
    SumParams p{a.y, a.P ? a.H : a.ldy, (int64_t)a.R * a.H, a.slots, a.weights, a.residual, a.ldr, a.out, a.ldo, a.R, a.H, a.k};
    const bool wide = a.out_dtype == TBIK_F32;
    const auto a16 = [](const void *q) { return (reinterpret_cast<uintptr_t>(q) & 15) == 0; };
    const int lanes = wide ? 4 : 8;
    const bool vector = a.H % 8 == 0 && a16(a.y) && a16(a.out) && (!a.residual || a16(a.residual)) && a.ldo % lanes == 0 && (!a.residual || a.ldr % lanes == 0) && (a.P || a.ldy % 8 == 0);
    const bool f16 = (a.P ? a.out_dtype : a.y_dtype) == TBIK_F16;
    if (wide) return f16 ? launch_sum_of<true, true>(p, a.P, a.T, vector, s) : launch_sum_of<false, true>(p, a.P, a.T, vector, s);
    return f16 ? launch_sum_of<true, false>(p, a.P, a.T, vector, s) : launch_sum_of<false, false>(p, a.P, a.T, vector, s);
}

}  // namespace tbik
