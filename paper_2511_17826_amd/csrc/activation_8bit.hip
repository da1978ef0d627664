// The gated activation (activation.hip) with an 8-bit output with scales: v = SiLU(gate) * up in fp32 as silu_mul() forms it, then 8 bits
// of v (eight_bit_rows.hpp) -- the operand of an 8-bit or microscaling down_proj.  HBM-bound: 4 bytes read and 1 written per element.
#include <algorithm>

#include "eight_bit_rows.hpp"

namespace tbik {

namespace {

template <bool F16>
__device__ __forceinline__ void activated(const Silu8Args &a, int64_t row, int64_t col, float (&v)[8]) {
    float g[8], u[8];
    unpack8<F16>(*reinterpret_cast<const uint4 *>(a.gate + row * a.ldg + col), g);
    unpack8<F16>(*reinterpret_cast<const uint4 *>(a.up + row * a.ldu + col), u);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = silu_mul(g[e], u[e]);
}

// Microscaling: a thread owns 8 consecutive channels, four consecutive threads a block of 32 (I % 32 == 0).
template <bool F16>
__global__ __launch_bounds__(256) void silu_mul_mx_kernel(const Silu8Args a) {
    const int64_t per_row = a.I >> 3, total = a.M * per_row, stride = (int64_t)gridDim.x * blockDim.x;
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < total; i += stride) {
        const int64_t row = i / per_row, c = i - row * per_row;
        float v[8];
        activated<F16>(a, row, c * 8, v);
        const int byte = block_scale_byte(block_max(largest_magnitude(v)), a.out.e5m2);
        *reinterpret_cast<uint2 *>(a.out.q + row * a.out.ldq + c * 8) = to_8_bits(v, block_factor(byte), a.out.e5m2);
        if ((c & 3) == 0) reinterpret_cast<uint8_t *>(a.out.scales)[row * a.out.lds + (c >> 2)] = (uint8_t)byte;
    }
}

// A scale per row: a workgroup owns a row and keeps its values in registers between the maximum and the output.
template <bool F16, int THREADS, int CPL>
__global__ __launch_bounds__(THREADS) void silu_mul_row_kernel(const Silu8Args a) {
    const int64_t row = blockIdx.x;
    const int per_row = a.I >> 3;
    __shared__ float maxima[THREADS / 64];
    float v[CPL][8], amax = 0.0f;
#pragma unroll
    for (int s = 0; s < CPL; ++s) {
        const int c = s * THREADS + threadIdx.x;
        if (c < per_row) {
            activated<F16>(a, row, (int64_t)c * 8, v[s]);
            amax = fmaxf(amax, largest_magnitude(v[s]));
        }
    }
    amax = wave_max(amax);
    if ((threadIdx.x & 63) == 0) maxima[threadIdx.x >> 6] = amax;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < THREADS / 64; ++i) amax = fmaxf(amax, maxima[i]);
    const float scale = row_scale_of(amax, a.out.e5m2), factor = 1.0f / scale;
#pragma unroll
    for (int s = 0; s < CPL; ++s) {
        const int c = s * THREADS + threadIdx.x;
        if (c < per_row) *reinterpret_cast<uint2 *>(a.out.q + row * a.out.ldq + (int64_t)c * 8) = to_8_bits(v[s], factor, a.out.e5m2);
    }
    if (threadIdx.x == 0) reinterpret_cast<float *>(a.out.scales)[row] = scale;
}

template <bool F16>
hipError_t launch_of(const Silu8Args &a, hipStream_t s) {
    if (a.out.micro) {
        int64_t blocks = ((int64_t)a.M * (a.I / 8) + 255) / 256;
        if (blocks > 256 * 64) blocks = 256 * 64;
        hipLaunchKernelGGL(silu_mul_mx_kernel<F16>, dim3((unsigned)blocks), dim3(256), 0, s, a);
    } else if (a.I <= 8 * 256 * 2) {          // two chunks of 8 per thread where a workgroup has threads enough: 4096 x 14336 51.9 us, 512 x 4 53.4, 256 x 8 56.7
        hipLaunchKernelGGL((silu_mul_row_kernel<F16, 256, 2>), dim3((unsigned)a.M), dim3(256), 0, s, a);
    } else if (a.I <= 8 * 512 * 2) {
        hipLaunchKernelGGL((silu_mul_row_kernel<F16, 512, 2>), dim3((unsigned)a.M), dim3(512), 0, s, a);
    } else if (a.I <= 8 * 1024 * 2) {
        hipLaunchKernelGGL((silu_mul_row_kernel<F16, 1024, 2>), dim3((unsigned)a.M), dim3(1024), 0, s, a);
    } else if (a.I <= 8 * 1024 * 4) {
        hipLaunchKernelGGL((silu_mul_row_kernel<F16, 1024, 4>), dim3((unsigned)a.M), dim3(1024), 0, s, a);
    } else {
        hipLaunchKernelGGL((silu_mul_row_kernel<F16, 1024, 8>), dim3((unsigned)a.M), dim3(1024), 0, s, a);
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_silu_mul_8bit(const Silu8Args &all, int dtype, hipStream_t s) {
    const int64_t most = all.out.micro ? all.M : kRowsOfALaunch;        // (a loop over the elements, or a workgroup per row)
    for (int64_t m = 0; m < all.M && all.I > 0; m += most) {
        const Silu8Args a{all.gate + m * all.ldg, all.ldg, all.up + m * all.ldu, all.ldu, all.out.from_row(m), std::min(most, all.M - m), all.I};
        const hipError_t e = dtype == TBIK_F16 ? launch_of<true>(a, s) : launch_of<false>(a, s);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace tbik
