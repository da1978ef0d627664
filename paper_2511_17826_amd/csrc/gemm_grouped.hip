// Products grouped by expert (16-bit operands): the reference kernel, which takes what the slices and tiles do not (grouped_kernel in tbik_api.hip).
//
//   Y[i] = X[rows[i]] W[e]   for the rows i of group e          each row's sum in the order of tbik_gemm (Sec. 4.2, App. D.1)
//
// The bits of a row are those of tbik_gemm on that row and its expert's weight: the same matrix instruction over the same k, the
// same chains, the same tree.
#include "grouped.hpp"

namespace tbik {

namespace {

// A row tile's 32 x 32 sums, lane and register as the 32x32 matrix instruction leaves them: row of register r.
__device__ __forceinline__ int row_of_register(int r, int lane) { return 8 * (r >> 2) + 4 * (lane >> 5) + (r & 3); }

template <bool F16>
__device__ __forceinline__ void store_element(const GroupedArgs &a, int shard, int row, int col, float v) {
    if (a.partials) a.partials[((int64_t)shard * a.M + row) * a.N + col] = v;
    else if (a.y_dtype == TBIK_F32) reinterpret_cast<float *>(a.Y)[(int64_t)row * a.ldy + col] = v;
    else reinterpret_cast<uint16_t *>(a.Y)[(int64_t)row * a.ldy + col] = (uint16_t)f32_to_16_bits<F16>(v);
}

// One wavefront per 32 x 32 tile and shard, operands straight from global memory (see gemm_reference.hip).  With the activation a
// wavefront computes the gate's tile and the up projection's.
template <bool F16>
__global__ __launch_bounds__(64) void gemm_grouped_reference_kernel(const GroupedArgs a, int row_tiles) {
    const int lane = threadIdx.x, i = lane & 31, g = lane >> 5;
    GroupMap<32> map;
    map.read(a.offsets, a.groups, a.M, lane);
    const int columns = a.swiglu ? a.N / 2 : a.N, n0 = blockIdx.x * 32, ns = a.ns / a.P;
    const int64_t kbase = (int64_t)blockIdx.z * ns * a.superleaf;
    for (int tile = blockIdx.y; tile < map.tiles; tile += row_tiles) {
        const GroupRows at = map.at(tile);
        const bool row_ok = at.first + i < at.end, col_ok = n0 + i < columns;
        const uint16_t *xrow = a.X + (int64_t)source_row(a.rows, row_ok ? at.first + i : at.first, a.tokens) * a.ldx;
        float gate[16];
        for (int half = 0; half <= a.swiglu; ++half) {
            const uint16_t *wcol = a.W + at.group * a.weight_stride + n0 + i + (half ? columns : 0);
            float stash[28][16];
            f32x16 acc;
            for (int j = 0; j < ns; ++j) {
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[r] = 0.0f;
                for (int kk = 0; kk < a.superleaf; kk += 16) {
                    const int64_t k = kbase + (int64_t)j * a.superleaf + kk + 8 * g;
                    union { uint4 u; bf16x8 v; } x, w;
                    x.u = make_uint4(0, 0, 0, 0);
                    if (row_ok) x.u = *reinterpret_cast<const uint4 *>(xrow + k);
                    uint32_t c[8];
#pragma unroll
                    for (int t = 0; t < 8; ++t) c[t] = col_ok ? (uint32_t)wcol[(k + t) * a.ldw] : 0u;
                    w.u = make_uint4(c[0] | (c[1] << 16), c[2] | (c[3] << 16), c[4] | (c[5] << 16), c[6] | (c[7] << 16));
                    acc = mfma_32x32x16<F16>(x.v, w.v, acc);
                }
                const int t = __builtin_ctz(~(unsigned)j);      // the carry-over step of the tree
                for (int l = 0; l < t; ++l) {
#pragma unroll
                    for (int r = 0; r < 16; ++r) acc[r] = stash[l][r] + acc[r];
                }
                if (j + 1 < ns) {
#pragma unroll
                    for (int r = 0; r < 16; ++r) stash[t][r] = acc[r];
                }
            }
            if (a.swiglu && half == 0) {
#pragma unroll
                for (int r = 0; r < 16; ++r) gate[r] = through_16_bits<F16>(acc[r]);
                continue;
            }
            if (!col_ok) continue;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int row = at.first + row_of_register(r, lane);
                if (row < at.end) store_element<F16>(a, blockIdx.z, row, n0 + i, a.swiglu ? silu_mul(gate[r], through_16_bits<F16>(acc[r])) : acc[r]);
            }
        }
    }
}

}  // namespace

hipError_t launch_gemm_grouped_reference(const GroupedArgs &a, hipStream_t s) {
    if (a.M <= 0 || a.N <= 0) return hipSuccess;
    const int columns = a.swiglu ? a.N / 2 : a.N;
    const int64_t most = (int64_t)a.M / 32 + a.groups;           // row tiles of any division of the rows
    const int row_tiles = (int)(most < 4096 ? most : 4096);
    const dim3 grid((unsigned)((columns + 31) / 32), (unsigned)row_tiles, (unsigned)a.P);
    if (a.x_dtype == TBIK_F16) hipLaunchKernelGGL(gemm_grouped_reference_kernel<true>, grid, dim3(64), 0, s, a, row_tiles);
    else hipLaunchKernelGGL(gemm_grouped_reference_kernel<false>, grid, dim3(64), 0, s, a, row_tiles);
    return hipGetLastError();
}

}  // namespace tbik
