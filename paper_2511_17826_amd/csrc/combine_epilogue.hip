// The top-of-tree combine (combine.hip) with the epilogue of the matrix products between the sum and the rounding: what ends
// a K-split product with an epilogue, and a tensor-parallel layer's all-reduce with the bias, the activation and the residual
// that follow it.  HBM-bound: 4 P bytes of partial sums per element, the residual and the output.
#include "epilogue.hpp"

namespace tbik {

namespace {

// How a call's operands can be read: in pieces of 4 elements from aligned addresses, or one by one.
struct CombinePieces {
    int out, residual, bias, col_scale;
};

// Four consecutive elements of a vector or of a row as they lie in memory, and their values: all of a thread's loads are under way
// before the first is converted.
__device__ __forceinline__ f32x4 raw_4(const void *p, int64_t i, int dtype, int whole) {
    uint32_t q[4] = {0, 0, 0, 0};
    if (dtype == TBIK_F32) {
        const float *f = reinterpret_cast<const float *>(p) + i;
        return whole ? *reinterpret_cast<const f32x4 *>(f) : f32x4{f[0], f[1], f[2], f[3]};
    }
    const uint16_t *h = reinterpret_cast<const uint16_t *>(p) + i;
    if (whole) {
        const uint2 two = *reinterpret_cast<const uint2 *>(h);
        q[0] = two.x;
        q[1] = two.y;
    } else {
        q[0] = h[0] | (uint32_t)h[1] << 16;
        q[1] = h[2] | (uint32_t)h[3] << 16;
    }
    return f32x4{__uint_as_float(q[0]), __uint_as_float(q[1]), 0.0f, 0.0f};
}
__device__ __forceinline__ void values_4(const f32x4 &raw, int dtype, float (&v)[4]) {
    float w[8];
    const uint4 q = make_uint4(__float_as_uint(raw[0]), __float_as_uint(raw[1]), 0, 0);
    if (dtype == TBIK_F16) unpack8<true>(q, w);
    else unpack8<false>(q, w);
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = dtype == TBIK_F32 ? raw[k] : w[k];
}

// N % 4 == 0: a thread owns 4 consecutive columns of one row.  STREAM: the planes are read around the caches, as in combine.hip.
template <int P, bool STREAM>
__global__ __launch_bounds__(256) void tree_combine_epilogue_vec4_kernel(const float *__restrict__ partials, const EpilogueParams e, void *Y,
                                                                         int64_t ldy, int64_t M, int64_t N, const CombinePieces pieces) {
    const int64_t per_row = N >> 2, total = M * per_row, plane = M * N, stride = (int64_t)gridDim.x * blockDim.x;
    for (int64_t q = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; q < total; q += stride) {
        const int64_t row = total < (int64_t)1 << 31 ? (unsigned)q / (unsigned)per_row : q / per_row;      // the short division where it is enough
        const int64_t col = (q - row * per_row) << 2;
        const float *src = partials + row * N + col;
        f32x4 in[P];
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const f32x4 *ptr = reinterpret_cast<const f32x4 *>(src + (int64_t)p * plane);
            in[p] = STREAM ? __builtin_nontemporal_load(ptr) : *ptr;
        }
        f32x4 r_raw = {0, 0, 0, 0}, b_raw = {0, 0, 0, 0}, c_raw = {0, 0, 0, 0};
        float v[1][4], cs[4], b[4], r[4], rs[1] = {0.0f};
        if (e.residual) r_raw = raw_4(e.residual, row * e.ldr + col, e.y_dtype, pieces.residual);
        if (e.bias) b_raw = raw_4(e.bias, col, e.bias_dtype, pieces.bias);
        if (e.col_scale) c_raw = raw_4(e.col_scale, col, TBIK_F32, pieces.col_scale);
        if (e.row_scale) rs[0] = e.row_scale[row];
        values_4(r_raw, e.y_dtype, r);
        values_4(b_raw, e.bias_dtype, b);
        values_4(c_raw, TBIK_F32, cs);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float t[P];
#pragma unroll
            for (int p = 0; p < P; ++p) t[p] = in[p][i];
            v[0][i] = tree_of<P>(t);
        }
        scale_and_bias(e, v, rs, cs, b);
        activate(e.act, v);
        if (e.residual) add_residual(v[0], r);
        if (e.y_dtype == TBIK_F32) {
            float *dst = reinterpret_cast<float *>(Y) + row * ldy + col;
            if (pieces.out) *reinterpret_cast<f32x4 *>(dst) = f32x4{v[0][0], v[0][1], v[0][2], v[0][3]};
            else { dst[0] = v[0][0]; dst[1] = v[0][1]; dst[2] = v[0][2]; dst[3] = v[0][3]; }
        } else {
            const bool f16 = e.y_dtype == TBIK_F16;
            const uint32_t lo = pack_16x2(v[0][0], v[0][1], f16), hi = pack_16x2(v[0][2], v[0][3], f16);
            uint16_t *dst = reinterpret_cast<uint16_t *>(Y) + row * ldy + col;
            if (pieces.out) *reinterpret_cast<uint2 *>(dst) = make_uint2(lo, hi);
            else { dst[0] = (uint16_t)lo; dst[1] = (uint16_t)(lo >> 16); dst[2] = (uint16_t)hi; dst[3] = (uint16_t)(hi >> 16); }
        }
    }
}

// Any N: an element per thread.
template <int P>
__global__ __launch_bounds__(256) void tree_combine_epilogue_scalar_kernel(const float *__restrict__ partials, const EpilogueParams e, void *Y, int64_t ldy, int64_t M, int64_t N) {
    const int64_t total = M * N, stride = (int64_t)gridDim.x * blockDim.x;
    for (int64_t q = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; q < total; q += stride) {
        const int64_t row = q / N, col = q - row * N;
        float v[P];
#pragma unroll
        for (int p = 0; p < P; ++p) v[p] = partials[(int64_t)p * total + q];
        finish_and_store(e, tree_of<P>(v), Y, ldy, row, col);
    }
}

template <int P>
hipError_t launch_p(const float *partials, const EpilogueParams &e, void *Y, int64_t ldy, int M, int N, hipStream_t s) {
    const bool vec = N % 4 == 0;
    const int64_t work = vec ? (int64_t)M * (N / 4) : (int64_t)M * N;
    int64_t blocks = (work + 255) / 256;
    if (blocks > 256 * 64) blocks = 256 * 64;      // grid-stride beyond 64 blocks per CU
    const auto whole = [](const void *p, int64_t ld, int dtype) { return (int)((reinterpret_cast<uintptr_t>(p) % (dtype == TBIK_F32 ? 16 : 8)) == 0 && ld % 4 == 0); };
    const CombinePieces pieces{whole(Y, ldy, e.y_dtype), whole(e.residual, e.ldr, e.y_dtype), whole(e.bias, 0, e.bias_dtype), whole(e.col_scale, 0, TBIK_F32)};
    const bool stream = (int64_t)P * M * N * 4 > ((int64_t)192 << 20);
    const dim3 grid((unsigned)blocks), block(256);
    if (vec && stream) hipLaunchKernelGGL((tree_combine_epilogue_vec4_kernel<P, true>), grid, block, 0, s, partials, e, Y, ldy, (int64_t)M, (int64_t)N, pieces);
    else if (vec) hipLaunchKernelGGL((tree_combine_epilogue_vec4_kernel<P, false>), grid, block, 0, s, partials, e, Y, ldy, (int64_t)M, (int64_t)N, pieces);
    else hipLaunchKernelGGL((tree_combine_epilogue_scalar_kernel<P>), grid, block, 0, s, partials, e, Y, ldy, (int64_t)M, (int64_t)N);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_tree_combine_epilogue(const float *partials, int P, const EpilogueParams &e, void *Y, int64_t ldy, int M, int N, hipStream_t s) {
    if (M <= 0 || N <= 0) return hipSuccess;
    switch (P) {
        case 1: return launch_p<1>(partials, e, Y, ldy, M, N, s);
        case 2: return launch_p<2>(partials, e, Y, ldy, M, N, s);
        case 4: return launch_p<4>(partials, e, Y, ldy, M, N, s);
        case 8: return launch_p<8>(partials, e, Y, ldy, M, N, s);
        case 16: return launch_p<16>(partials, e, Y, ldy, M, N, s);
        case 32: return launch_p<32>(partials, e, Y, ldy, M, N, s);
        case 64: return launch_p<64>(partials, e, Y, ldy, M, N, s);
        default: return hipErrorInvalidValue;
    }
}

}  // namespace tbik
