// The top-of-tree combine (combine.hip) with the epilogue of the matrix products between the sum and the rounding: what ends
// a K-split product with an epilogue, and a tensor-parallel layer's all-reduce with the bias, the activation and the residual
// that follow it.  HBM-bound: 4 P bytes of partial sums per element, the residual and the output.
#include "epilogue.hpp"

namespace tbik {

// VEC: a thread owns 4 consecutive columns of one row (N % 4 == 0); else one element.
template <int P, bool VEC>
__global__ __launch_bounds__(256) void tree_combine_epilogue_kernel(const float *__restrict__ partials, const EpilogueParams e, void *Y,
                                                                    int64_t ldy, int64_t M, int64_t N, int vec_out) {
    constexpr int W = VEC ? 4 : 1;
    const int64_t per_row = N / W, total = M * per_row, plane = M * N;
    const int64_t stride = (int64_t)gridDim.x * blockDim.x;
    for (int64_t q = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; q < total; q += stride) {
        const int64_t row = q / per_row, col = (q - row * per_row) * W;
        if constexpr (!VEC) {
            float v[P];
#pragma unroll
            for (int p = 0; p < P; ++p) v[p] = partials[(int64_t)p * plane + q];
            finish_and_store(e, tree_of<P>(v), Y, ldy, row, col);
        } else {
            f32x4 in[P];
#pragma unroll
            for (int p = 0; p < P; ++p) in[p] = *reinterpret_cast<const f32x4 *>(partials + (int64_t)p * plane + row * N + col);
            float y[1][4], cs[4] = {0, 0, 0, 0}, b[4] = {0, 0, 0, 0}, r[4] = {0, 0, 0, 0}, rs[1] = {0.0f};
            float (&v)[4] = y[0];
            if (e.row_scale) rs[0] = e.row_scale[row];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (e.col_scale) cs[i] = e.col_scale[col + i];
                if (e.bias) b[i] = widened(e.bias, col + i, e.bias_dtype);
                if (e.residual) r[i] = widened(e.residual, row * e.ldr + col + i, e.y_dtype);
                float t[P];
#pragma unroll
                for (int p = 0; p < P; ++p) t[p] = in[p][i];
                v[i] = tree_of<P>(t);
            }
            scale_and_bias(e, y, rs, cs, b);
            activate(e.act, v);
            if (e.residual) add_residual(v, r);
            if (e.y_dtype == TBIK_F32) {
                float *dst = reinterpret_cast<float *>(Y) + row * ldy + col;
                if (vec_out) *reinterpret_cast<f32x4 *>(dst) = f32x4{v[0], v[1], v[2], v[3]};
                else { dst[0] = v[0]; dst[1] = v[1]; dst[2] = v[2]; dst[3] = v[3]; }
            } else {
                const bool f16 = e.y_dtype == TBIK_F16;
                const uint32_t lo = pack_16x2(v[0], v[1], f16), hi = pack_16x2(v[2], v[3], f16);
                uint16_t *dst = reinterpret_cast<uint16_t *>(Y) + row * ldy + col;
                if (vec_out) *reinterpret_cast<uint2 *>(dst) = make_uint2(lo, hi);
                else { dst[0] = (uint16_t)lo; dst[1] = (uint16_t)(lo >> 16); dst[2] = (uint16_t)hi; dst[3] = (uint16_t)(hi >> 16); }
            }
        }
    }
}

template <int P>
static hipError_t launch_p(const float *partials, const EpilogueParams &e, void *Y, int64_t ldy, int M, int N, hipStream_t s) {
    const bool vec = N % 4 == 0 && (reinterpret_cast<uintptr_t>(partials) & 15) == 0;
    const int64_t work = vec ? (int64_t)M * (N / 4) : (int64_t)M * N;
    int64_t blocks = (work + 255) / 256;
    if (blocks > 256 * 64) blocks = 256 * 64;      // grid-stride beyond 64 blocks per CU
    const int piece = e.y_dtype == TBIK_F32 ? 16 : 8;
    const auto pieces = [&](const void *p, int64_t ld) { return (reinterpret_cast<uintptr_t>(p) % piece) == 0 && ld % 4 == 0; };
    const dim3 grid((unsigned)blocks), block(256);
    auto launch = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, grid, block, 0, s, partials, e, Y, ldy, (int64_t)M, (int64_t)N, (int)pieces(Y, ldy));
    };
    if (vec) launch(tree_combine_epilogue_kernel<P, true>);
    else launch(tree_combine_epilogue_kernel<P, false>);
    return hipGetLastError();
}

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
