// The output tile of a tiled GEMM kernel through the epilogue (epilogue.hpp).
#pragma once

#include "epilogue.hpp"
#include "tile_store.hpp"

namespace tbik {

// Whether the residual can be read in pieces of 16 bytes with 32-bit offsets.
inline bool residual_in_vectors(const EpilogueParams &e) {
    const int64_t row_bytes = e.ldr * (e.y_dtype == TBIK_F32 ? 4 : 2);
    return !e.residual || ((reinterpret_cast<uintptr_t>(e.residual) & 15) == 0 && row_bytes % 16 == 0 && row_bytes < kMaxVectorRowBytes);
}

// A wavefront's accumulators, 32 MT rows from row0 on and 32 NT columns from col0 on, to Y.  As the plain store does it, a block
// row goes through `patch` (32 x 32 NT floats of LDS, the wavefront's own), so that a lane holds 8 consecutive columns of one
// row; the lane's columns are the same in every row, so their scales and biases are loaded once.  The residual comes in pieces of
// 16 bytes, all of the tile's 16-bit ones under way before the first is used.  `last`: the last row of the wavefront's tile
// that exists (below 32 MT - 1: FULL is false); rows past it are neither read nor written, so Y may be the residual itself.
// Offsets inside 32 rows are 32 bits (kMaxVectorRowBytes).  FULL: a fixed number of store instructions, MT * 4 of 16 bits, MT * 8 of fp32 (NT == 2; half of that for NT == 1).
template <bool FULL, int MT, int NT>
__device__ __forceinline__ void store_with_epilogue(const Acc<MT, NT> &acc, float *patch, const EpilogueParams &e, void *Y, int64_t ldy,
                                                    int row0, int col0, int last, int lane) {
    constexpr int WCOLS = 32 * NT, CPR = WCOLS / 8, RPI = 64 / CPR, N_IT = 32 / RPI;
    const int lrow = lane / CPR, lc = lane % CPR;
    const int col = col0 + lc * 8;
    const bool wide = e.y_dtype == TBIK_F32, f16 = e.y_dtype == TBIK_F16;
    const int es = wide ? 4 : 2;
    float cs[8] = {0, 0, 0, 0, 0, 0, 0, 0}, b[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (!FULL && last < 0) return;                             // uniform
    const char *const res = e.residual ? reinterpret_cast<const char *>(e.residual) + ((int64_t)row0 * e.ldr + col0) * es : nullptr;
    char *const out = reinterpret_cast<char *>(Y) + ((int64_t)row0 * ldy + col0) * es;
    tile_u32x4 r16[MT][N_IT];
    float rs[MT][N_IT];
#pragma unroll
    for (int a = 0; a < MT; ++a)
#pragma unroll
        for (int it = 0; it < N_IT; ++it) {
            r16[a][it] = tile_u32x4{0, 0, 0, 0};
            rs[a][it] = 0.0f;
            if (!FULL && last < 32 * a) continue;              // uniform
            const int row = it * RPI + lrow, safe = FULL ? row : min(row, last - 32 * a);
            if (res && !wide) r16[a][it] = *reinterpret_cast<const tile_u32x4 *>(res + a * 64 * e.ldr + (unsigned)(safe * (int)e.ldr + lc * 8) * 2u);
            if (e.row_scale) rs[a][it] = e.row_scale[row0 + a * 32 + safe];
        }
    if (e.col_scale) {
#pragma unroll
        for (int i = 0; i < 8; ++i) cs[i] = e.col_scale[col + i];
    }
    if (e.bias) {
#pragma unroll
        for (int i = 0; i < 8; ++i) b[i] = widened(e.bias, col + i, e.bias_dtype);
    }
    const bool activated = e.act != TBIK_ACT_NONE;
#pragma unroll
    for (int a = 0; a < MT; ++a) {
        if (!FULL && last < 32 * a) continue;
        fill_patch(acc, a, patch, lane);
        if (activated) {
            // A loop, and back into the patch: unrolled with the stores, the five activations are 30 KiB of code per kernel.
#pragma nounroll
            for (int it = 0; it < N_IT; ++it) {
                const int row = it * RPI + lrow;
                f32x4 *at = reinterpret_cast<f32x4 *>(patch + row * WCOLS + lc * 8);
                float v[8] = {at[0][0], at[0][1], at[0][2], at[0][3], at[1][0], at[1][1], at[1][2], at[1][3]};
                float rsv = 0.0f;
                if (e.row_scale) rsv = e.row_scale[row0 + a * 32 + (FULL ? row : min(row, last - 32 * a))];
                scale_and_bias(e, v, rsv, cs, b);
                activate(e.act, v);
                at[0] = f32x4{v[0], v[1], v[2], v[3]};
                at[1] = f32x4{v[4], v[5], v[6], v[7]};
            }
        }
#pragma unroll
        for (int it = 0; it < N_IT; ++it) {
            const int row = it * RPI + lrow;
            const f32x4 *rd = reinterpret_cast<const f32x4 *>(patch + row * WCOLS + lc * 8);
            const f32x4 lo = rd[0], hi = rd[1];
            float v[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
            if (!activated) scale_and_bias(e, v, rs[a][it], cs, b);
            if (res) {
                float r[8];
                if (wide) {
                    const int safe = FULL ? row : min(row, last - 32 * a);
                    const f32x4 *src = reinterpret_cast<const f32x4 *>(res + a * 128 * e.ldr + (unsigned)(safe * (int)e.ldr + lc * 8) * 4u);
                    const f32x4 r0 = src[0], r1 = src[1];
#pragma unroll
                    for (int i = 0; i < 4; ++i) { r[i] = r0[i]; r[4 + i] = r1[i]; }
                } else {
                    const uint4 q = make_uint4(r16[a][it][0], r16[a][it][1], r16[a][it][2], r16[a][it][3]);
                    if (f16) unpack8<true>(q, r);
                    else unpack8<false>(q, r);
                }
                add_residual(v, r);
            }
            if (FULL || row <= last - 32 * a) {
                char *dst = out + a * 32 * ldy * es + (unsigned)(row * (int)ldy + lc * 8) * (unsigned)es;
                if (wide) {
                    *reinterpret_cast<f32x4 *>(dst) = f32x4{v[0], v[1], v[2], v[3]};
                    *reinterpret_cast<f32x4 *>(dst + 16) = f32x4{v[4], v[5], v[6], v[7]};
                } else {
                    *reinterpret_cast<tile_u32x4 *>(dst) = tile_u32x4{pack_16x2(v[0], v[1], f16), pack_16x2(v[2], v[3], f16),
                                                                      pack_16x2(v[4], v[5], f16), pack_16x2(v[6], v[7], f16)};
                }
            }
        }
    }
}

// The same element by element: columns that end inside the tile, rows that are not 16-byte aligned.
template <int MT, int NT>
__device__ __forceinline__ void store_elements_with_epilogue(const Acc<MT, NT> &acc, float *patch, const EpilogueParams &e, void *Y, int64_t ldy,
                                                             int row0, int col0, int M, int N, int lane) {
    constexpr int WCOLS = 32 * NT;
#pragma unroll
    for (int a = 0; a < MT; ++a) {
        fill_patch(acc, a, patch, lane);
#pragma nounroll
        for (int i = lane; i < 32 * WCOLS; i += 64) {
            const int row = row0 + a * 32 + i / WCOLS, col = col0 + i % WCOLS;
            if (row < M && col < N) finish_and_store(e, patch[i], Y, ldy, row, col);
        }
    }
}

}  // namespace tbik
