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
// Offsets inside 32 rows are 32 bits (kMaxVectorRowBytes).  WIDE: fp32 output.  f16: which 16-bit output (a constant where the
// kernel knows).  FULL: a fixed number of store instructions, MT * 4 of 16 bits, MT * 8 of fp32 (NT == 2; half of that for NT == 1).
template <bool FULL, bool WIDE, int MT, int NT, class Flag>
__device__ __forceinline__ void store_with_epilogue(const Acc<MT, NT> &acc, float *patch, const EpilogueParams &e, void *Y, int64_t ldy,
                                                    int row0, int col0, int last, int lane, Flag f16) {
    constexpr int WCOLS = 32 * NT, CPR = WCOLS / 8, RPI = 64 / CPR, N_IT = 32 / RPI, ES = WIDE ? 4 : 2;
    if (!FULL && last < 0) return;                             // uniform
    const int lrow = lane / CPR, lc = lane % CPR;
    const int col = col0 + lc * 8;
    const char *const res = e.residual ? reinterpret_cast<const char *>(e.residual) + ((int64_t)row0 * e.ldr + col0) * ES : nullptr;
    char *const out = reinterpret_cast<char *>(Y) + ((int64_t)row0 * ldy + col0) * ES;
    const unsigned out_lane = (unsigned)(lrow * (int)ldy + lc * 8) * ES, out_step = (unsigned)(RPI * (int)ldy) * ES;
    tile_u32x4 r16[MT][N_IT];
    if (res && !WIDE) {
#pragma unroll
        for (int a = 0; a < MT; ++a)
#pragma unroll
            for (int it = 0; it < N_IT; ++it) {
                if (!FULL && last < 32 * a) continue;          // uniform
                const int row = it * RPI + lrow, safe = FULL ? row : min(row, last - 32 * a);
                r16[a][it] = *reinterpret_cast<const tile_u32x4 *>(res + a * 64 * e.ldr + (unsigned)(safe * (int)e.ldr + lc * 8) * 2u);
            }
    }
    float rs[MT][N_IT], cs[8], b[8];
    const bool vectors = e.row_scale || e.col_scale || e.bias, activated = e.act != TBIK_ACT_NONE;
    if (vectors) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            cs[i] = e.col_scale ? e.col_scale[col + i] : 0.0f;
            b[i] = e.bias ? widened(e.bias, col + i, e.bias_dtype) : 0.0f;
        }
#pragma unroll
        for (int a = 0; a < MT; ++a)
#pragma unroll
            for (int it = 0; it < N_IT; ++it) {
                const int row = a * 32 + it * RPI + lrow;
                rs[a][it] = e.row_scale ? e.row_scale[row0 + (FULL ? row : min(row, last))] : 0.0f;
            }
    }
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
                float v[1][8] = {{at[0][0], at[0][1], at[0][2], at[0][3], at[1][0], at[1][1], at[1][2], at[1][3]}};
                if (vectors) {
                    const float rsv[1] = {e.row_scale ? e.row_scale[row0 + a * 32 + (FULL ? row : min(row, last - 32 * a))] : 0.0f};
                    scale_and_bias(e, v, rsv, cs, b);
                }
                activate(e.act, v[0]);
                at[0] = f32x4{v[0][0], v[0][1], v[0][2], v[0][3]};
                at[1] = f32x4{v[0][4], v[0][5], v[0][6], v[0][7]};
            }
        }
        float v[N_IT][8];                                      // one absent part, one branch for the block row
#pragma unroll
        for (int it = 0; it < N_IT; ++it) {
            const f32x4 *rd = reinterpret_cast<const f32x4 *>(patch + (it * RPI + lrow) * WCOLS + lc * 8);
            const f32x4 lo = rd[0], hi = rd[1];
#pragma unroll
            for (int i = 0; i < 4; ++i) { v[it][i] = lo[i]; v[it][4 + i] = hi[i]; }
        }
        if (vectors && !activated) scale_and_bias(e, v, rs[a], cs, b);
        if (res) {
#pragma unroll
            for (int it = 0; it < N_IT; ++it) {
                float r[8];
                if constexpr (WIDE) {
                    const int row = it * RPI + lrow, safe = FULL ? row : min(row, last - 32 * a);
                    const f32x4 *src = reinterpret_cast<const f32x4 *>(res + a * 128 * e.ldr + (unsigned)(safe * (int)e.ldr + lc * 8) * 4u);
                    const f32x4 r0 = src[0], r1 = src[1];
#pragma unroll
                    for (int i = 0; i < 4; ++i) { r[i] = r0[i]; r[4 + i] = r1[i]; }
                } else {
                    const uint4 q = make_uint4(r16[a][it][0], r16[a][it][1], r16[a][it][2], r16[a][it][3]);
                    if (f16) unpack8<true>(q, r);
                    else unpack8<false>(q, r);
                }
                add_residual(v[it], r);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int it = 0; it < N_IT; ++it) {
            if (!FULL && it * RPI + lrow > last - 32 * a) continue;
            char *dst = out + a * 32 * ldy * ES + (out_lane + it * out_step);
            if constexpr (WIDE) {
                *reinterpret_cast<f32x4 *>(dst) = f32x4{v[it][0], v[it][1], v[it][2], v[it][3]};
                *reinterpret_cast<f32x4 *>(dst + 16) = f32x4{v[it][4], v[it][5], v[it][6], v[it][7]};
            } else {
                tile_u32x4 o;
                if (f16) o = tile_u32x4{pack_f16x2(v[it][0], v[it][1]), pack_f16x2(v[it][2], v[it][3]), pack_f16x2(v[it][4], v[it][5]), pack_f16x2(v[it][6], v[it][7])};
                else o = tile_u32x4{pack_bf16x2(v[it][0], v[it][1]), pack_bf16x2(v[it][2], v[it][3]), pack_bf16x2(v[it][4], v[it][5]), pack_bf16x2(v[it][6], v[it][7])};
                *reinterpret_cast<tile_u32x4 *>(dst) = o;
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
