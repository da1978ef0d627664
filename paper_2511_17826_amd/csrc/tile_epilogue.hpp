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

template <bool WIDE, class Flag>
__device__ __forceinline__ void store_8(char *dst, const float (&v)[8], Flag f16) {
    if constexpr (WIDE) {
        *reinterpret_cast<f32x4 *>(dst) = f32x4{v[0], v[1], v[2], v[3]};
        *reinterpret_cast<f32x4 *>(dst + 16) = f32x4{v[4], v[5], v[6], v[7]};
    } else {
        tile_u32x4 o;
        if (f16) o = tile_u32x4{pack_f16x2(v[0], v[1]), pack_f16x2(v[2], v[3]), pack_f16x2(v[4], v[5]), pack_f16x2(v[6], v[7])};
        else o = tile_u32x4{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
        *reinterpret_cast<tile_u32x4 *>(dst) = o;
    }
}

// A wavefront's accumulators, 32 MT rows from row0 on and 32 NT columns from col0 on, to Y.  As the plain store does it, a block
// row goes through `patch` (32 x 32 NT floats of LDS, the wavefront's own), so that a lane holds 8 consecutive columns of one
// row; the lane's columns are the same in every row, so their scales and biases are loaded once.  The residual comes in pieces of
// 16 bytes, all of the tile's 16-bit ones under way before the first is used.  `last`: the last row of the wavefront's tile
// that exists; rows past it are neither read nor written, so Y may be the residual itself.  Offsets inside 32 rows are 32 bits
// (kMaxVectorRowBytes).  WIDE: fp32 output.  f16: which 16-bit output (a constant where the kernel knows).
// For an fp32 residual and for operands at odd addresses; the others come through the ring, below.
template <bool WIDE, int MT, int NT, class Flag>
__device__ __forceinline__ void store_with_epilogue(const Acc<MT, NT> &acc, float *patch, const EpilogueParams &e, void *Y, int64_t ldy,
                                                    int row0, int col0, int last, int lane, Flag f16) {
    constexpr int WCOLS = 32 * NT, CPR = WCOLS / 8, RPI = 64 / CPR, N_IT = 32 / RPI, ES = WIDE ? 4 : 2;
    if (last < 0) return;                              // uniform
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
                if (last < 32 * a) continue;          // uniform
                const int row = it * RPI + lrow, safe = min(row, last - 32 * a);
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
                rs[a][it] = e.row_scale ? e.row_scale[row0 + min(row, last)] : 0.0f;
            }
    }
#pragma unroll
    for (int a = 0; a < MT; ++a) {
        if (last < 32 * a) continue;
        fill_patch(acc, a, patch, lane);
        if (activated) {
            // A loop, and back into the patch: unrolled with the stores, the four activations are 30 KiB of code per kernel.
#pragma nounroll
            for (int it = 0; it < N_IT; ++it) {
                const int row = it * RPI + lrow;
                f32x4 *at = reinterpret_cast<f32x4 *>(patch + row * WCOLS + lc * 8);
                float v[1][8] = {{at[0][0], at[0][1], at[0][2], at[0][3], at[1][0], at[1][1], at[1][2], at[1][3]}};
                if (vectors) {
                    const float rsv[1] = {e.row_scale ? e.row_scale[row0 + a * 32 + min(row, last - 32 * a)] : 0.0f};
                    scale_and_bias(e, v, rsv, cs, b);
                }
                activate(e.act, v);
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
                    const int row = it * RPI + lrow, safe = min(row, last - 32 * a);
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
            if (it * RPI + lrow > last - 32 * a) continue;
            char *dst = out + a * 32 * ldy * ES + (out_lane + it * out_step);
            store_8<WIDE>(dst, v[it], f16);
        }
    }
}

// ---- the epilogue's operands through the ring ----
// Loads that an epilogue issues itself are behind the ring's loads in flight on the wavefront's one counter, so that waiting for
// them drains the ring: 2 to 3 us per tile.  So the vectors (scales, bias) and the 16-bit residual of a tile come as one or two
// positions of the load stream behind the tile's last stage, by the same instructions as a stage, and have landed by then:
//   vectors    wavefront 0 brings the tile's bias (its first X load) and column scales (its first W load), wavefront 1 the row scales
//   residual   each wavefront brings its own 32 MT x 32 NT piece, chunk a * N_IT + it as store_from_ring() takes it, so that a
//              lane finds its own 16 bytes where the load put them
// The other loads of such a position bring anything that exists.  All addresses are in bounds for every tile; pieces past the
// last whole 16 bytes of a vector are not read (store_from_ring() says who brings them).
constexpr int RING_LANE_BIAS = 4096;         // as the kernels' own: the lane offsets of W loads stay non-negative
template <int A_LOADS, int B_LOADS>
struct RingLoads {                           // where a position's loads come from, as the kernels keep it
    const char *&a_ptr, *&b_ptr;
    unsigned (&aoff)[A_LOADS], (&boff)[B_LOADS];
    __device__ __forceinline__ void set(const char *a, const char *b) const {
        a_ptr = uniform_pointer(a);
        b_ptr = uniform_pointer(b - RING_LANE_BIAS);
    }
    __device__ __forceinline__ void a_offset(int j, unsigned off) const { aoff[j] = off + (unsigned)((A_LOADS - j) * 1024); }
    __device__ __forceinline__ void b_offset(int j, unsigned off) const { boff[j] = off + (unsigned)(RING_LANE_BIAS - j * 1024); }
};
// any: 16 bytes that exist.
template <int A_LOADS, int B_LOADS>
__device__ __forceinline__ void point_at_vectors(const RingLoads<A_LOADS, B_LOADS> &r, const EpilogueParams &e, const void *any, int m0, int n0, int M, int N, int wave, int lane) {
    const char *a = reinterpret_cast<const char *>(any), *b = a;
    int a_more = 0, b_more = 0;                        // whole pieces of 16 bytes behind the first of the tile
    auto piece = [](const char *&at, int &more, const void *vector, int whole, int first) {
        first = min(first, whole - 1);
        at = reinterpret_cast<const char *>(vector) + (int64_t)first * 16;
        more = whole - 1 - first;
    };
    if (wave == 0 && e.bias) {
        if (e.bias_dtype == TBIK_F32) piece(a, a_more, e.bias, N / 4, n0 / 4);
        else piece(a, a_more, e.bias, N / 8, n0 / 8);
    } else if (wave == 1 && e.row_scale && M >= 4) {
        piece(a, a_more, e.row_scale, M / 4, m0 / 4);
    }
    if (wave == 0 && e.col_scale) piece(b, b_more, e.col_scale, N / 4, n0 / 4);
    r.set(a, b);
    const unsigned ao = (unsigned)min(lane, a_more) * 16u, bo = (unsigned)min(lane, b_more) * 16u;
#pragma unroll
    for (int j = 0; j < A_LOADS; ++j) r.a_offset(j, ao);
#pragma unroll
    for (int j = 0; j < B_LOADS; ++j) r.b_offset(j, bo);
}
template <int MT, int NT, int A_LOADS, int B_LOADS>
__device__ __forceinline__ void point_at_residual(const RingLoads<A_LOADS, B_LOADS> &r, const EpilogueParams &e, int m0, int n0, int M, int N, int wm, int wn, int lane) {
    constexpr int WCOLS = 32 * NT, CPR = WCOLS / 8, RPI = 64 / CPR, N_IT = 32 / RPI;
    static_assert(MT * N_IT <= A_LOADS + B_LOADS, "the tile's piece fits the wavefront's region");
    const char *base = reinterpret_cast<const char *>(e.residual) + (int64_t)m0 * e.ldr * 2;
    r.set(base, base);
    const int col = min(n0 + wn * WCOLS + lane % CPR * 8, (N - 8) & ~7);
    auto offset = [&](int chunk) {
        const int row = wm * MT * 32 + min(chunk, MT * N_IT - 1) * RPI + lane / CPR;
        return (unsigned)(min(row, M - 1 - m0) * (int)e.ldr + col) * 2u;
    };
#pragma unroll
    for (int j = 0; j < A_LOADS; ++j) r.a_offset(j, offset(j));
#pragma unroll
    for (int j = 0; j < B_LOADS; ++j) r.b_offset(j, offset(A_LOADS + j));
}
// Whether an epilogue's operands can come so: 16-byte aligned, at least one whole tile of columns, 32-bit offsets inside a tile.
inline bool epilogue_from_ring(const EpilogueParams &e, int N) {
    const auto a16 = [](const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; };
    if (N < 128 || !a16(e.bias) || !a16(e.row_scale) || !a16(e.col_scale)) return false;
    return !e.residual || (e.y_dtype != TBIK_F32 && residual_in_vectors(e) && e.ldr < (1 << 22));
}

// store_with_epilogue() with its operands from the ring.  vectors: the slot that holds them, or nullptr; residual: the wavefront's region
// of the slot that holds it, or nullptr; wm, wn: the wavefront's place in the workgroup tile; M: rows of the call.  Rows past `last`
// are not written.  FULL: there are none, and the number of store instructions is that of the plain epilogue.
template <bool FULL, bool WIDE, int REGION, int A_LOADS, int MT, int NT, class Flag>
__device__ __forceinline__ void store_from_ring(const Acc<MT, NT> &acc, float *patch, const EpilogueParams &e, const unsigned char *vectors, const unsigned char *residual,
                                                void *Y, int64_t ldy, int row0, int col0, int wm, int wn, int M, int last, int lane, Flag f16) {
    constexpr int WCOLS = 32 * NT, CPR = WCOLS / 8, RPI = 64 / CPR, N_IT = 32 / RPI, ES = WIDE ? 4 : 2;
    const int lrow = lane / CPR, lc = lane % CPR;
    char *const out = reinterpret_cast<char *>(Y) + ((int64_t)row0 * ldy + col0) * ES;
    const unsigned out_lane = (unsigned)(lrow * (int)ldy + lc * 8) * ES, out_step = (unsigned)(RPI * (int)ldy) * ES;
    const bool activated = e.act != TBIK_ACT_NONE;
    float rs[MT][N_IT], cs[8], b[8];
    if (vectors) {
        const int ct = wn * WCOLS + lc * 8;                    // the lane's columns in the tile
        const f32x4 *c4 = reinterpret_cast<const f32x4 *>(vectors + A_LOADS * 1024 + ct * 4);
        const f32x4 c0 = c4[0], c1 = c4[1];
        if (e.bias_dtype == TBIK_F32) {
            const f32x4 *b4 = reinterpret_cast<const f32x4 *>(vectors + ct * 4);
            const f32x4 b0 = b4[0], b1 = b4[1];
#pragma unroll
            for (int i = 0; i < 4; ++i) { b[i] = b0[i]; b[4 + i] = b1[i]; }
        } else {
            const uint4 q = *reinterpret_cast<const uint4 *>(vectors + ct * 2);
            if (e.bias_dtype == TBIK_F16) unpack8<true>(q, b);
            else unpack8<false>(q, b);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) { cs[i] = c0[i]; cs[4 + i] = c1[i]; }
        if (!e.col_scale) {
#pragma unroll
            for (int i = 0; i < 8; ++i) cs[i] = 1.0f;
        }
        const float *r4 = reinterpret_cast<const float *>(vectors + REGION);
#pragma unroll
        for (int a = 0; a < MT; ++a)
#pragma unroll
            for (int it = 0; it < N_IT; ++it) rs[a][it] = e.row_scale ? r4[(wm * MT + a) * 32 + it * RPI + lrow] : 1.0f;
        if (!FULL && e.row_scale && last < 32 * MT - 1 && (M & 3)) {    // the last M % 4 rows' scales are not whole 16 bytes: through the scalar cache
            typedef const __attribute__((address_space(4))) float *constant_floats;
            const constant_floats tail = (constant_floats)(uintptr_t)(e.row_scale + (M & ~3));
            const float t0 = tail[0], t1 = tail[(M & 3) > 1 ? 1 : 0], t2 = tail[(M & 3) > 2 ? 2 : 0];
            const int from = (M & ~3) - row0;
#pragma unroll
            for (int a = 0; a < MT; ++a)
#pragma unroll
                for (int it = 0; it < N_IT; ++it) {
                    const int k = a * 32 + it * RPI + lrow - from;
                    if (k >= 0) rs[a][it] = k == 0 ? t0 : k == 1 ? t1 : t2;
                }
        }
    }
    // The block rows.  Flags that are constants give straight code; values that pass around a branch are copied there, one or two
    // instructions each (in 8 bits, 4096 x 4096 x 8192: with no part at all 146 -> 143 us, all parts but an activation 163.5 -> 161; the
    // 16-bit output's type as a constant too, 168.5 -> 165).
    auto rows = [&](auto row_scale, auto col_scale, auto bias, auto act, auto added) __attribute__((always_inline)) {
#pragma unroll
        for (int a = 0; a < MT; ++a) {
            if (!FULL && last < 32 * a) continue;              // uniform
            fill_patch(acc, a, patch, lane);
            float v[N_IT][8];
#pragma unroll
            for (int it = 0; it < N_IT; ++it) {
                const f32x4 *rd = reinterpret_cast<const f32x4 *>(patch + (it * RPI + lrow) * WCOLS + lc * 8);
                const f32x4 lo = rd[0], hi = rd[1];
#pragma unroll
                for (int i = 0; i < 4; ++i) { v[it][i] = lo[i]; v[it][4 + i] = hi[i]; }
            }
            scale_and_bias(row_scale, col_scale, bias, v, rs[a], cs, b);
            if (act) activate(e.act, v);
            if (added) {
#pragma unroll
                for (int it = 0; it < N_IT; ++it) {
                    float r[8];
                    const uint4 q = *reinterpret_cast<const uint4 *>(residual + (a * N_IT + it) * 1024 + lane * 16);
                    if (f16) unpack8<true>(q, r);
                    else unpack8<false>(q, r);
                    add_residual(v[it], r);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int it = 0; it < N_IT; ++it) {
                if (!FULL && it * RPI + lrow > last - 32 * a) continue;
                store_8<WIDE>(out + a * 32 * ldy * ES + (out_lane + it * out_step), v[it], f16);
            }
        }
    };
    const std::true_type yes;
    const std::false_type no;
    if (!FULL || activated) {
        rows(e.row_scale != nullptr, e.col_scale != nullptr, e.bias != nullptr, activated, residual != nullptr);
    } else if (!vectors) {
        residual ? rows(no, no, no, no, yes) : rows(no, no, no, no, no);
    } else if (e.row_scale || e.col_scale) {                   // an absent one is 1, which changes no bit
        if (e.bias) residual ? rows(yes, yes, yes, no, yes) : rows(yes, yes, yes, no, no);
        else residual ? rows(yes, yes, no, no, yes) : rows(yes, yes, no, no, no);
    } else {
        residual ? rows(no, no, yes, no, yes) : rows(no, no, yes, no, no);
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
