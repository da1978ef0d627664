// The parts of the products on 4-bit weights: an element's widening, and stages in LDS.  See gemm_w4.hip.
#pragma once

#include <algorithm>
#include <atomic>
#include <type_traits>

#include "tbik_device.hpp"
#include "tbik_internal.hpp"
#include "tile_store.hpp"

namespace tbik {

struct W4Params {
    const uint16_t *X;
    const uint8_t *W;
    const uint16_t *scales;
    const uint8_t *zeros;
    float *partials;
    void *Y;
    int64_t ldx, ldw, lds, ldz, ldy;
    int64_t plane;                         // floats of a shard's partial sums
    int M, N;
    int y_f32;
    int superleaf, groups_per_leaf;
    int units_per_group;                   // of the call's UNIT
    int stages_per_leaf;                   // of the call's stage
    int leaves_per_wave, active_waves, leaves_per_shard;
    int vector_stores;
    int row_bytes;                         // slices of one row: LDS for the row's part of a wavefront's k, whole loads
    int s_dwords, z_dwords;                // of a channel in a chunk of scales, of zero points
    int s_inverse, z_inverse;              // 65536 over them, rounded up: quotients of numbers below 1024
    int group_bytes;                       // LDS of a wavefront for its chunks of both
};

constexpr int W4_WAVES = 8;                // of a slice, and of the general kernel's workgroup

// Eight elements of one dword, element i in bits 4 i .. 4 i + 3, as 16-bit floats of (q - zero) / 16 in order.  `zero`: ZeroPoint of the channel's group.
// bf16: a float per element (v_cvt_off_f32_i4 of the 4-bit two's complement number q - 8, whose byte selection costs nothing; with zero points the bytes q - zero
// through v_cvt_f32_i32), then the upper halves of two as one register: exact.  14 instructions (19 with zero points).
// fp16: 1024 + q has q in its low bits; one packed subtraction of 1024 + zero for two of them, exact.  13 instructions.
template <bool F16, bool ZEROS>
struct ZeroPoint {
    uint32_t v;
    __device__ __forceinline__ explicit ZeroPoint(int zero = 8) {
        if constexpr (F16) {
            const uint32_t h = 0xe400u + (uint32_t)zero;             // -(1024 + zero)
            v = h | (h << 16);
        } else {
            v = (uint32_t)(128 - zero) * 0x01010101u;
        }
    }
};
typedef _Float16 w4_f16x2 __attribute__((ext_vector_type(2)));
// Two elements a byte: byte B of `even` holds element 2 B in its low bits, of `odd` element 2 B + 1.
template <int B>
__device__ __forceinline__ uint32_t byte_of(uint32_t v) { return B == 3 ? v >> 24 : (v >> (8 * B)) & 0xffu; }
template <bool F16, bool ZEROS>
__device__ __forceinline__ bf16x8 widened_levels(uint32_t w, const ZeroPoint<F16, ZEROS> &zero) {
    union { uint32_t u[4]; w4_f16x2 h[4]; bf16x8 v; } out;
    if constexpr (F16) {
        const uint32_t odd = w >> 4;
        const w4_f16x2 less = __builtin_bit_cast(w4_f16x2, zero.v);
        out.u[0] = __builtin_amdgcn_perm(odd, w, 0x0c040c00u);       // bytes B of w and of odd, one in each half
        out.u[1] = __builtin_amdgcn_perm(odd, w, 0x0c050c01u);
        out.u[2] = __builtin_amdgcn_perm(odd, w, 0x0c060c02u);
        out.u[3] = __builtin_amdgcn_perm(odd, w, 0x0c070c03u);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            asm("v_and_or_b32 %0, %1, %2, %3" : "=v"(out.u[i]) : "v"(out.u[i]), "s"(0x000f000fu), "v"(0x64006400u));      // (left to the compiler it is two instructions)
            out.h[i] = out.h[i] + less;
        }
    } else {
        float v[8];
        if constexpr (ZEROS) {
            const uint32_t even = ((w & 0x0f0f0f0fu) + zero.v) ^ 0x80808080u, odd = (((w >> 4) & 0x0f0f0f0fu) + zero.v) ^ 0x80808080u;      // signed bytes q - zero
            v[0] = (float)(int8_t)even; v[2] = (float)(int8_t)(even >> 8); v[4] = (float)(int8_t)(even >> 16); v[6] = (float)(int8_t)(even >> 24);
            v[1] = (float)(int8_t)odd; v[3] = (float)(int8_t)(odd >> 8); v[5] = (float)(int8_t)(odd >> 16); v[7] = (float)(int8_t)(odd >> 24);
        } else {
            const uint32_t even = w ^ 0x88888888u;
            uint32_t odd = even >> 4;
            asm("" : "+v"(odd));                                     // a register of its own, whose bytes the conversions select
            v[0] = __builtin_amdgcn_cvt_off_f32_i4(even); v[2] = __builtin_amdgcn_cvt_off_f32_i4(byte_of<1>(even));
            v[4] = __builtin_amdgcn_cvt_off_f32_i4(byte_of<2>(even)); v[6] = __builtin_amdgcn_cvt_off_f32_i4(byte_of<3>(even));
            v[1] = __builtin_amdgcn_cvt_off_f32_i4(odd); v[3] = __builtin_amdgcn_cvt_off_f32_i4(byte_of<1>(odd));
            v[5] = __builtin_amdgcn_cvt_off_f32_i4(byte_of<2>(odd)); v[7] = __builtin_amdgcn_cvt_off_f32_i4(byte_of<3>(odd));
        }
#pragma unroll
        for (int b = 0; b < 4; ++b) out.u[b] = __builtin_amdgcn_perm(__float_as_uint(v[2 * b + 1]), __float_as_uint(v[2 * b]), 0x07060302u);
    }
    return out.v;
}
// What the scale is multiplied by: the bf16 elements without zero points come as sixteenths.
template <bool F16, bool ZEROS>
constexpr float kLevelUnit = F16 || ZEROS ? 1.0f : 16.0f;

template <bool F16>
__device__ __forceinline__ float widened_16(uint16_t h) { return F16 ? (float)__builtin_bit_cast(_Float16, h) : bf16_bits_to_f32(h); }

template <bool F16>
__device__ __forceinline__ f32x4 mfma_16x16x32(bf16x8 a, bf16x8 b, f32x4 c) {
    if constexpr (F16)
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// The sums of 16 MR rows and 16 NB channels: block (a, b) is 16 x 16, the lane has rows 4 (lane / 16) .. + 3 of channel lane % 16.
template <int MR, int NB = 2>
struct W4Sums {
    f32x4 t[MR][NB];
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int a = 0; a < MR; ++a)
#pragma unroll
            for (int b = 0; b < NB; ++b) t[a][b] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }
};
// Finished subtrees of up to 2^LEVELS superleaves (the carry-over scheme of App. D.1): `leaf`, counted from 0, has ended in acc.
template <int MR, int NB, int LEVELS>
struct W4Stash {
    f32x4 s[MR][NB][LEVELS];
    __device__ __forceinline__ void push(W4Sums<MR, NB> &acc, int leaf, bool more) {
        const int t = __builtin_ctz(~leaf);
#pragma unroll
        for (int a = 0; a < MR; ++a)
#pragma unroll
            for (int b = 0; b < NB; ++b) {
#pragma unroll
                for (int l = 0; l < LEVELS; ++l)
                    if (l < t) {
#pragma unroll
                        for (int r = 0; r < 4; ++r) acc.t[a][b][r] = s[a][b][l][r] + acc.t[a][b][r];
                    }
            }
        if (!more) return;
#pragma unroll
        for (int a = 0; a < MR; ++a)
#pragma unroll
            for (int b = 0; b < NB; ++b) {
#pragma unroll
                for (int l = 0; l < LEVELS; ++l)
                    if (LEVELS == 1 || l == t) s[a][b][l] = acc.t[a][b];
            }
        acc.clear();
    }
};

// T over 2^levels superleaves, levels <= L: a nest of loops, each of two trips or (above `levels`) one, whose first trip parks its subtree's sum in a slot of
// its own.  (With the stash above, whose slot is chosen when it is used, tiles of 64 rows spill.)
template <int L>
struct W4Walk {
    template <class Leaf, int MR, int SLOTS>
    __device__ __forceinline__ static void run(Leaf &leaf, W4Sums<MR> &acc, W4Sums<MR> (&slots)[SLOTS], int levels) {
        const int trips = L <= levels ? 2 : 1;
#pragma nounroll
        for (int half = 0; half < trips; ++half) {
            W4Walk<L - 1>::run(leaf, acc, slots, levels);
            if (half + 1 < trips) {
                slots[L - 1] = acc;
            } else if (half == 1) {
#pragma unroll
                for (int a = 0; a < MR; ++a)
#pragma unroll
                    for (int b = 0; b < 2; ++b)
#pragma unroll
                        for (int r = 0; r < 4; ++r) acc.t[a][b][r] = slots[L - 1].t[a][b][r] + acc.t[a][b][r];
            }
        }
    }
};
template <>
struct W4Walk<0> {
    template <class Leaf, int MR, int SLOTS>
    __device__ __forceinline__ static void run(Leaf &leaf, W4Sums<MR> &acc, W4Sums<MR> (&)[SLOTS], int) { leaf(acc); }
};

// ---- stages in LDS (slices and tiles) ----
// A stage is 64 S k.  Of one wavefront it holds rows of X (128 S bytes) and the 32 S bytes of each of its channels.  Chunks of 16 bytes are swapped
// about within a row so that the rows of a read meet different banks.
// S = 2 where superleaves are whole stages of 128 k: with 64, whose 32 bytes of a channel are a quarter of a cache line, the weight alone came in at
// 1.6 TB/s (27 rows, K = 12288, N = 4096 without the loads of X and the scales 16.6 us; so 7.3).
// Scales and zero points come in chunks of up to 32 groups, the next one on its way while one is used: a load for every stage touched a cache line of every channel
// and was more than half of all requests to the caches (same shape, 2.0 million).
template <int N>
__device__ __forceinline__ void w4_wait_loads() {
    static_assert(N >= 0 && N < 64, "vmcnt range");
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
template <int N>
__device__ __forceinline__ void w4_wait_loads_and_barrier() {
    static_assert(N >= 0 && N < 64, "vmcnt range");
    asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(N) : "memory");
}

// What a chunk's number is XORed with in row r of X and in channel r of the weight.
template <int S>
__device__ __forceinline__ int x_swizzle(int r) { return S == 1 ? (r >> 1) & 7 : r & 15; }
template <int S>
__device__ __forceinline__ int w_swizzle(int r) { return S == 1 ? 0 : S == 2 ? (r >> 2) & 3 : (r >> 1) & 7; }

// The group of one unit after another.
struct GroupWalk {
    unsigned g;
    int left;
    int units;                             // of a group
    __device__ __forceinline__ explicit GroupWalk(int units_per_group) : g(0), left(units_per_group), units(units_per_group) {}
    __device__ __forceinline__ bool next() {       // true: the unit was the group's last
        if (--left != 0) return false;
        left = units;
        ++g;
        return true;
    }
};

constexpr int W4_CHUNK = 32;               // groups
// LDS of a chunk of `dwords` for each of `channels`: whole loads.
__host__ __device__ constexpr int w4_chunk_bytes(int channels, int dwords) { return (channels * dwords * 4 + 255) & ~255; }
__host__ __device__ constexpr int w4_chunk_buffers(int groups) { return groups > W4_CHUNK ? 2 : 1; }

// The scales (ELEMENT == 2) or zero points (ELEMENT == 1) of CHANNELS channels from n0 on, groups from g0 on, `groups` of them: dwords, each channel's from the aligned
// one that holds its first element, so a channel's last dword may hold bytes behind its row.
template <int ELEMENT, int CHANNELS>
struct W4Groups {
    const char *ptr;                       // aligned
    unsigned low;                          // of the first channel's first element from there
    int pitch, last_channel, groups, dwords, inverse;
    unsigned at;                           // in LDS
    int bytes;                             // of a chunk there

    __device__ __forceinline__ W4Groups(const void *first, int64_t ld, int channels_left, int n, int d, int inv, unsigned where) {
        low = (unsigned)(reinterpret_cast<uintptr_t>(first) & 3);
        ptr = uniform_pointer(reinterpret_cast<const char *>(first) - low);
        pitch = (int)ld * ELEMENT;
        last_channel = channels_left - 1;
        groups = n;
        dwords = d;
        inverse = inv;
        at = where;
        bytes = w4_chunk_bytes(CHANNELS, d);
    }
    // Byte of channel c's first element from ptr.
    __device__ __forceinline__ unsigned start(int c) const { return low + (unsigned)(min(c, last_channel) * pitch); }
    __device__ __forceinline__ void issue(int chunk, int lane) const {
        const unsigned first = chunk * W4_CHUNK * ELEMENT;
        for (int j = 0; j * 64 < CHANNELS * dwords; ++j) {
            const int i = min(j * 64 + lane, CHANNELS * dwords - 1), c = (i * inverse) >> 16, d = i - c * dwords;
            const unsigned s = start(c), end = (s + groups * ELEMENT - 1) & ~3u;               // the dword of the last element
            load_4B_per_lane_to_lds<0, true>(ptr, min(((s + first) & ~3u) + d * 4, end), at + (chunk & 1) * bytes + j * 256);
        }
    }
    // The dword of group g (uniform) of channel c, whose start is s, and the element in its low bits.
    __device__ __forceinline__ unsigned dword(const unsigned char *chunks, unsigned g, int c, unsigned s) const {
        const unsigned byte = (s & 3) + (g % W4_CHUNK) * ELEMENT;                              // a chunk's bytes are a multiple of four
        return *reinterpret_cast<const unsigned *>(chunks + (g / W4_CHUNK & 1) * bytes + (c * dwords + (byte >> 2)) * 4);
    }
    static __device__ __forceinline__ unsigned element(unsigned dword, unsigned g, unsigned s) { return dword >> (8 * (((s & 3) + g * ELEMENT) & 3)); }
};

// One wavefront's stream: the weight of 16 NB channels from n0 on, superleaves from `leaf` on, `leaves` of them; their scales and zero points.
template <bool ZEROS, int S, int NB = 2>
struct W4Stream {
    static constexpr int LOADS = S * NB / 2, BYTES = LOADS * 1024;             // of a stage
    static_assert(LOADS >= 1, "whole loads");
    const char *w_ptr;
    unsigned w_off[LOADS];                 // of the lane
    W4Groups<2, 16 * NB> scales;
    W4Groups<1, 16 * NB> zeros;
    const unsigned char *group_at;         // both in LDS, the zero points behind the scales

    static __device__ __forceinline__ int scale_bytes(const W4Params &p, int leaves) { return w4_chunk_buffers(leaves * p.groups_per_leaf) * w4_chunk_bytes(16 * NB, p.s_dwords); }
    // group_lds, group_at: LDS for the chunks, p.group_bytes.
    __device__ __forceinline__ W4Stream(const W4Params &p, int n0, int leaf, int leaves, int lane, unsigned group_lds, const unsigned char *groups)
        : scales(p.scales + n0 * p.lds + (int64_t)leaf * p.groups_per_leaf, p.lds, p.N - n0, leaves * p.groups_per_leaf, p.s_dwords, p.s_inverse, group_lds),
          zeros(ZEROS ? p.zeros + n0 * p.ldz + (int64_t)leaf * p.groups_per_leaf : nullptr, p.ldz, p.N - n0, leaves * p.groups_per_leaf, p.z_dwords, p.z_inverse,
                group_lds + scale_bytes(p, leaves)),
          group_at(groups) {
        w_ptr = uniform_pointer(reinterpret_cast<const char *>(p.W + n0 * p.ldw + (int64_t)leaf * p.superleaf / 2));
#pragma unroll
        for (int j = 0; j < LOADS; ++j) {  // 64 chunks each, 2 S of a channel
            const int r = j * (32 / S) + lane / (2 * S), c = (lane % (2 * S)) ^ w_swizzle<S>(r);
            w_off[j] = (unsigned)(min(r, p.N - 1 - n0) * (int)p.ldw + c * 16);
        }
    }
    __device__ __forceinline__ void issue_groups(int chunk, int lane) const {
        scales.issue(chunk, lane);
        if constexpr (ZEROS) zeros.issue(chunk, lane);
    }
    // The next stage's loads to LDS address `where` (uniform).  `more`: there is a stage behind it; else the next issue loads it again.
    __device__ __forceinline__ void issue(unsigned where, bool more) {
#pragma unroll
        for (int j = 0; j < LOADS; ++j) load_16B_per_lane_to_lds<0, true>(w_ptr, w_off[j], where + j * 1024);
        if (more) w_ptr += 32 * S;
    }
};

// Multiplies a stage: rows x_rows[a] (the lane's row of X of block a in the stage, in LDS) times the stage's weight at st.  sum: the running group's; a group that ends
// goes through its scale into acc.  lane % 16: the row of X and the channel of a block; quarter: lane / 16.
// WHOLE: a group is one unit, so nothing branches within a stage, and its scales and zero points are read ahead of everything that waits for LDS instead of at
// the group's end (27 rows, K 12288 x N 4096, groups of 64 with zero points 17.4 -> 15.8 us with its combination).
template <int UNIT, bool WHOLE, bool F16, bool ZEROS, int S, int MR, int NB = 2>
struct W4Multiplier {
    using Stream = W4Stream<ZEROS, S, NB>;
    static constexpr int UNITS = 64 * S / UNIT, STEPS = UNIT / 32;      // units of a stage, instructions of a unit
    unsigned s_start[NB], z_start[NB];
    int w_at[NB], w_sw, l16, quarter;
    const unsigned char *scales, *zeros;   // in LDS
    int asked;                             // chunks of them
    GroupWalk walk;
    W4Sums<MR, NB> sum;

    __device__ __forceinline__ W4Multiplier(const W4Params &p, const Stream &stream, int lane) : walk(p.units_per_group) {
        l16 = lane & 15;
        quarter = lane >> 4;
        w_sw = w_swizzle<S>(l16);                          // of both of the lane's channels
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            s_start[b] = stream.scales.start(b * 16 + l16);
            z_start[b] = ZEROS ? stream.zeros.start(b * 16 + l16) : 0u;
            w_at[b] = (b * 16 + l16) * (32 * S);
        }
        scales = stream.group_at;
        zeros = stream.group_at + (stream.zeros.at - stream.scales.at);
        asked = 1;
        sum.clear();
    }
    __device__ __forceinline__ unsigned scale_dword(const Stream &stream, unsigned g, int b) const { return stream.scales.dword(scales, g, b * 16 + l16, s_start[b]); }
    __device__ __forceinline__ unsigned zero_dword(const Stream &stream, unsigned g, int b) const { return ZEROS ? stream.zeros.dword(zeros, g, b * 16 + l16, z_start[b]) : 0u; }
    __device__ __forceinline__ float scale_of(const Stream &stream, unsigned dword, unsigned g, int b) const {
        return widened_16<F16>((uint16_t)stream.scales.element(dword, g, s_start[b])) * kLevelUnit<F16, ZEROS>;
    }
    // Ahead of a stage: asks for the chunk behind the one in use, whose place the chunk before that has left.
    __device__ __forceinline__ void prefetch_groups(const Stream &stream, int lane) {
        if (asked < (int)(walk.g / W4_CHUNK) + 2 && asked * W4_CHUNK < stream.scales.groups) stream.issue_groups(asked++, lane);
    }
    __device__ __forceinline__ void stage(const Stream &stream, const unsigned char *st, const unsigned char *const (&x_rows)[MR], int x_sw, W4Sums<MR, NB> &acc) {
        // Of whole groups the stage's scales and zero points are read at once, ahead of everything that waits for LDS.
        uint32_t scale_dwords[WHOLE ? UNITS : 1][NB], zero_dwords[WHOLE ? UNITS : 1][NB];
        if constexpr (WHOLE) {
#pragma unroll
            for (int u = 0; u < UNITS; ++u)
#pragma unroll
                for (int b = 0; b < NB; ++b) zero_dwords[u][b] = zero_dword(stream, walk.g + u, b);
#pragma unroll
            for (int u = 0; u < UNITS; ++u)
#pragma unroll
                for (int b = 0; b < NB; ++b) scale_dwords[u][b] = scale_dword(stream, walk.g + u, b);
        }
#pragma unroll
        for (int u = 0; u < UNITS; ++u) {
            uint32_t words[NB][STEPS];
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                if constexpr (UNIT == 128) {               // chunk `quarter` of the unit's four
                    const uint4 v = *reinterpret_cast<const uint4 *>(st + w_at[b] + (((4 * u + quarter) ^ w_sw) << 4));
                    words[b][0] = v.x; words[b][1] = v.y; words[b][2] = v.z; words[b][3] = v.w;
                } else if constexpr (UNIT == 64) {         // half a chunk
                    const uint2 v = *reinterpret_cast<const uint2 *>(st + w_at[b] + (((2 * u + (quarter >> 1)) ^ w_sw) << 4) + (quarter & 1) * 8);
                    words[b][0] = v.x; words[b][1] = v.y;
                } else {
                    words[b][0] = *reinterpret_cast<const uint32_t *>(st + w_at[b] + ((u ^ w_sw) << 4) + quarter * 4);
                }
            }
            // The rows' fragments of all the unit's instructions at once: with one instruction's at a time 64 rows waited for LDS at each (K 4096 x N 12288, 256
            // rows 52.0 us, so 49.2).
            bf16x8 x[STEPS][MR];
#pragma unroll
            for (int i = 0; i < STEPS; ++i)
#pragma unroll
                for (int a = 0; a < MR; ++a) x[i][a] = *reinterpret_cast<const bf16x8 *>(x_rows[a] + (((u * (UNIT / 8) + quarter * STEPS + i) ^ x_sw) << 4));
            if constexpr (WHOLE) {
                sum.clear();
                if (u == 0 && UNITS > 1) __builtin_amdgcn_sched_barrier(0);
            }
            ZeroPoint<F16, ZEROS> zero[NB];
            if constexpr (ZEROS) {
#pragma unroll
                for (int b = 0; b < NB; ++b)
                    zero[b] = ZeroPoint<F16, ZEROS>((int)(stream.zeros.element(WHOLE ? zero_dwords[WHOLE ? u : 0][b] : zero_dword(stream, walk.g, b), walk.g, z_start[b]) & 15u));
            }
#pragma unroll
            for (int i = 0; i < STEPS; ++i) {
#pragma unroll
                for (int b = 0; b < NB; ++b) {
                    const bf16x8 w = widened_levels<F16, ZEROS>(words[b][i], zero[b]);
#pragma unroll
                    for (int a = 0; a < MR; ++a) sum.t[a][b] = mfma_16x16x32<F16>(x[i][a], w, sum.t[a][b]);
                }
            }
            const unsigned g = walk.g;
            if constexpr (WHOLE) ++walk.g;
            else if (!walk.next()) continue;
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                const float scale = scale_of(stream, WHOLE ? scale_dwords[WHOLE ? u : 0][b] : scale_dword(stream, g, b), g, b);
#pragma unroll
                for (int a = 0; a < MR; ++a)
#pragma unroll
                    for (int r = 0; r < 4; ++r) acc.t[a][b][r] = __builtin_fmaf(scale, sum.t[a][b][r], acc.t[a][b][r]);
            }
            if constexpr (!WHOLE) sum.clear();
        }
    }
};

template <bool F16>
__device__ __forceinline__ void w4_store(const W4Params &p, int shard, int row, int col, float v) {
    if (p.partials) p.partials[shard * p.plane + (int64_t)row * p.N + col] = v;
    else if (p.y_f32) reinterpret_cast<float *>(p.Y)[(int64_t)row * p.ldy + col] = v;
    else reinterpret_cast<uint16_t *>(p.Y)[(int64_t)row * p.ldy + col] = (uint16_t)f32_to_16_bits<F16>(v);
}
// T over the wavefronts' sums in LDS, STRIDE floats apart.
template <int STRIDE>
__device__ __forceinline__ float tree_of_waves(const float *red, int active, int at) {
    float v[W4_WAVES];
#pragma unroll
    for (int w = 0; w < W4_WAVES; ++w) v[w] = red[w < active ? w * STRIDE + at : at];
#pragma unroll
    for (int s = 1; s < W4_WAVES; s *= 2)
#pragma unroll
        for (int r = 0; r < W4_WAVES; r += 2 * s)
            if (r + s < active) v[r] = v[r] + v[r + s];
    return v[0];
}

}  // namespace tbik
