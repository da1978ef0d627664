// Tree-Based MatMul of 16-bit rows on a 4-bit weight with a scale per group of consecutive k and channel.
//
//   Y[m,n] = T over superleaves of  sum over groups g of the superleaf, ascending:  acc = fma(scale[n,g], S_g, acc), acc from +0
//   S_g    = sum over k of the group of  x[m,k] (q[n,k] - zero[n,g])     chained matrix instructions from +0
// q - zero is a whole number of -15 .. 15 and exact in either 16-bit format, so the weight is never rounded: the scale multiplies a
// group's fp32 sum, once per group, row and channel.  How an element becomes a 16-bit float is at widened_levels.
//
// An instruction multiplies 16 k of 32 channels; which 16 of a unit of 64 (or 32, for groups that no 64 divides) it takes is chosen so that a
// lane's elements of the whole unit are 16 (8) consecutive bytes: half of the lanes take the unit's first half, the others its second.  The three
// kernels below share that map, the chains and the tree, so they give the same bits:
//   slices   up to 16 rows in one launch: a workgroup takes 32 channels and all of a shard's K, its eight wavefronts consecutive superleaves each (whole and in
//            order: Sec. 4.2, App. D.1); each streams its part of the weight, of the rows and of the scales through a ring of stages in
//            LDS of its own (direct global->LDS loads, no barrier until the sums are there), and the upper levels of the tree run over their sums (App. C)
//   tiles    more rows: a workgroup takes 128 channels and 32, 64 or 128 rows, which its four wavefronts share; few tiles split K (fp32 planes, combined by
//            the same tree), which the rows' traffic decides: a slice would read all of X for every 32 channels
//   general  any legal shape, operands straight from memory to registers
#include <algorithm>
#include <atomic>
#include <type_traits>

#include "tbik_device.hpp"
#include "tbik_internal.hpp"
#include "tile_store.hpp"
#include "tree_walk.hpp"

namespace tbik {

namespace {

struct W4Params {
    const uint16_t *X;
    const uint8_t *W;
    const uint16_t *scales;
    const uint8_t *zeros;
    float *partials;
    void *Y;
    int64_t ldx, ldw, lds, ldz, ldy;
    int M, N;
    int y_f32;
    int group, superleaf;
    int leaves_per_wave, active_waves, leaves_per_shard;
    int vector_stores;
    int row_bytes;                         // slices of one row: LDS for the row's part of a wavefront's k, whole loads
};

typedef uint32_t w4_u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t w4_u32x2 __attribute__((ext_vector_type(2)));

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



constexpr int W4_WAVES = 8;                // of a slice, and of the general kernel's workgroup

// ---- stages in LDS (slices and tiles) ----
// A stage is 64 S k.  Of one wavefront it holds rows of X (128 S bytes), the 32 S bytes of each of 32 channels, and a dword per lane and pair of units with the
// scale (and one with the zero point) of the unit's group: lanes 0 .. 31 the even unit, lanes 32 .. 63 the odd one.  Chunks of 16 bytes are swapped
// about within a row so that the rows of a read meet different banks.
// S = 2 where superleaves are whole stages of 128 k: with 64, whose 32 bytes of a channel are a quarter of a cache line, the weight alone came in at
// 1.6 TB/s (27 rows, K = 12288, N = 4096 without the loads of X and the scales 16.6 us).
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
    int g, left;
    int units;                             // of a group
    __device__ __forceinline__ explicit GroupWalk(int units_per_group) : g(0), left(units_per_group), units(units_per_group) {}
    __device__ __forceinline__ bool next() {       // true: the unit was the group's last
        if (--left != 0) return false;
        left = units;
        ++g;
        return true;
    }
};

// One wavefront's stream of weight, scales and zero points: 32 channels from n0 on, k from k0 on.
template <int UNIT, bool ZEROS, int S>
struct W4Stream {
    static constexpr int UNITS = 64 * S / UNIT, PAIRS = (UNITS + 1) / 2;
    static constexpr int LOADS = S + PAIRS * (ZEROS ? 2 : 1);
    static constexpr int SCALES = S * 1024, ZERO_POINTS = SCALES + PAIRS * 256, BYTES = ZERO_POINTS + (ZEROS ? PAIRS * 256 : 0);
    const char *w_ptr, *s_ptr, *z_ptr;
    unsigned w_off[S], s_off, z_off;       // of the lane; s_off and z_off count from an aligned dword
    GroupWalk walk;                        // of the stream's next unit

    __device__ __forceinline__ W4Stream(const W4Params &p, int n0, int64_t k0, int lane) : walk(p.group / UNIT) {
        const uint8_t *w = p.W + n0 * p.ldw + k0 / 2;
        const uint16_t *sc = p.scales + n0 * p.lds + k0 / p.group;
        w_ptr = uniform_pointer(reinterpret_cast<const char *>(w));
#pragma unroll
        for (int j = 0; j < S; ++j) {      // 64 chunks each, 2 S of a channel
            const int r = j * (32 / S) + lane / (2 * S), c = (lane % (2 * S)) ^ w_swizzle<S>(r);
            w_off[j] = (unsigned)(min(r, p.N - 1 - n0) * (int)p.ldw + c * 16);
        }
        const int channel = min(lane & 31, p.N - 1 - n0);
        const unsigned s_low = (unsigned)(reinterpret_cast<uintptr_t>(sc) & 3);
        s_ptr = uniform_pointer(reinterpret_cast<const char *>(sc) - s_low);
        s_off = s_low + (unsigned)(channel * (int)p.lds) * 2u;
        z_ptr = nullptr;
        z_off = 0;
        if constexpr (ZEROS) {
            const uint8_t *z = p.zeros + n0 * p.ldz + k0 / p.group;
            const unsigned z_low = (unsigned)(reinterpret_cast<uintptr_t>(z) & 3);
            z_ptr = uniform_pointer(reinterpret_cast<const char *>(z) - z_low);
            z_off = z_low + (unsigned)(channel * (int)p.ldz);
        }
    }
    // The next stage's loads to LDS address `at` (uniform): weight, scales, zero points.  A scale's dword holds its neighbour too.
    // `more`: there is a stage behind it; else the next issue loads it again.
    __device__ __forceinline__ void issue(unsigned at, int lane, bool more) {
#pragma unroll
        for (int j = 0; j < S; ++j) load_16B_per_lane_to_lds<0, true>(w_ptr, w_off[j], at + j * 1024);
        GroupWalk behind = walk;
#pragma unroll
        for (int q = 0; q < PAIRS; ++q) {
            int g = behind.g;
            behind.next();
            if constexpr (UNITS > 1) {
                if (lane >= 32) g = behind.g;
                behind.next();
            }
            load_4B_per_lane_to_lds<0, true>(s_ptr, (s_off + 2u * g) & ~3u, at + SCALES + q * 256);
            if constexpr (ZEROS) load_4B_per_lane_to_lds<0, true>(z_ptr, (z_off + g) & ~3u, at + ZERO_POINTS + q * 256);
        }
        if (more) {
            walk = behind;
            w_ptr += 32 * S;
        }
    }
    // From the stage at `st` in LDS, for unit u of it, which is group g's.
    template <bool F16>
    __device__ __forceinline__ ZeroPoint<F16, ZEROS> zero(const unsigned char *st, int u, int g, int li) const {
        const unsigned z = *reinterpret_cast<const unsigned *>(st + ZERO_POINTS + (u * 32 + li) * 4);
        return ZeroPoint<F16, ZEROS>((int)((z >> (8u * ((z_off + g) & 3u))) & 15u));
    }
    template <bool F16>
    __device__ __forceinline__ float scale(const unsigned char *st, int u, int g, int li) const {
        const unsigned s = *reinterpret_cast<const unsigned *>(st + SCALES + (u * 32 + li) * 4);
        return widened_16<F16>((uint16_t)(s >> (8u * ((s_off + 2u * g) & 2u)))) * kLevelUnit<F16, ZEROS>;
    }
};

// Multiplies a stage: rows x_rows[a] (the lane's row of X in the stage, in LDS) times the stage's weight at st.  sum: the running group's; a group
// that ends goes through its scale into acc.
template <int UNIT, bool F16, bool ZEROS, int S, int MT>
__device__ __forceinline__ void multiply_stage(const W4Stream<UNIT, ZEROS, S> &stream, const unsigned char *st, const unsigned char *const (&x_rows)[MT], int x_sw,
                                               GroupWalk &walk, Acc<MT, 1> &sum, Acc<MT, 1> &acc, int li, int lg) {
    const int w_sw = w_swizzle<S>(li);
#pragma unroll
    for (int h = 0; h < S; ++h) {                      // 64 k each
        w4_u32x4 words;
        if constexpr (UNIT == 64) {
            words = *reinterpret_cast<const w4_u32x4 *>(st + li * (32 * S) + (((2 * h + lg) ^ w_sw) << 4));
        } else {
            const w4_u32x2 a = *reinterpret_cast<const w4_u32x2 *>(st + li * (32 * S) + (((2 * h) ^ w_sw) << 4) + lg * 8),
                           b = *reinterpret_cast<const w4_u32x2 *>(st + li * (32 * S) + (((2 * h + 1) ^ w_sw) << 4) + lg * 8);
            words = w4_u32x4{a[0], a[1], b[0], b[1]};
        }
        bf16x8 x[4][MT];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int chunk = 8 * h + (UNIT == 64 ? lg * 4 + i : (i >> 1) * 4 + lg * 2 + (i & 1));
#pragma unroll
            for (int a = 0; a < MT; ++a) x[i][a] = *reinterpret_cast<const bf16x8 *>(x_rows[a] + ((chunk ^ x_sw) << 4));
        }
        constexpr int UNITS = 64 / UNIT;
#pragma unroll
        for (int u = 0; u < UNITS; ++u) {
            ZeroPoint<F16, ZEROS> zero;
            if constexpr (ZEROS) zero = stream.template zero<F16>(st, h * UNITS + u, walk.g, li);
            const float scale = stream.template scale<F16>(st, h * UNITS + u, walk.g, li);
#pragma unroll
            for (int i = u * (4 / UNITS); i < (u + 1) * (4 / UNITS); ++i) {
                const bf16x8 w = widened_levels<F16, ZEROS>(words[i], zero);
#pragma unroll
                for (int a = 0; a < MT; ++a) sum.t[a][0] = mfma_32x32x16<F16>(x[i][a], w, sum.t[a][0]);
            }
            if (walk.next()) {
#pragma unroll
                for (int a = 0; a < MT; ++a)
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        acc.t[a][0][r] = __builtin_fmaf(scale, sum.t[a][0][r], acc.t[a][0][r]);
                        sum.t[a][0][r] = 0.0f;
                    }
            }
        }
    }
}

template <int MT>
__device__ __forceinline__ void clear(Acc<MT, 1> &acc) {
#pragma unroll
    for (int a = 0; a < MT; ++a)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc.t[a][0][r] = 0.0f;
}

// The wavefronts' sums in LDS (32 x 32 each), four wavefronts or eight: T over them for element `at`.
__device__ __forceinline__ float tree_of_waves(const float *red, int active, int at) {
    float v[W4_WAVES];
#pragma unroll
    for (int w = 0; w < W4_WAVES; ++w) v[w] = red[w < active ? w * 1024 + at : at];
#pragma unroll
    for (int s = 1; s < W4_WAVES; s *= 2)
#pragma unroll
        for (int r = 0; r < W4_WAVES; r += 2 * s)
            if (r + s < active) v[r] = v[r] + v[r + s];
    return v[0];
}
template <bool F16>
__device__ __forceinline__ void store_sum(const W4Params &p, int shard, int row, int col, float v) {
    if (p.partials) p.partials[((int64_t)shard * p.M + row) * p.N + col] = v;
    else if (p.y_f32) reinterpret_cast<float *>(p.Y)[(int64_t)row * p.ldy + col] = v;
    else reinterpret_cast<uint16_t *>(p.Y)[(int64_t)row * p.ldy + col] = (uint16_t)f32_to_16_bits<F16>(v);
}

template <int REST, class Consume>
__device__ __forceinline__ void w4_last_stages(int stages, Consume &consume) {
    if (stages > REST) consume(std::integral_constant<int, REST>{}, std::false_type{});
    if constexpr (REST > 0) w4_last_stages<REST - 1>(stages, consume);
}

// XR: rows of X in a stage, 8 or 16; or 1: the one row's part of the wavefront's k lies behind its ring from the start.  LEVELS: of the tree in a wavefront.
template <int UNIT, bool F16, bool ZEROS, int S, int XR, int RING, int LEVELS>
__global__ __launch_bounds__(64 * W4_WAVES, (RING == 2 || XR == 1) && LEVELS <= 1 ? 4 : 2) void gemm_w4_slice_kernel(const W4Params p) {
    using Stream = W4Stream<UNIT, ZEROS, S>;
    constexpr bool ONE = XR == 1;
    constexpr int X_LOADS = ONE ? 0 : XR * S / 8, X_BYTES = X_LOADS * 1024, STAGE = X_BYTES + Stream::BYTES, LOADS = X_LOADS + Stream::LOADS;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int li = lane & 31, lg = lane >> 5;
    const int n0 = blockIdx.x * 32;
    Acc<1, 1> acc;
    if (wave < p.active_waves) {
        const int64_t k0 = (int64_t)(blockIdx.z * p.leaves_per_shard + wave * p.leaves_per_wave) * p.superleaf;
        const int stages_per_leaf = p.superleaf / (64 * S), stages = p.leaves_per_wave * stages_per_leaf;
        Stream stream(p, n0, k0, lane);
        const char *x_ptr = uniform_pointer(reinterpret_cast<const char *>(p.X + k0));
        unsigned x_off[ONE ? 1 : X_LOADS];
#pragma unroll
        for (int j = 0; j < X_LOADS; ++j) {            // rows behind the last one read it once more; they are not stored
            const int r = j * (8 / S) + lane / (8 * S), c = (lane % (8 * S)) ^ x_swizzle<S>(r);
            x_off[j] = (unsigned)(min(r, p.M - 1) * (int)p.ldx + c * 8) * 2u;
        }
        const int wave_bytes = RING * STAGE + (ONE ? p.row_bytes : 0);
        const unsigned ring = (unsigned)(uintptr_t)(__attribute__((address_space(3))) unsigned char *)smem + wave * wave_bytes;
        if constexpr (ONE) {                           // 512 k a load; behind the part's end its last chunk
            for (int j = 0; j * 1024 < p.row_bytes; ++j)
                load_16B_per_lane_to_lds<0, true>(x_ptr, (unsigned)min(j * 1024 + lane * 16, stages * (128 * S) - 16), ring + RING * STAGE + j * 1024);
        }
        auto issue = [&](int slot) __attribute__((always_inline)) {
            const unsigned at = ring + slot * STAGE;
#pragma unroll
            for (int j = 0; j < X_LOADS; ++j) load_16B_per_lane_to_lds<0, true>(x_ptr, x_off[j], at + j * 1024);
            x_ptr += 128 * S;
            stream.issue(at + X_BYTES, lane, true);
        };
        const unsigned char *const mine = smem + wave * wave_bytes;
        const int xr = li & (XR - 1), x_sw = ONE ? 0 : x_swizzle<S>(xr);
        const unsigned char *row = mine + RING * STAGE;
        GroupWalk walk(p.group / UNIT);
        Acc<1, 1> sum;
        f32x16 stash[LEVELS > 0 ? LEVELS : 1];
        int left = stages_per_leaf, leaf = 0, slot = 0;
        clear(acc);
        clear(sum);
        auto consume = [&](auto rest, auto again) __attribute__((always_inline)) {
            w4_wait_loads<decltype(rest)::value * LOADS>();
            const unsigned char *const st = mine + slot * STAGE;
            const unsigned char *const x_rows[1] = {ONE ? row : st + xr * (128 * S)};
            row += 128 * S;
            multiply_stage<UNIT, F16, ZEROS, S, 1>(stream, st + X_BYTES, x_rows, x_sw, walk, sum, acc, li, lg);
            if constexpr (decltype(again)::value) {    // the stage's bytes are in registers before its slot is filled again
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                issue(slot);
            }
            slot = slot + 1 == RING ? 0 : slot + 1;
            if (--left == 0) {                         // a superleaf ends: the carry-over step of the tree
                left = stages_per_leaf;
                const int t = __builtin_ctz(~leaf);
#pragma unroll
                for (int l = 0; l < LEVELS; ++l)
                    if (l < t) {
#pragma unroll
                        for (int r = 0; r < 16; ++r) acc.t[0][0][r] = stash[l][r] + acc.t[0][0][r];
                    }
                if (++leaf < p.leaves_per_wave) {
#pragma unroll
                    for (int l = 0; l < LEVELS; ++l)
                        if (l == t) stash[l] = acc.t[0][0];
                    clear(acc);
                }
            }
        };
#pragma unroll
        for (int i = 0; i < RING; ++i)
            if (i < stages) issue(i);
        for (int s = RING; s < stages; ++s) consume(std::integral_constant<int, RING - 1>{}, std::true_type{});
        w4_last_stages<RING - 1>(stages, consume);
    }
    __syncthreads();                                   // the rings have been read: the sums take their place
    float *const red = reinterpret_cast<float *>(smem);
    if (wave < p.active_waves) {
#pragma unroll
        for (int r = 0; r < 16; ++r) red[wave * 1024 + (8 * (r >> 2) + 4 * lg + (r & 3)) * 32 + li] = acc.t[0][0][r];
    }
    __syncthreads();
    const int row = threadIdx.x / 32, col = n0 + threadIdx.x % 32;                 // 16 rows of 32
    if (row < p.M && col < p.N) store_sum<F16>(p, blockIdx.z, row, col, tree_of_waves(red, p.active_waves, threadIdx.x));
}

// 32 MT rows times 128 channels; four wavefronts share the rows of X in LDS.  blockIdx.z: the shard or the part of a split K.
// KG: groups of four wavefronts that halve the part's superleaves among them, the upper half's sums joined in LDS: with few rows a wavefront's conversions
// and its matrix instructions take turns, and a second one on its vector unit fills the gaps.
template <int UNIT, bool F16, bool ZEROS, int S, int MT, int RING, int KG>
__global__ __launch_bounds__(256 * KG, MT == 4 ? 1 : 2) void gemm_w4_tiled_kernel(const W4Params p) {
    using Stream = W4Stream<UNIT, ZEROS, S>;
    constexpr int X_LOADS = MT * S, REGION = X_LOADS * 1024 + Stream::BYTES, STAGE = 4 * REGION, LOADS = X_LOADS + Stream::LOADS;      // a region is what one wavefront loads
    extern __shared__ __attribute__((aligned(16))) unsigned char all_smem[];
    const int lane = threadIdx.x & 63, every_wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wave = every_wave & 3, part = every_wave >> 2;
    unsigned char *const smem = all_smem + part * (RING * STAGE);
    const int li = lane & 31, lg = lane >> 5;
    const int m0 = blockIdx.y * 32 * MT, n0 = blockIdx.x * 128 + wave * 32;
    const int leaves = p.leaves_per_shard / KG;
    const int64_t k0 = (int64_t)(blockIdx.z * p.leaves_per_shard + part * leaves) * p.superleaf;
    const int stages_per_leaf = p.superleaf / (64 * S), stages = leaves * stages_per_leaf;
    Stream stream(p, min(n0, p.N - 1), k0, lane);
    const char *x_ptr = uniform_pointer(reinterpret_cast<const char *>(p.X + (int64_t)m0 * p.ldx + k0));
    unsigned x_off[X_LOADS];
#pragma unroll
    for (int j = 0; j < X_LOADS; ++j) {                // 8 / S rows each; rows behind the last one read it once more
        const int r = wave * 8 * MT + j * (8 / S) + lane / (8 * S), c = (lane % (8 * S)) ^ x_swizzle<S>(r);
        x_off[j] = (unsigned)(min(r, p.M - 1 - m0) * (int)p.ldx + c * 8) * 2u;
    }
    const unsigned lds = (unsigned)(uintptr_t)(__attribute__((address_space(3))) unsigned char *)smem + wave * REGION;
    int to_issue = stages;                             // stages that are not yet on their way
    auto issue = [&](int slot) __attribute__((always_inline)) {
        const unsigned at = lds + slot * STAGE;
#pragma unroll
        for (int j = 0; j < X_LOADS; ++j) load_16B_per_lane_to_lds<0, true>(x_ptr, x_off[j], at + j * 1024);
        const bool more = --to_issue > 0;              // the last stage is loaded again behind itself (nobody consumes it)
        stream.issue(at + X_LOADS * 1024, lane, more);
        if (more) x_ptr += 128 * S;
    };
    int x_at[MT];
#pragma unroll
    for (int a = 0; a < MT; ++a) {
        const int r = a * 32 + li;
        x_at[a] = (r / (8 * MT)) * REGION + (r % (8 * MT)) * (128 * S);
    }
    const int x_sw = x_swizzle<S>(li);                 // of every one of the lane's rows
    GroupWalk walk(p.group / UNIT);
    int cur = 0;
    Acc<MT, 1> acc, sum;
    f32x16 stash[MT][4];                               // finished subtrees of up to 16 superleaves
    clear(sum);
    clear(acc);
#pragma unroll
    for (int i = 0; i < RING - 1; ++i) issue(i);
    for (int leaf = 0; leaf < leaves; ++leaf) {
#pragma nounroll
        for (int s = 0; s < stages_per_leaf; ++s) {
            // Own loads of this stage have landed, and behind the barrier everybody's; the slot of the stage before has been read.
            w4_wait_loads_and_barrier<LOADS * (RING - 2)>();
            issue(cur == 0 ? RING - 1 : cur - 1);
            const unsigned char *const st = smem + cur * STAGE;
            const unsigned char *x_rows[MT];
#pragma unroll
            for (int i = 0; i < MT; ++i) x_rows[i] = st + x_at[i];
            multiply_stage<UNIT, F16, ZEROS, S, MT>(stream, st + wave * REGION + X_LOADS * 1024, x_rows, x_sw, walk, sum, acc, li, lg);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            cur = cur + 1 == RING ? 0 : cur + 1;
        }
        const int t = __builtin_ctz(~leaf);            // a superleaf ends: the carry-over step of the tree
        const bool more = leaf + 1 < leaves;
#pragma unroll
        for (int a = 0; a < MT; ++a) {
#pragma unroll
            for (int l = 0; l < 4; ++l)
                if (l < t) {
#pragma unroll
                    for (int r = 0; r < 16; ++r) acc.t[a][0][r] = stash[a][l][r] + acc.t[a][0][r];
                }
        }
        if (more) {
#pragma unroll
            for (int a = 0; a < MT; ++a) {
#pragma unroll
                for (int l = 0; l < 4; ++l)
                    if (l == t) stash[a][l] = acc.t[a][0];
            }
            clear(acc);
        }
    }
    w4_wait_loads_and_barrier<0>();                    // no load may still be writing LDS; all stages have been read
    if constexpr (KG == 2) {                           // left half + right half, the last level of the tree
        float *const half = reinterpret_cast<float *>(all_smem) + wave * (MT * 1024);
        if (part == 1) {
#pragma unroll
            for (int a = 0; a < MT; ++a)
#pragma unroll
                for (int r = 0; r < 16; ++r) half[a * 1024 + r * 64 + lane] = acc.t[a][0][r];
        }
        __syncthreads();
        if (part == 1) return;
#pragma unroll
        for (int a = 0; a < MT; ++a)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc.t[a][0][r] = acc.t[a][0][r] + half[a * 1024 + r * 64 + lane];
    }
    const int last = min(p.M - 1 - m0, 32 * MT - 1);
    if (n0 >= p.N) return;
    float *const patch = reinterpret_cast<float *>(all_smem) + wave * (MT * 1024);
    if (p.vector_stores && n0 + 32 <= p.N) {
        if (p.partials) store_ragged_f32(acc, patch, p.partials + ((int64_t)blockIdx.z * p.M + m0) * p.N + n0, p.N, last, lane, false);
        else if (p.y_f32) store_ragged_f32(acc, patch, reinterpret_cast<float *>(p.Y) + (int64_t)m0 * p.ldy + n0, p.ldy, last, lane, false);
        else store_ragged_16bit<F16>(acc, patch, reinterpret_cast<uint16_t *>(p.Y) + (int64_t)m0 * p.ldy + n0, p.ldy, last, lane);
        return;
    }
    if (n0 + li >= p.N) return;
#pragma unroll
    for (int a = 0; a < MT; ++a)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int row = a * 32 + 8 * (r >> 2) + 4 * lg + (r & 3);
            if (row <= last) store_sum<F16>(p, blockIdx.z, m0 + row, n0 + li, acc.t[a][0][r]);
        }
}

// ---- any legal shape ----
// UNIT: k of a lane pair's unit, 64 or 32.
template <int UNIT, bool F16, bool ZEROS>
__global__ __launch_bounds__(64 * W4_WAVES, 2) void gemm_w4_kernel(const W4Params p) {
    constexpr int STEPS = UNIT / 16, DEPTH = UNIT == 64 ? 4 : 8;
    using Words = std::conditional_t<UNIT == 64, w4_u32x4, w4_u32x2>;
    __shared__ float red[W4_WAVES * 1024];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int li = lane & 31, lg = lane >> 5;
    const int n0 = blockIdx.x * 32, m0 = blockIdx.y * 32;
    const int first_leaf = blockIdx.z * p.leaves_per_shard + wave * p.leaves_per_wave;
    f32x16 acc;
    if (wave < p.active_waves) {
        const int channel = min(n0 + li, p.N - 1);
        const int64_t k0 = (int64_t)first_leaf * p.superleaf;
        const uint8_t *w_at = p.W + channel * p.ldw + k0 / 2 + lg * (UNIT / 4);
        const uint16_t *s_at = p.scales + channel * p.lds + k0 / p.group;
        const uint8_t *z_at = ZEROS ? p.zeros + channel * p.ldz + k0 / p.group : nullptr;
        // Rows behind the last one read it once more; they are not stored.
        const uint16_t *x_at = p.X + (int64_t)min(m0 + li, p.M - 1) * p.ldx + k0 + lg * (UNIT / 2);
        const int units = p.leaves_per_wave * (p.superleaf / UNIT), units_per_group = p.group / UNIT, groups_per_leaf = p.superleaf / p.group;
        Words w[DEPTH];
        uint4 x[DEPTH][STEPS];
        auto fetch = [&](int d) __attribute__((always_inline)) {
            w[d] = *reinterpret_cast<const Words *>(w_at);
#pragma unroll
            for (int i = 0; i < STEPS; ++i) x[d][i] = *reinterpret_cast<const uint4 *>(x_at + 8 * i);
            w_at += UNIT / 2;
            x_at += UNIT;
        };
#pragma unroll
        for (int d = 0; d < DEPTH; ++d)
            if (d < units) fetch(d);
        f32x16 stash[4], sum;
        int left_in_group = units_per_group, left_in_leaf = groups_per_leaf, leaf = 0;
        float scale = widened_16<F16>(*s_at) * kLevelUnit<F16, ZEROS>;              // of the group that is being summed
        ZeroPoint<F16, ZEROS> zero;
        if constexpr (ZEROS) zero = ZeroPoint<F16, ZEROS>(*z_at & 15);
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[r] = sum[r] = 0.0f;
        for (int u0 = 0; u0 < units; u0 += DEPTH) {
#pragma unroll
            for (int d = 0; d < DEPTH; ++d) {
                if (u0 + d >= units) continue;
#pragma unroll
                for (int i = 0; i < STEPS; ++i)
                    sum = mfma_32x32x16<F16>(__builtin_bit_cast(bf16x8, x[d][i]), widened_levels<F16, ZEROS>(w[d][i], zero), sum);
                if (u0 + d + DEPTH < units) fetch(d);
                if (--left_in_group == 0) {
                    left_in_group = units_per_group;
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        acc[r] = __builtin_fmaf(scale, sum[r], acc[r]);
                        sum[r] = 0.0f;
                    }
                    if (u0 + d + 1 < units) {
                        scale = widened_16<F16>(*++s_at) * kLevelUnit<F16, ZEROS>;
                        if constexpr (ZEROS) zero = ZeroPoint<F16, ZEROS>(*++z_at & 15);
                    }
                    if (--left_in_leaf == 0) {                                      // a superleaf ends: the carry-over step of the tree
                        left_in_leaf = groups_per_leaf;
                        const int t = __builtin_ctz(~leaf);
#pragma unroll
                        for (int l = 0; l < 4; ++l)
                            if (l < t) {
#pragma unroll
                                for (int r = 0; r < 16; ++r) acc[r] = stash[l][r] + acc[r];
                            }
                        if (++leaf < p.leaves_per_wave) {
#pragma unroll
                            for (int l = 0; l < 4; ++l)
                                if (l == t) stash[l] = acc;
#pragma unroll
                            for (int r = 0; r < 16; ++r) acc[r] = 0.0f;
                        }
                    }
                }
            }
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) red[wave * 1024 + (8 * (r >> 2) + 4 * lg + (r & 3)) * 32 + li] = acc[r];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 1024 / (64 * W4_WAVES); ++i) {
        const int at = i * 64 * W4_WAVES + threadIdx.x, row = m0 + at / 32, col = n0 + at % 32;
        if (row >= p.M || col >= p.N) continue;
        float v[W4_WAVES];
#pragma unroll
        for (int w = 0; w < W4_WAVES; ++w) v[w] = red[w < p.active_waves ? w * 1024 + at : at];
#pragma unroll
        for (int s = 1; s < W4_WAVES; s *= 2)
#pragma unroll
            for (int r = 0; r < W4_WAVES; r += 2 * s)
                if (r + s < p.active_waves) v[r] = v[r] + v[r + s];
        if (p.partials) p.partials[((int64_t)blockIdx.z * p.M + row) * p.N + col] = v[0];
        else if (p.y_f32) reinterpret_cast<float *>(p.Y)[(int64_t)row * p.ldy + col] = v[0];
        else reinterpret_cast<uint16_t *>(p.Y)[(int64_t)row * p.ldy + col] = (uint16_t)f32_to_16_bits<F16>(v[0]);
    }
}

template <class Kernel>
hipError_t allow_lds(Kernel k, int lds, std::atomic<unsigned> &allowed) {
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 32) dev = 32;      // 32: not remembered, set every time
    if (dev >= 32 || !((allowed.load(std::memory_order_relaxed) >> dev) & 1u)) { // bit d: the attribute is set on device d
        const hipError_t e = hipFuncSetAttribute((const void *)k, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
        if (e != hipSuccess) return e;
        if (dev < 32) allowed.fetch_or(1u << dev, std::memory_order_relaxed);
    }
    return hipSuccess;
}

template <int UNIT, bool F16, bool ZEROS, int S, int XR, int RING, int LEVELS>
hipError_t launch_slice_of(const W4Params &p, int shards, hipStream_t s) {
    constexpr int ring = RING * ((XR == 1 ? 0 : XR * S * 128) + W4Stream<UNIT, ZEROS, S>::BYTES);
    static_assert(W4_WAVES * ring <= 160 * 1024 && ring >= 4096, "LDS of a compute unit; room for the sums");
    const int lds = W4_WAVES * (ring + (XR == 1 ? p.row_bytes : 0));
    auto k = gemm_w4_slice_kernel<UNIT, F16, ZEROS, S, XR, RING, LEVELS>;
    static std::atomic<unsigned> allowed{0};
    const hipError_t e = allow_lds(k, XR == 1 ? 160 * 1024 : lds, allowed);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(k, dim3((unsigned)((p.N + 31) / 32), 1, (unsigned)shards), dim3(64 * W4_WAVES), lds, s, p);
    return hipGetLastError();
}
// Stages in flight: all that LDS holds while every workgroup has a compute unit to itself; with more workgroups than compute units two, which lets
// two workgroups share one.
template <int UNIT, bool F16, bool ZEROS, int S, int XR, int LEVELS>
hipError_t launch_slice(const W4Params &p, int shards, hipStream_t s) {
    constexpr int deep = S == 1 ? (XR == 8 ? 6 : 4) : XR == 8 ? 3 : 2;
    const int64_t blocks = ((int64_t)p.N + 31) / 32 * shards;
    if (blocks <= 256) return launch_slice_of<UNIT, F16, ZEROS, S, XR, deep, LEVELS>(p, shards, s);
    return launch_slice_of<UNIT, F16, ZEROS, S, XR, 2, LEVELS>(p, shards, s);
}
template <int UNIT, bool F16, bool ZEROS, int S, int MT, int RING, int KG = 1>
hipError_t launch_tile(const W4Params &p, int shards, hipStream_t s) {
    constexpr int lds = KG * RING * 4 * (MT * S * 1024 + W4Stream<UNIT, ZEROS, S>::BYTES);
    static_assert(lds <= 160 * 1024 && lds >= 4 * MT * 4096, "LDS of a compute unit; room for the sums and the patches");
    auto k = gemm_w4_tiled_kernel<UNIT, F16, ZEROS, S, MT, RING, KG>;
    static std::atomic<unsigned> allowed{0};
    const hipError_t e = allow_lds(k, lds, allowed);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(k, dim3((unsigned)((p.N + 127) / 128), (unsigned)((p.M + 32 * MT - 1) / (32 * MT)), (unsigned)shards), dim3(256 * KG), lds, s, p);
    return hipGetLastError();
}

template <int UNIT, bool F16, bool ZEROS, int S>
hipError_t launch_slice_rows(const W4Params &all, int shards, hipStream_t s) {
    W4Params p = all;
    p.row_bytes = (p.leaves_per_wave * p.superleaf * 2 + 1023) & ~1023;
    if (p.M == 1 && p.row_bytes <= 8192) return p.leaves_per_wave <= 2 ? launch_slice_of<UNIT, F16, ZEROS, S, 1, S == 1 ? 5 : 3, 1>(p, shards, s) : launch_slice_of<UNIT, F16, ZEROS, S, 1, S == 1 ? 5 : 3, 4>(p, shards, s);
    if (p.M <= 8) return p.leaves_per_wave <= 2 ? launch_slice<UNIT, F16, ZEROS, S, 8, 1>(p, shards, s) : launch_slice<UNIT, F16, ZEROS, S, 8, 4>(p, shards, s);
    return p.leaves_per_wave <= 2 ? launch_slice<UNIT, F16, ZEROS, S, 16, 1>(p, shards, s) : launch_slice<UNIT, F16, ZEROS, S, 16, 4>(p, shards, s);
}
template <int UNIT, bool F16, bool ZEROS, int S>
hipError_t launch_tile_rows(const W4Params &p, int shards, hipStream_t s) {
    const bool halves = p.leaves_per_shard % 2 == 0;
    if (p.M <= 32) return halves ? launch_tile<UNIT, F16, ZEROS, S, 1, S == 1 ? 6 : 4, 2>(p, shards, s) : launch_tile<UNIT, F16, ZEROS, S, 1, S == 1 ? 6 : 4>(p, shards, s);
    if (p.M <= 64) return halves ? launch_tile<UNIT, F16, ZEROS, S, 2, S == 1 ? 5 : 2, 2>(p, shards, s) : launch_tile<UNIT, F16, ZEROS, S, 2, S == 1 ? 5 : 3>(p, shards, s);
    return launch_tile<UNIT, F16, ZEROS, S, 4, S == 1 ? 6 : 3>(p, shards, s);
}
template <int UNIT, bool F16, bool ZEROS>
hipError_t launch_w4_of(const W4Args &a, const W4Params &all, hipStream_t s) {
    W4Params p = all;
    const int ns = a.ns / a.P;                         // superleaves of a shard
    switch (w4_kernel(a)) {
        case W4_SLICES:
            p.leaves_per_wave = ns > W4_WAVES ? ns / W4_WAVES : 1;
            p.active_waves = ns > W4_WAVES ? W4_WAVES : ns;
            return a.superleaf % 128 == 0 ? launch_slice_rows<UNIT, F16, ZEROS, 2>(p, a.P, s) : launch_slice_rows<UNIT, F16, ZEROS, 1>(p, a.P, s);
        case W4_TILES: return a.superleaf % 128 == 0 ? launch_tile_rows<UNIT, F16, ZEROS, 2>(p, a.P, s) : launch_tile_rows<UNIT, F16, ZEROS, 1>(p, a.P, s);
        default: {
            p.leaves_per_wave = ns > W4_WAVES ? ns / W4_WAVES : 1;
            p.active_waves = ns > W4_WAVES ? W4_WAVES : ns;
            if (p.leaves_per_wave > 16) return hipErrorInvalidValue;
            for (int64_t m0 = 0; m0 < a.M; m0 += 32 * 4096) {          // 4096 row tiles a launch
                W4Params q = p;
                q.M = (int)(a.M - m0 < 32 * 4096 ? a.M - m0 : 32 * 4096);
                q.X += m0 * a.ldx;
                if (q.Y) q.Y = static_cast<char *>(q.Y) + m0 * a.ldy * (p.y_f32 ? 4 : 2);
                if (q.partials) q.partials += m0 * a.N;
                hipLaunchKernelGGL((gemm_w4_kernel<UNIT, F16, ZEROS>), dim3((unsigned)((a.N + 31) / 32), (unsigned)((q.M + 31) / 32), (unsigned)a.P), dim3(64 * W4_WAVES), 0, s, q);
            }
            return hipGetLastError();
        }
    }
}

}  // namespace

// Slices up to 16 rows, tiles beyond; `a.P`: shards, or the parts of a split K.
int w4_kernel(const W4Args &a) {
    const int ns = a.ns / a.P;
    const bool ring = a.superleaf % 64 == 0 && a.ldx < (1 << 22) && a.ldw < (1 << 22) && a.lds < (1 << 22) && a.ldz < (1 << 22);      // 32-bit lane offsets
    if (!ring) return W4_GENERAL;
    if (a.M <= 16) return W4_SLICES;
    return ns <= 16 && (int64_t)a.M <= 32 * 65535 ? W4_TILES : W4_GENERAL;
}

hipError_t launch_gemm_w4(const W4Args &a, hipStream_t s) {
    if (a.M <= 0 || a.N <= 0) return hipSuccess;
    W4Params p;
    p.X = a.X; p.W = reinterpret_cast<const uint8_t *>(a.W); p.scales = a.scales; p.zeros = a.zeros;
    p.partials = a.partials; p.Y = a.Y;
    p.ldx = a.ldx; p.ldw = a.ldw; p.lds = a.lds; p.ldz = a.ldz; p.ldy = a.ldy;
    p.M = a.M; p.N = a.N;
    p.y_f32 = a.y_dtype == TBIK_F32;
    p.group = a.group; p.superleaf = a.superleaf;
    p.leaves_per_shard = a.ns / a.P;
    p.leaves_per_wave = p.active_waves = 0;
    const void *out = a.partials ? (const void *)a.partials : a.Y;
    const int64_t ld_bytes = a.partials ? (int64_t)a.N * 4 : a.ldy * (p.y_f32 ? 4 : 2);
    p.vector_stores = (reinterpret_cast<uintptr_t>(out) & 15) == 0 && ld_bytes % 16 == 0 && ld_bytes < kMaxVectorRowBytes;
    const bool f16 = a.x_dtype == TBIK_F16, zeros = a.zeros != nullptr;
    if (a.group % 64 == 0) {
        if (zeros) return f16 ? launch_w4_of<64, true, true>(a, p, s) : launch_w4_of<64, false, true>(a, p, s);
        return f16 ? launch_w4_of<64, true, false>(a, p, s) : launch_w4_of<64, false, false>(a, p, s);
    }
    if (zeros) return f16 ? launch_w4_of<32, true, true>(a, p, s) : launch_w4_of<32, false, true>(a, p, s);
    return f16 ? launch_w4_of<32, true, false>(a, p, s) : launch_w4_of<32, false, false>(a, p, s);
}

}  // namespace tbik
