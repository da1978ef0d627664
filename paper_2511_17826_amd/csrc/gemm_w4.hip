// Tree-Based MatMul of 16-bit rows on a 4-bit weight with a scale per group of consecutive k and channel.
//
//   Y[m,n] = T over superleaves of  sum over groups g of the superleaf, ascending:  acc = fma(scale[n,g], S_g, acc), acc from +0
//   S_g    = sum over k of the group of  x[m,k] (q[n,k] - zero[n,g])     chained matrix instructions from +0
// q - zero is a whole number of -15 .. 15 and exact in either 16-bit format, so the weight is never rounded: the scale multiplies a
// group's fp32 sum, once per group, row and channel.  How an element becomes a 16-bit float is at widened_levels.
//
// An instruction (16x16x32: of 16 rows and channels) multiplies 32 k; which 32 of a unit of 128 (64 in groups of 64, 32 where 128 does not divide the group else) it
// takes is chosen so that a lane's elements of the whole unit are 16 (8, 4) consecutive bytes: a quarter of the lanes takes a quarter of the unit.  The
// kernels share that map, the chains and the tree, so they give the same bits:
//   slices   16 rows: a workgroup takes 32 or 16 channels and all of a shard's K, its up to eight wavefronts consecutive superleaves each (whole and in
//            order: Sec. 4.2, App. D.1); each streams its part of the weight, of the rows and of the scales through a ring of stages in
//            LDS of its own (direct global->LDS loads, no barrier until the sums are there), and the upper levels of the tree run over their sums (App. C)
//   tiles    a workgroup takes 128 channels and 32 or 64 rows, which its wavefronts share; few tiles split K (fp32 planes, combined by
//            the same tree)
//   general  any legal shape, operands straight from memory to registers
// Slices read the weight once every 16 rows, tiles leave compute units idle where there are few of them: up to 16 rows are slices, and more where there would be
// up to W4_FEW_TILES tiles (shards counted).  Tiles / slices, us, without room for a split, bf16: K 12288 x N 4096, groups of 128, 32 rows (32 tiles) 48.0 / 19.0,
// 64 rows (32) 64.7 / 34.4, 128 rows (64) 64.9 / 64.0, 256 rows (128) 65 / 124; 2 shards, 64 rows (64) 33.8 / 27.1, 256 rows (256) 37 / 102; K 5120 x N 5120, 32
// rows (40) 21.7 / 12.1, 2 shards (80) 12.6 / 15.0; 8 shards of K 12288 x N 4096, 17 rows 10.0 / 34.6, 16 rows 10.4 / 10.6, one row 10.1 / 8.3.
// What bounds slices and low tiles is the latency of a stage, not a rate: LDS reads, 13 to 19 instructions to widen 8 elements of a lane, products that wait for
// them, with two wavefronts on a vector unit (27 rows, K 12288 x N 4096, fp16, groups of 64 with zero points: 13.5 us of a tile, without its loads 12.9 before
// the last steps, without widening and products 9.5, the empty kernel 5.2).
// This file holds the bf16 kernels, and gemm_w4_f16.hip those of fp16.
#include "w4.hpp"

#ifndef TBIK_W4_F16
#define TBIK_W4_F16 false
#endif

namespace tbik {

namespace {

template <int REST, class Consume>
__device__ __forceinline__ void w4_last_stages(int stages, Consume &consume) {
    if (stages > REST) consume(std::integral_constant<int, REST>{}, std::false_type{});
    if constexpr (REST > 0) w4_last_stages<REST - 1>(stages, consume);
}

// XR: rows of X in a stage, 8 or 16; or 1: the one row's part of the wavefront's k lies behind its ring from the start (K 4096 x N 12288 8.1 us instead of 8.4).
// LEVELS: of the tree in a wavefront.  blockIdx.y: 16 rows each.
template <int UNIT, bool WHOLE, bool F16, bool ZEROS, int S, int NB, int XR, int RING, int LEVELS>
__global__ __launch_bounds__(64 * W4_WAVES, XR == 1 ? (LEVELS == 1 && RING == 2 ? 6 : 4) : RING == 2 ? 4 : 2) void gemm_w4_slice_kernel(const W4Params p) {
    constexpr bool ONE = XR == 1;
    using Stream = W4Stream<ZEROS, S, NB>;
    constexpr int X_LOADS = ONE ? 0 : XR * S / 8, X_BYTES = X_LOADS * 1024, STAGE = X_BYTES + Stream::BYTES, LOADS = X_LOADS + Stream::LOADS;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n0 = blockIdx.x * (16 * NB), m0 = blockIdx.y * 16;
    W4Sums<1, NB> acc;
    const int first_leaf = blockIdx.z * p.leaves_per_shard + wave * p.leaves_per_wave, stages = p.leaves_per_wave * p.stages_per_leaf;
    const int row_at = RING * STAGE, groups_at = row_at + (ONE ? p.row_bytes : 0), wave_bytes = groups_at + p.group_bytes;
    const unsigned ring = (unsigned)(uintptr_t)(__attribute__((address_space(3))) unsigned char *)smem + wave * wave_bytes;
    const unsigned char *const mine = smem + wave * wave_bytes;
    Stream stream(p, n0, first_leaf, p.leaves_per_wave, lane, ring + groups_at, mine + groups_at);
    stream.issue_groups(0, lane);
    const char *x_ptr = uniform_pointer(reinterpret_cast<const char *>(p.X + (int64_t)m0 * p.ldx + (int64_t)first_leaf * p.superleaf));
    unsigned x_off[ONE ? 1 : X_LOADS];
#pragma unroll
    for (int j = 0; j < X_LOADS; ++j) {            // rows behind the last one read it once more; they are not stored
        const int r = j * (8 / S) + lane / (8 * S), c = (lane % (8 * S)) ^ x_swizzle<S>(r);
        x_off[j] = (unsigned)(min(r, p.M - 1 - m0) * (int)p.ldx + c * 8) * 2u;
    }
    if constexpr (ONE) {                           // 512 k a load; behind the part's end its last chunk
        for (int j = 0; j * 1024 < p.row_bytes; ++j)
            load_16B_per_lane_to_lds<0, true>(x_ptr, (unsigned)min(j * 1024 + lane * 16, stages * (128 * S) - 16), ring + row_at + j * 1024);
    }
    auto issue = [&](int slot) __attribute__((always_inline)) {
        const unsigned at = ring + slot * STAGE;
#pragma unroll
        for (int j = 0; j < X_LOADS; ++j) load_16B_per_lane_to_lds<0, true>(x_ptr, x_off[j], at + j * 1024);
        x_ptr += 128 * S;
        stream.issue(at + X_BYTES, true);
    };
#pragma unroll
    for (int i = 0; i < RING; ++i)
        if (i < stages) issue(i);
    const int xr = lane & 15 & (XR - 1), x_sw = ONE ? 0 : x_swizzle<S>(xr);
    const unsigned char *row = mine + row_at;
    W4Multiplier<UNIT, WHOLE, F16, ZEROS, S, 1, NB> multiplier(p, stream, lane);
    W4Stash<1, NB, LEVELS> stash;
    int left = p.stages_per_leaf, leaf = 0, slot = 0;
    acc.clear();
    auto consume = [&](auto rest, auto again) __attribute__((always_inline)) {
        w4_wait_loads<decltype(rest)::value * LOADS>();
        multiplier.prefetch_groups(stream, lane);
        const unsigned char *const st = mine + slot * STAGE;
        const unsigned char *const x_rows[1] = {ONE ? row : st + xr * (128 * S)};
        row += 128 * S;
        multiplier.stage(stream, st + X_BYTES, x_rows, x_sw, acc);
        if constexpr (decltype(again)::value) {    // the stage's bytes are in registers before its slot is filled again
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            issue(slot);
        }
        slot = slot + 1 == RING ? 0 : slot + 1;
        if (--left == 0) {                         // a superleaf ends
            left = p.stages_per_leaf;
            stash.push(acc, leaf, leaf + 1 < p.leaves_per_wave);
            ++leaf;
        }
    };
    for (int s = RING; s < stages; ++s) consume(std::integral_constant<int, RING - 1>{}, std::true_type{});
    w4_last_stages<RING - 1>(stages, consume);
    __syncthreads();                                   // the rings have been read: the sums take their place
    float *const red = reinterpret_cast<float *>(smem);
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int r = 0; r < 4; ++r) red[wave * 512 + (4 * (lane >> 4) + r) * 32 + b * 16 + (lane & 15)] = acc.t[0][b][r];
    __syncthreads();
    for (int at = threadIdx.x; at < 512; at += 64 * p.active_waves) {              // 16 rows of 32
        const int row = m0 + at / 32, channel = at % 32;
        if (row < p.M && channel < 16 * NB && n0 + channel < p.N) w4_store<F16>(p, blockIdx.z, row, n0 + channel, tree_of_waves<512>(red, p.active_waves, at));
    }
}

// 32 MT rows (MT 1 or 2) times 128 channels; four wavefronts share the rows of X in LDS.  blockIdx.z: the shard or the part of a split K.
// KG: groups of four wavefronts that halve the part's superleaves among them, the upper half's sums joined in LDS: with few rows a wavefront's conversions
// and its matrix instructions take turns, and a second one on its vector unit fills the gaps.  That is why there are no tiles of 128 rows, whose registers leave room
// for one: K 4096 x N 12288, 128 rows 33.8 us (64: 25.7), 256 rows 52.6 (49.2); K 5120 x N 5120, 192 rows 42.7 (25.6).  More stages in flight than these change nothing.
template <int UNIT, bool WHOLE, bool F16, bool ZEROS, int S, int MT, int RING, int KG>
__global__ __launch_bounds__(256 * KG, 2) void gemm_w4_tiled_kernel(const W4Params p) {
    using Stream = W4Stream<ZEROS, S>;
    constexpr int MR = 2 * MT;
    constexpr int X_LOADS = MT * S, REGION = X_LOADS * 1024 + Stream::BYTES, STAGE = 4 * REGION, LOADS = X_LOADS + Stream::LOADS;      // a region is what one wavefront loads
    extern __shared__ __attribute__((aligned(16))) unsigned char all_smem[];
    const int lane = threadIdx.x & 63, every_wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wave = every_wave & 3, part = every_wave >> 2;
    unsigned char *const smem = all_smem + part * (RING * STAGE);
    const int l16 = lane & 15, quarter = lane >> 4;
    const int m0 = blockIdx.y * 32 * MT, n0 = blockIdx.x * 128 + wave * 32;
    const int leaves = p.leaves_per_shard / KG, stages = leaves * p.stages_per_leaf;
    const int first_leaf = blockIdx.z * p.leaves_per_shard + part * leaves;
    const unsigned all_lds = (unsigned)(uintptr_t)(__attribute__((address_space(3))) unsigned char *)all_smem;
    const int groups_at = KG * RING * STAGE + every_wave * p.group_bytes;
    Stream stream(p, min(n0, p.N - 1), first_leaf, leaves, lane, all_lds + groups_at, all_smem + groups_at);
    stream.issue_groups(0, lane);
    const char *x_ptr = uniform_pointer(reinterpret_cast<const char *>(p.X + (int64_t)m0 * p.ldx + (int64_t)first_leaf * p.superleaf));
    unsigned x_off[X_LOADS];
#pragma unroll
    for (int j = 0; j < X_LOADS; ++j) {                // 8 / S rows each; rows behind the last one read it once more
        const int r = wave * 8 * MT + j * (8 / S) + lane / (8 * S), c = (lane % (8 * S)) ^ x_swizzle<S>(r);
        x_off[j] = (unsigned)(min(r, p.M - 1 - m0) * (int)p.ldx + c * 8) * 2u;
    }
    const unsigned lds = all_lds + part * (RING * STAGE) + wave * REGION;
    int to_issue = stages;                             // stages that are not yet on their way
    auto issue = [&](int slot) __attribute__((always_inline)) {
        const unsigned at = lds + slot * STAGE;
#pragma unroll
        for (int j = 0; j < X_LOADS; ++j) load_16B_per_lane_to_lds<0, true>(x_ptr, x_off[j], at + j * 1024);
        const bool more = --to_issue > 0;              // the last stage is loaded again behind itself (nobody consumes it)
        stream.issue(at + X_LOADS * 1024, more);
        if (more) x_ptr += 128 * S;
    };
#pragma unroll
    for (int i = 0; i < RING - 1; ++i) issue(i);
    int x_at[MR];
#pragma unroll
    for (int a = 0; a < MR; ++a) {
        const int r = a * 16 + l16;
        x_at[a] = (r / (8 * MT)) * REGION + (r % (8 * MT)) * (128 * S);
    }
    const int x_sw = x_swizzle<S>(l16);                // of every one of the lane's rows
    int cur = 0;
    W4Multiplier<UNIT, WHOLE, F16, ZEROS, S, MR> multiplier(p, stream, lane);
    W4Sums<MR> acc;
    // A part has up to 16 superleaves, its halves up to 8; undivided parts are single superleaves (launch_tile_rows).
    constexpr int LEVELS = KG == 2 ? 3 : 0;
    W4Sums<MR> slots[LEVELS > 0 ? LEVELS : 1];
    auto superleaf = [&](W4Sums<MR> &acc) __attribute__((always_inline)) {
        acc.clear();
#pragma nounroll
        for (int s = 0; s < p.stages_per_leaf; ++s) {
            // Own loads of this stage have landed, and behind the barrier everybody's; the slot of the stage before has been read.
            w4_wait_loads_and_barrier<LOADS * (RING - 2)>();
            issue(cur == 0 ? RING - 1 : cur - 1);
            multiplier.prefetch_groups(stream, lane);
            const unsigned char *const st = smem + cur * STAGE;
            const unsigned char *x_rows[MR];
#pragma unroll
            for (int a = 0; a < MR; ++a) x_rows[a] = st + x_at[a];
            multiplier.stage(stream, st + wave * REGION + X_LOADS * 1024, x_rows, x_sw, acc);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            cur = cur + 1 == RING ? 0 : cur + 1;
        }
    };
    W4Walk<LEVELS>::run(superleaf, acc, slots, __builtin_ctz(leaves));
    w4_wait_loads_and_barrier<0>();                    // no load may still be writing LDS; all stages have been read
    if constexpr (KG == 2) {                           // left half + right half, the last level of the tree
        float *const half = reinterpret_cast<float *>(all_smem) + wave * (MT * 1024);
        if (part == 1) {
#pragma unroll
            for (int a = 0; a < MR; ++a)
#pragma unroll
                for (int b = 0; b < 2; ++b) *reinterpret_cast<f32x4 *>(half + ((a * 2 + b) * 64 + lane) * 4) = acc.t[a][b];
        }
        __syncthreads();
        if (part == 1) return;
#pragma unroll
        for (int a = 0; a < MR; ++a)
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const f32x4 right = *reinterpret_cast<const f32x4 *>(half + ((a * 2 + b) * 64 + lane) * 4);
#pragma unroll
                for (int r = 0; r < 4; ++r) acc.t[a][b][r] = acc.t[a][b][r] + right[r];
            }
    }
    if (n0 >= p.N) return;
    const int last = min(p.M - 1 - m0, 32 * MT - 1);
    if (!p.vector_stores || n0 + 32 > p.N) {
#pragma unroll
        for (int a = 0; a < MR; ++a)
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int row = a * 16 + 4 * quarter + r, col = n0 + b * 16 + l16;
                    if (row <= last && col < p.N) w4_store<F16>(p, blockIdx.z, m0 + row, col, acc.t[a][b][r]);
                }
        return;
    }
    // 32 rows at a time through a patch of the wavefront's own, so that a lane holds consecutive columns of one row and stores 16 bytes.
    float *const patch = reinterpret_cast<float *>(all_smem) + wave * (MT * 1024);
#pragma unroll
    for (int a = 0; a < MT; ++a) {
        if (32 * a > last) continue;                   // uniform
#pragma unroll
        for (int q = 0; q < 2; ++q)
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int r = 0; r < 4; ++r) patch[(q * 16 + 4 * quarter + r) * 32 + b * 16 + l16] = acc.t[2 * a + q][b][r];
        if (p.partials || p.y_f32) {
            float *const out = p.partials ? p.partials + blockIdx.z * p.plane + (int64_t)m0 * p.N + n0 : reinterpret_cast<float *>(p.Y) + (int64_t)m0 * p.ldy + n0;
            const int64_t ld = p.partials ? p.N : p.ldy;
#pragma unroll
            for (int it = 0; it < 4; ++it) {
                const int row = it * 8 + lane / 8;
                if (32 * a + row <= last) *reinterpret_cast<f32x4 *>(out + (32 * a + row) * ld + (lane % 8) * 4) = *reinterpret_cast<const f32x4 *>(patch + row * 32 + (lane % 8) * 4);
            }
        } else {
            uint16_t *const out = reinterpret_cast<uint16_t *>(p.Y) + (int64_t)m0 * p.ldy + n0;
#pragma unroll
            for (int it = 0; it < 2; ++it) {
                const int row = it * 16 + lane / 4;
                if (32 * a + row <= last) *reinterpret_cast<tile_u32x4 *>(out + (32 * a + row) * p.ldy + (lane % 4) * 8) = pack_8<F16>(patch + row * 32 + (lane % 4) * 8);
            }
        }
    }
}

// Any legal shape: 32 rows and 32 channels, eight wavefronts along K, operands from memory to registers, two units ahead.
template <int UNIT, bool F16, bool ZEROS>
__global__ __launch_bounds__(64 * W4_WAVES, 2) void gemm_w4_kernel(const W4Params p) {
    constexpr int STEPS = UNIT / 32, DEPTH = UNIT == 128 ? 2 : 4;
    __shared__ float red[W4_WAVES * 1024];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l16 = lane & 15, quarter = lane >> 4;
    const int n0 = blockIdx.x * 32, m0 = blockIdx.y * 32;
    if (wave < p.active_waves) {
        const int first_leaf = blockIdx.z * p.leaves_per_shard + wave * p.leaves_per_wave;
        const int64_t k0 = (int64_t)first_leaf * p.superleaf, g0 = (int64_t)first_leaf * p.groups_per_leaf;
        const uint8_t *w_at[2], *z_at[2];
        const uint16_t *s_at[2], *x_at[2];
#pragma unroll
        for (int b = 0; b < 2; ++b) {                  // rows and channels behind the last one read it once more; they are not stored
            const int channel = min(n0 + b * 16 + l16, p.N - 1);
            w_at[b] = p.W + channel * p.ldw + k0 / 2 + quarter * (UNIT / 8);
            s_at[b] = p.scales + channel * p.lds + g0;
            z_at[b] = ZEROS ? p.zeros + channel * p.ldz + g0 : nullptr;
            x_at[b] = p.X + (int64_t)min(m0 + b * 16 + l16, p.M - 1) * p.ldx + k0 + quarter * (UNIT / 4);
        }
        const int units = p.leaves_per_wave * p.groups_per_leaf * p.units_per_group;
        uint32_t w[DEPTH][2][STEPS];
        uint4 x[DEPTH][2][STEPS];
        auto fetch = [&](int d) __attribute__((always_inline)) {
#pragma unroll
            for (int b = 0; b < 2; ++b) {
#pragma unroll
                for (int i = 0; i < STEPS; ++i) {
                    w[d][b][i] = reinterpret_cast<const uint32_t *>(w_at[b])[i];
                    x[d][b][i] = *reinterpret_cast<const uint4 *>(x_at[b] + 8 * i);
                }
                w_at[b] += UNIT / 2;
                x_at[b] += UNIT;
            }
        };
#pragma unroll
        for (int d = 0; d < DEPTH; ++d)
            if (d < units) fetch(d);
        W4Sums<2> acc, sum;
        W4Stash<2, 2, 4> stash;
        acc.clear();
        sum.clear();
        GroupWalk walk(p.units_per_group);
        int left = p.groups_per_leaf, leaf = 0;
        float scale[2];
        ZeroPoint<F16, ZEROS> zero[2];
        auto group = [&](int g) __attribute__((always_inline)) {
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                scale[b] = widened_16<F16>(s_at[b][g]) * kLevelUnit<F16, ZEROS>;
                if constexpr (ZEROS) zero[b] = ZeroPoint<F16, ZEROS>(z_at[b][g] & 15);
            }
        };
        group(0);
        for (int u0 = 0; u0 < units; u0 += DEPTH) {
#pragma unroll
            for (int d = 0; d < DEPTH; ++d) {
                if (u0 + d >= units) continue;
#pragma unroll
                for (int i = 0; i < STEPS; ++i)
#pragma unroll
                    for (int b = 0; b < 2; ++b) {
                        const bf16x8 v = widened_levels<F16, ZEROS>(w[d][b][i], zero[b]);
#pragma unroll
                        for (int a = 0; a < 2; ++a) sum.t[a][b] = mfma_16x16x32<F16>(__builtin_bit_cast(bf16x8, x[d][a][i]), v, sum.t[a][b]);
                    }
                if (u0 + d + DEPTH < units) fetch(d);
                if (walk.next()) {
#pragma unroll
                    for (int a = 0; a < 2; ++a)
#pragma unroll
                        for (int b = 0; b < 2; ++b)
#pragma unroll
                            for (int r = 0; r < 4; ++r) acc.t[a][b][r] = __builtin_fmaf(scale[b], sum.t[a][b][r], acc.t[a][b][r]);
                    sum.clear();
                    if (u0 + d + 1 < units) group(walk.g);
                    if (--left == 0) {
                        left = p.groups_per_leaf;
                        stash.push(acc, leaf, leaf + 1 < p.leaves_per_wave);
                        ++leaf;
                    }
                }
            }
        }
#pragma unroll
        for (int a = 0; a < 2; ++a)
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int r = 0; r < 4; ++r) red[wave * 1024 + (a * 16 + 4 * quarter + r) * 32 + b * 16 + l16] = acc.t[a][b][r];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 1024 / (64 * W4_WAVES); ++i) {
        const int at = i * 64 * W4_WAVES + threadIdx.x, row = m0 + at / 32, col = n0 + at % 32;
        if (row < p.M && col < p.N) w4_store<F16>(p, blockIdx.z, row, col, tree_of_waves<1024>(red, p.active_waves, at));
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

// The chunks of scales and zero points of a wavefront that walks `leaves` superleaves of `channels`.
void chunks_of(W4Params &p, int channels, int leaves, bool zeros) {
    const int groups = leaves * p.groups_per_leaf, most = std::min(groups, W4_CHUNK), buffers = w4_chunk_buffers(groups);
    p.s_dwords = (2 * most + 5) / 4;                   // the first element may lie 2 bytes into its dword, a zero point 3
    p.z_dwords = (most + 6) / 4;
    p.s_inverse = 65536 / p.s_dwords + 1;
    p.z_inverse = 65536 / p.z_dwords + 1;
    p.group_bytes = buffers * (w4_chunk_bytes(channels, p.s_dwords) + (zeros ? w4_chunk_bytes(channels, p.z_dwords) : 0));
}
constexpr int most_group_bytes(int channels, bool zeros) {
    return 2 * (w4_chunk_bytes(channels, (2 * W4_CHUNK + 5) / 4) + (zeros ? w4_chunk_bytes(channels, (W4_CHUNK + 6) / 4) : 0));
}

template <int UNIT, bool WHOLE, bool F16, bool ZEROS, int S, int NB, int XR, int RING, int LEVELS>
hipError_t launch_slice_of(const W4Params &all, int shards, hipStream_t s) {
    constexpr int row = XR == 1 ? 8192 : 0;
    constexpr int ring = RING * ((XR == 1 ? 0 : XR * S * 128) + W4Stream<ZEROS, S, NB>::BYTES), most = W4_WAVES * (ring + row + most_group_bytes(16 * NB, ZEROS));
    static_assert(most <= 160 * 1024 && ring >= 2048, "LDS of a compute unit; room for the sums");
    W4Params p = all;
    chunks_of(p, 16 * NB, p.leaves_per_wave, ZEROS);
    const int lds = p.active_waves * (ring + (XR == 1 ? p.row_bytes : 0) + p.group_bytes);
    auto k = gemm_w4_slice_kernel<UNIT, WHOLE, F16, ZEROS, S, NB, XR, RING, LEVELS>;
    static std::atomic<unsigned> allowed{0};
    const hipError_t e = allow_lds(k, most, allowed);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(k, dim3((unsigned)((p.N + 16 * NB - 1) / (16 * NB)), (unsigned)((p.M + 15) / 16), (unsigned)shards), dim3(64 * p.active_waves), lds, s, p);
    return hipGetLastError();
}
template <int UNIT, bool WHOLE, bool F16, bool ZEROS, int S, int NB, int XR, int RING>
hipError_t launch_slice(const W4Params &p, int shards, hipStream_t s) {
    return p.leaves_per_wave <= 2 ? launch_slice_of<UNIT, WHOLE, F16, ZEROS, S, NB, XR, RING, 1>(p, shards, s) : launch_slice_of<UNIT, WHOLE, F16, ZEROS, S, NB, XR, RING, 4>(p, shards, s);
}
template <int UNIT, bool WHOLE, bool F16, bool ZEROS, int S, int MT, int RING, int KG = 1>
hipError_t launch_tile(const W4Params &all, int shards, hipStream_t s) {
    constexpr int rings = KG * RING * 4 * (MT * S * 1024 + W4Stream<ZEROS, S>::BYTES), most = rings + 4 * KG * most_group_bytes(32, ZEROS);
    static_assert(most <= 160 * 1024 && rings >= 4 * MT * 4096, "LDS of a compute unit; room for the sums and the patches");
    W4Params p = all;
    chunks_of(p, 32, p.leaves_per_shard / KG, ZEROS);
    const int lds = rings + 4 * KG * p.group_bytes;
    auto k = gemm_w4_tiled_kernel<UNIT, WHOLE, F16, ZEROS, S, MT, RING, KG>;
    static std::atomic<unsigned> allowed{0};
    const hipError_t e = allow_lds(k, most, allowed);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(k, dim3((unsigned)((p.N + 127) / 128), (unsigned)((p.M + 32 * MT - 1) / (32 * MT)), (unsigned)shards), dim3(256 * KG), lds, s, p);
    return hipGetLastError();
}

// Stages in flight: three while every workgroup has a compute unit to itself; with more workgroups than compute units two, which lets
// more of them share one (16 rows are too large for that either way).  16 channels a slice where 32 leave half of the compute units idle (8 rows, K 12288 x
// N 4096 13.7 -> 9.8 us, 16 rows 15.2 -> 12.0), for one row, and where there are so many that three workgroups share a compute unit (8 rows, K 4096 x N 12288
// 10.2 -> 9.5; with 16 rows, where two do not fit, 12.9 would become 14.4; of 160 slices, 5120 x 5120, 8.1 either way with 8 rows and 8.1 -> 11 with 16).
template <int UNIT, bool WHOLE, bool F16, bool ZEROS, int S>
hipError_t launch_row(const W4Params &p, int shards, hipStream_t s) {
    if (((int64_t)p.N + 15) / 16 * shards <= 256) return launch_slice<UNIT, WHOLE, F16, ZEROS, S, 1, 1, 3>(p, shards, s);
    return launch_slice<UNIT, WHOLE, F16, ZEROS, S, 1, 1, 2>(p, shards, s);
}
template <int UNIT, bool WHOLE, bool F16, bool ZEROS, int S>
hipError_t launch_slice_rows(const W4Params &all, int shards, hipStream_t s) {
    W4Params p = all;
    p.row_bytes = (p.leaves_per_wave * p.superleaf * 2 + 1023) & ~1023;
    if constexpr (S == 2) {
        if (p.M == 1 && p.row_bytes <= 8192) {
            if (p.superleaf % 256 != 0) return launch_row<UNIT, WHOLE, F16, ZEROS, 2>(p, shards, s);
            p.stages_per_leaf = p.superleaf / 256;
            return launch_row<UNIT, WHOLE, F16, ZEROS, 4>(p, shards, s);
        }
    }
    if constexpr (S == 1) return p.M > 8 ? launch_slice<UNIT, WHOLE, F16, ZEROS, 1, 2, 16, 4>(p, shards, s) : launch_slice<UNIT, WHOLE, F16, ZEROS, 1, 2, 8, 6>(p, shards, s);
    else {
        const int64_t slices = ((int64_t)p.N + 31) / 32 * shards;
        if (slices <= 128) return p.M > 8 ? launch_slice<UNIT, WHOLE, F16, ZEROS, S, 1, 16, 3>(p, shards, s) : launch_slice<UNIT, WHOLE, F16, ZEROS, S, 1, 8, 3>(p, shards, s);
        if (p.M > 8) return launch_slice<UNIT, WHOLE, F16, ZEROS, S, 2, 16, 2>(p, shards, s);
        if (slices <= 256) return launch_slice<UNIT, WHOLE, F16, ZEROS, S, 2, 8, 3>(p, shards, s);
        return launch_slice<UNIT, WHOLE, F16, ZEROS, S, 1, 8, 2>(p, shards, s);
    }
}
template <int UNIT, bool WHOLE, bool F16, bool ZEROS, int S>
hipError_t launch_tile_rows(const W4Params &p, int shards, hipStream_t s) {
    const bool halves = p.leaves_per_shard % 2 == 0;   // a power of two: or one
    if (w4_tile_rows(p.M) == 32) return halves ? launch_tile<UNIT, WHOLE, F16, ZEROS, S, 1, S == 1 ? 6 : 3, 2>(p, shards, s) : launch_tile<UNIT, WHOLE, F16, ZEROS, S, 1, S == 1 ? 6 : 4>(p, shards, s);
    return halves ? launch_tile<UNIT, WHOLE, F16, ZEROS, S, 2, S == 1 ? 4 : 2, 2>(p, shards, s) : launch_tile<UNIT, WHOLE, F16, ZEROS, S, 2, S == 1 ? 5 : 3>(p, shards, s);
}
template <int UNIT, bool WHOLE, bool F16, bool ZEROS>
hipError_t launch_unit(const W4Args &a, const W4Params &all, hipStream_t s) {
    W4Params p = all;
    const int ns = a.ns / a.P, kernel = w4_kernel(a);  // ns: superleaves of a shard
    const bool two = UNIT == 128 || a.superleaf % 128 == 0;
    p.units_per_group = a.group / UNIT;
    p.stages_per_leaf = a.superleaf / (two ? 128 : 64);
    p.leaves_per_wave = ns > W4_WAVES ? ns / W4_WAVES : 1;
    p.active_waves = ns > W4_WAVES ? W4_WAVES : ns;
    if constexpr (UNIT < 128) {
        if (kernel == W4_SLICES && !two) return launch_slice_rows<UNIT, WHOLE, F16, ZEROS, 1>(p, a.P, s);
        if (kernel == W4_TILES && !two) return launch_tile_rows<UNIT, WHOLE, F16, ZEROS, 1>(p, a.P, s);
    }
    if (kernel == W4_SLICES) return launch_slice_rows<UNIT, WHOLE, F16, ZEROS, 2>(p, a.P, s);
    if (kernel == W4_TILES) return launch_tile_rows<UNIT, WHOLE, F16, ZEROS, 2>(p, a.P, s);
    for (int64_t m0 = 0; m0 < a.M; m0 += 32 * 4096) {  // 4096 row tiles a launch
        W4Params q = p;
        q.M = (int)(a.M - m0 < 32 * 4096 ? a.M - m0 : 32 * 4096);
        q.X += m0 * a.ldx;
        if (q.partials) q.partials += m0 * a.N;
        else q.Y = static_cast<char *>(q.Y) + m0 * a.ldy * (p.y_f32 ? 4 : 2);
        hipLaunchKernelGGL((gemm_w4_kernel<UNIT, F16, ZEROS>), dim3((unsigned)((a.N + 31) / 32), (unsigned)((q.M + 31) / 32), (unsigned)a.P), dim3(64 * W4_WAVES), 0, s, q);
    }
    return hipGetLastError();
}

template <int UNIT, bool WHOLE, bool F16>
hipError_t launch_zeros(const W4Args &a, const W4Params &p, hipStream_t s) {
    return a.zeros ? launch_unit<UNIT, WHOLE, F16, true>(a, p, s) : launch_unit<UNIT, WHOLE, F16, false>(a, p, s);
}

}  // namespace

#ifdef TBIK_W4_F16_UNIT
hipError_t launch_gemm_w4_f16(const W4Args &a, const W4Params &p, hipStream_t s) {
#else
// Slices up to 16 rows and where there are no more than W4_FEW_TILES tiles, tiles beyond; `a.P`: shards, or the parts of a split K.  The general kernel takes what the
// rings' 32-bit offsets and stages of 64 k do not reach, and tiles of more than 16 superleaves: the product splits K where the workspace has room, but shards'
// sums do not (2048 rows, K 8192 x N 4096, one shard of 32 superleaves 781 us, of 16 186).
int w4_kernel(const W4Args &a) {
    const int ns = a.ns / a.P;
    const bool ring = a.superleaf % 64 == 0 && a.ldx < (1 << 22) && a.ldw < (1 << 22) && a.lds < (1 << 22) && a.ldz < (1 << 22);      // 32-bit lane offsets
    if (!ring) return W4_GENERAL;
    if (a.M <= 16 || w4_tiles(a.M, a.N) * a.P <= W4_FEW_TILES) return W4_SLICES;
    return ns <= 16 && (int64_t)a.M <= 32 * 65535 ? W4_TILES : W4_GENERAL;
}

hipError_t launch_gemm_w4_f16(const W4Args &a, const W4Params &p, hipStream_t s);

hipError_t launch_gemm_w4(const W4Args &a, hipStream_t s) {
    if (a.M <= 0 || a.N <= 0) return hipSuccess;
    W4Params p{};
    p.X = a.X; p.W = reinterpret_cast<const uint8_t *>(a.W); p.scales = a.scales; p.zeros = a.zeros;
    p.partials = a.partials; p.Y = a.Y;
    p.ldx = a.ldx; p.ldw = a.ldw; p.lds = a.lds; p.ldz = a.ldz; p.ldy = a.ldy;
    p.M = a.M; p.N = a.N;
    p.plane = (int64_t)a.M * a.N;
    p.y_f32 = a.y_dtype == TBIK_F32;
    p.superleaf = a.superleaf; p.groups_per_leaf = a.superleaf / a.group;
    p.leaves_per_shard = a.ns / a.P;
    const void *out = a.partials ? (const void *)a.partials : a.Y;
    const int64_t ld_bytes = a.partials ? (int64_t)a.N * 4 : a.ldy * (p.y_f32 ? 4 : 2);
    p.vector_stores = (reinterpret_cast<uintptr_t>(out) & 15) == 0 && ld_bytes % 16 == 0;
    if (a.x_dtype == TBIK_F16) return launch_gemm_w4_f16(a, p, s);
#endif
    if (a.group == 128) return launch_zeros<128, true, TBIK_W4_F16>(a, p, s);
    if (a.group == 64) return launch_zeros<64, true, TBIK_W4_F16>(a, p, s);
    if (a.group == 32) return launch_zeros<32, true, TBIK_W4_F16>(a, p, s);
    if (a.group % 128 == 0) return launch_zeros<128, false, TBIK_W4_F16>(a, p, s);
    return launch_zeros<32, false, TBIK_W4_F16>(a, p, s);
}

}  // namespace tbik
