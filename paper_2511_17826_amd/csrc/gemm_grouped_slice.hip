// Products grouped by expert for groups of few rows (16-bit operands): a workgroup takes a slice of 64 columns of one group's weight, up to
// 32 of its rows and all of a shard's K, in one launch and without a workspace.
//
// What bounds it is the weights' stream: every touched expert's weight is read once (once per 32 rows).  The tiled kernels give a wavefront a
// column block and all of K, so a workgroup's stream is as long as K and few groups leave compute units idle; here the wavefronts
// take consecutive superleaves each (whole superleaves, in order: Sec. 4.2, App. D.1), each streams its own part of the slice and of the
// rows through a ring of steps in LDS of its own (direct global->LDS loads of whole 128-byte lines, no barrier until the
// sums are there), and the upper levels of the tree run over the wavefronts' sums in LDS (App. C).  The matrix instruction and the k that it takes are
// those of the tiled kernels, so the bits are.  With the activation a slice is 32 gate columns and the same 32 up columns.
#include <atomic>
#include <type_traits>

#include "grouped.hpp"

namespace tbik {

namespace {

template <int V>
using Int = std::integral_constant<int, V>;

typedef short slice_v4i16 __attribute__((ext_vector_type(4)));

constexpr int STEP_K = 32;
constexpr int SLICE_COLUMNS = 64, SLICE_ROWS = 32;
constexpr int X_BYTES = SLICE_ROWS * STEP_K * 2, W_BYTES = STEP_K * SLICE_COLUMNS * 2, STEP_BYTES = X_BYTES + W_BYTES;      // a step in LDS: rows of X, then of W
constexpr int STEP_LOADS = STEP_BYTES / 1024;
constexpr int RED_FLOATS = SLICE_ROWS * SLICE_COLUMNS;                 // a wavefront's sums

struct SliceParams {
    const uint16_t *X, *W;
    const int32_t *offsets, *rows;
    float *partials;
    void *Y;
    int64_t ldx, ldw, ldy, weight_stride;
    int M, N, tokens, groups;
    int columns;                        // of the output: N, or N / 2 with the activation
    int slices;
    int y_f32, swiglu;
    int steps_per_leaf, leaves_per_wave, active_waves;
    int64_t k_per_shard;
    int vector_stores;                  // four columns of the output at a time
};

template <int N>
__device__ __forceinline__ void wait_loads() {
    static_assert(N >= 0 && N < 64, "vmcnt range");
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
// The last steps of a wavefront's stream: REST more are in flight behind the one that is waited for.
template <int REST, class Consume>
__device__ __forceinline__ void last_steps(int steps, Consume &consume) {
    if (steps > REST) consume(Int<REST>{}, std::false_type{});
    if constexpr (REST > 0) last_steps<REST - 1>(steps, consume);
}

template <int WAVES, int RING, bool F16>
__global__ __launch_bounds__(64 * WAVES, 2) void gemm_grouped_slice_kernel(const SliceParams p) {
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int li = lane & 31, lg = lane >> 5;
    GroupMap<SLICE_ROWS> map;
    map.read(p.offsets, p.groups, p.M, lane);
    // With the activation a slice takes half a cache line of gate columns and half of one of up columns: two neighbours, which read the same lines, run on one
    // XCD (workgroups go to the eight in turn), or each fetches them for itself.
    int block = blockIdx.x;
    if (p.swiglu && (block | 15) < (int)gridDim.x) block = (block & ~15) + (block & 7) * 2 + ((block >> 3) & 1);
    const int tile = block / p.slices;
    if (tile >= map.tiles) return;                                     // the grid is for any division of the rows
    const GroupRows at = map.at(tile);
    const int tile_rows = min(at.end - at.first, SLICE_ROWS);
    const int c0 = (block % p.slices) * (p.swiglu ? SLICE_COLUMNS / 2 : SLICE_COLUMNS);      // first column of the output
    const int64_t kbase = blockIdx.y * p.k_per_shard;

    f32x16 acc[2];
    if (wave < p.active_waves) {
        const int steps = p.leaves_per_wave * p.steps_per_leaf;
        const int64_t k0 = kbase + (int64_t)wave * steps * STEP_K;
        // Load j of a step brings 64 chunks of 16 bytes in LDS order; rows behind the tile's last re-read that one, columns behind N the last eight.
        // The instruction offset moves the LDS and the global address alike, hence the lane bias.
        const uint16_t *first_row = p.rows ? p.X : p.X + (int64_t)at.first * p.ldx;
        const char *x_ptr = uniform_pointer(reinterpret_cast<const char *>(first_row + k0));
        const char *w_ptr = uniform_pointer(reinterpret_cast<const char *>(p.W + at.group * p.weight_stride + k0 * p.ldw + c0) - 4096);
        const int64_t w_step = (int64_t)STEP_K * p.ldw * 2;
        unsigned xoff[2], woff[4];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int r = 16 * j + (lane >> 2), c = (lane & 3) ^ ((r >> 2) & 3);
            int row = min(r, tile_rows - 1);
            if (p.rows) row = source_row(p.rows, at.first + row, p.tokens);
            xoff[j] = (unsigned)(row * (int)p.ldx + c * 8) * 2u + (unsigned)((2 - j) * 1024);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int kk = 8 * j + (lane >> 3), c = (lane & 7) ^ (kk & 2);
            const int col = p.swiglu ? (c >> 2) * p.columns + min((c & 3) * 8, p.columns - 8 - c0) : min(c * 8, p.N - 8 - c0);
            woff[j] = (unsigned)(kk * (int)p.ldw + col) * 2u + (unsigned)(4096 - j * 1024);
        }
        const unsigned ring = (unsigned)(uintptr_t)(__attribute__((address_space(3))) unsigned char *)smem + wave * RING * STEP_BYTES;
        auto issue = [&](int slot) __attribute__((always_inline)) {
            const unsigned m0v = ring + slot * STEP_BYTES + X_BYTES;
            load_16B_per_lane_to_lds<0, true>(w_ptr, woff[0], m0v);
            load_16B_per_lane_to_lds<1024, false>(w_ptr, woff[1], m0v);
            load_16B_per_lane_to_lds<2048, false>(w_ptr, woff[2], m0v);
            load_16B_per_lane_to_lds<3 * 1024, false>(w_ptr, woff[3], m0v);
            load_16B_per_lane_to_lds<-2048, false>(x_ptr, xoff[0], m0v);
            load_16B_per_lane_to_lds<-1024, false>(x_ptr, xoff[1], m0v);
            x_ptr += STEP_K * 2;
            w_ptr += w_step;
        };
        // A lane's fragments (see gemm_tiled.hip): row li of X, chunk 2 ks + lg; of W eight consecutive k of a column as two transposed halves.
        // Chunk c of row r of X lies at c ^ (r / 4 % 4), chunk c of row k of W at c ^ (k & 2), so that the rows of a read meet different banks.
        const int x_at = li * (STEP_K * 2), x_sw = (li >> 2) & 3;
        const int l16 = lane & 15, e = l16 >> 2;
        int w_at[2];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            const int col = b * 32 + ((lane >> 4) & 1) * 16 + (l16 & 3) * 4;
            w_at[b] = X_BYTES + (lg * 8 + e) * (SLICE_COLUMNS * 2) + (((col >> 3) ^ (e & 2)) << 4) + ((col >> 2) & 1) * 8;
        }
        const unsigned char *const ring_rd = smem + wave * RING * STEP_BYTES;
        f32x16 stash0[4], stash1[4];                                   // finished subtrees of the two column blocks
        int left = p.steps_per_leaf, leaf = 0, slot = 0;
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[b][r] = 0.0f;

        auto consume = [&](auto rest, auto again) __attribute__((always_inline)) {
            wait_loads<decltype(rest)::value * STEP_LOADS>();
            const unsigned char *const s = ring_rd + slot * STEP_BYTES;
            bf16x8 x[2];
            union Fragment {
                slice_v4i16 h[2];
                bf16x8 v;
            } w[2][2];
#pragma unroll
            for (int ks = 0; ks < 2; ++ks) {
                x[ks] = *reinterpret_cast<const bf16x8 *>(s + x_at + (((2 * ks + lg) ^ x_sw) << 4));
#pragma unroll
                for (int b = 0; b < 2; ++b)
#pragma unroll
                    for (int h = 0; h < 2; ++h)
                        w[ks][b].h[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                            (__attribute__((address_space(3))) slice_v4i16 *)(s + w_at[b] + (16 * ks + 4 * h) * (SLICE_COLUMNS * 2)));
            }
            if constexpr (decltype(again)::value) {                    // the step's bytes are in registers before its slot is filled again
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                issue(slot);
            }
#pragma unroll
            for (int ks = 0; ks < 2; ++ks)
#pragma unroll
                for (int b = 0; b < 2; ++b) acc[b] = mfma_32x32x16<F16>(x[ks], w[ks][b].v, acc[b]);
            slot = slot + 1 == RING ? 0 : slot + 1;
            if (--left == 0) {                                         // a superleaf ends: the carry-over step of the tree
                const int t = __builtin_ctz(~leaf);
#pragma unroll
                for (int l = 0; l < 4; ++l)
                    if (l < t) {
#pragma unroll
                        for (int r = 0; r < 16; ++r) acc[0][r] = stash0[l][r] + acc[0][r];
#pragma unroll
                        for (int r = 0; r < 16; ++r) acc[1][r] = stash1[l][r] + acc[1][r];
                    }
                left = p.steps_per_leaf;
                if (++leaf < p.leaves_per_wave) {
#pragma unroll
                    for (int l = 0; l < 4; ++l)
                        if (l == t) stash0[l] = acc[0];
#pragma unroll
                    for (int l = 0; l < 4; ++l)
                        if (l == t) stash1[l] = acc[1];
#pragma unroll
                    for (int b = 0; b < 2; ++b)
#pragma unroll
                        for (int r = 0; r < 16; ++r) acc[b][r] = 0.0f;
                }
            }
        };
#pragma unroll
        for (int i = 0; i < RING; ++i)
            if (i < steps) issue(i);
        for (int s = RING; s < steps; ++s) consume(Int<RING - 1>{}, std::true_type{});
        last_steps<RING - 1>(steps, consume);
    }
    __syncthreads();                                                   // the rings have been read: the sums take their place
    float *const red = reinterpret_cast<float *>(smem);
    if (wave < p.active_waves) {
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) red[wave * RED_FLOATS + (8 * (r >> 2) + 4 * lg + (r & 3)) * SLICE_COLUMNS + b * 32 + li] = acc[b][r];
    }
    __syncthreads();
    // T over the wavefronts' sums of four consecutive columns.
    auto sum_at = [&](int where) __attribute__((always_inline)) {
        f32x4 v[WAVES];
#pragma unroll
        for (int w = 0; w < WAVES; ++w) v[w] = *reinterpret_cast<const f32x4 *>(red + (w < p.active_waves ? w * RED_FLOATS : 0) + where);
#pragma unroll
        for (int s = 1; s < WAVES; s *= 2)
#pragma unroll
            for (int r = 0; r < WAVES; r += 2 * s)
                if (r + s < p.active_waves) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) v[r][i] = v[r][i] + v[r + s][i];
                }
        return v[0];
    };
    const int quads = p.swiglu ? SLICE_COLUMNS / 8 : SLICE_COLUMNS / 4;         // of a row of the slice
    for (int q = threadIdx.x; q < SLICE_ROWS * quads; q += 64 * WAVES) {
        const int r = q / quads, c = (q % quads) * 4, col = c0 + c;
        if (r >= tile_rows || col >= p.columns) continue;
        f32x4 v = sum_at(r * SLICE_COLUMNS + c);
        if (p.swiglu) {
            const f32x4 up = sum_at(r * SLICE_COLUMNS + SLICE_COLUMNS / 2 + c);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = silu_mul(through_16_bits<F16>(v[i]), through_16_bits<F16>(up[i]));
        }
        const int64_t row = at.first + r;
        if (p.partials || p.y_f32) {
            float *dst = p.partials ? p.partials + ((int64_t)blockIdx.y * p.M + row) * p.N + col : reinterpret_cast<float *>(p.Y) + row * p.ldy + col;
            if (p.vector_stores && col + 4 <= p.columns) *reinterpret_cast<f32x4 *>(dst) = v;
            else
                for (int i = 0; i < 4 && col + i < p.columns; ++i) dst[i] = v[i];
        } else {
            uint16_t *dst = reinterpret_cast<uint16_t *>(p.Y) + row * p.ldy + col;
            const uint32_t lo = pack_16x2<F16>(v[0], v[1]), hi = pack_16x2<F16>(v[2], v[3]);
            if (p.vector_stores && col + 4 <= p.columns) *reinterpret_cast<uint2 *>(dst) = make_uint2(lo, hi);
            else
                for (int i = 0; i < 4 && col + i < p.columns; ++i) dst[i] = (uint16_t)((i < 2 ? lo : hi) >> (16 * (i & 1)));
        }
    }
}

template <int WAVES, int RING, bool F16>
hipError_t launch_slices(const GroupedArgs &a, const SliceParams &p, unsigned blocks, hipStream_t s) {
    constexpr int lds = WAVES * RING * STEP_BYTES;
    static_assert(lds <= 160 * 1024 && RING * STEP_BYTES >= RED_FLOATS * 4, "LDS of a compute unit; room for the sums");
    auto k = gemm_grouped_slice_kernel<WAVES, RING, F16>;
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 32) dev = 32;      // 32: not remembered, set every time
    static std::atomic<unsigned> lds_allowed{0};                                 // bit d: the attribute is set on device d
    if (dev >= 32 || !((lds_allowed.load(std::memory_order_relaxed) >> dev) & 1u)) {
        hipError_t e = hipFuncSetAttribute((const void *)k, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
        if (e != hipSuccess) return e;
        if (dev < 32) lds_allowed.fetch_or(1u << dev, std::memory_order_relaxed);
    }
    hipLaunchKernelGGL(k, dim3(blocks, (unsigned)a.P), dim3(64 * WAVES), lds, s, p);
    return hipGetLastError();
}

inline int slices_of(const GroupedArgs &a) { return a.swiglu ? (a.N / 2 + 31) / 32 : (a.N + 63) / 64; }

}  // namespace

bool gemm_grouped_slice_supports(const GroupedArgs &a) {
    if (a.N % 8 != 0 || (a.swiglu && a.N % 16 != 0) || a.superleaf % STEP_K != 0) return false;
    if (a.ns / a.P > 16 * 4) return false;                                       // four levels per wavefront
    if (a.ldx >= (1 << 22) || a.ldw >= (1 << 22)) return false;                  // 32-bit lane offsets
    if (a.rows && (int64_t)a.tokens * a.ldx * 2 > 0xffffffffll - 8192) return false;      // gathered rows: unsigned ones from the first row of X
    return slices_of(a) * grouped_tiles(a, SLICE_ROWS) < (1 << 23);              // a grid has fewer than 2^32 threads
}

hipError_t launch_gemm_grouped_slice(const GroupedArgs &a, hipStream_t s) {
    if (a.M <= 0 || a.N <= 0) return hipSuccess;
    if (!gemm_grouped_slice_supports(a)) return hipErrorInvalidValue;
    const int ns = a.ns / a.P;
    const int64_t blocks = slices_of(a) * grouped_tiles(a, SLICE_ROWS);
    // While there are no more workgroups than compute units, one has all of LDS: eight wavefronts along K, or with few superleaves four and a ring twice as deep;
    // else four, two workgroups to a compute unit.
    const bool alone = blocks * a.P <= 256;
    const int waves = alone && ns > 4 ? 8 : 4;
    SliceParams p;
    p.X = a.X; p.W = a.W; p.offsets = a.offsets; p.rows = a.rows;
    p.partials = a.partials; p.Y = a.Y;
    p.ldx = a.ldx; p.ldw = a.ldw; p.ldy = a.ldy; p.weight_stride = a.weight_stride;
    p.M = a.M; p.N = a.N; p.tokens = a.tokens; p.groups = a.groups;
    p.columns = a.swiglu ? a.N / 2 : a.N;
    p.slices = slices_of(a);
    p.y_f32 = a.y_dtype == TBIK_F32;
    p.swiglu = a.swiglu;
    p.steps_per_leaf = a.superleaf / STEP_K;
    p.leaves_per_wave = ns > waves ? ns / waves : 1;
    p.active_waves = ns > waves ? waves : ns;
    p.k_per_shard = (int64_t)a.K / a.P;
    const void *out = a.partials ? (const void *)a.partials : a.Y;
    const int64_t ld = a.partials ? a.N : a.ldy;
    const int bytes = a.partials || p.y_f32 ? 16 : 8;                            // of four columns
    p.vector_stores = (reinterpret_cast<uintptr_t>(out) & (bytes - 1)) == 0 && ld % 4 == 0;
    if (waves == 8) return a.x_dtype == TBIK_F16 ? launch_slices<8, 3, true>(a, p, (unsigned)blocks, s) : launch_slices<8, 3, false>(a, p, (unsigned)blocks, s);
    if (alone) return a.x_dtype == TBIK_F16 ? launch_slices<4, 6, true>(a, p, (unsigned)blocks, s) : launch_slices<4, 6, false>(a, p, (unsigned)blocks, s);
    return a.x_dtype == TBIK_F16 ? launch_slices<4, 3, true>(a, p, (unsigned)blocks, s) : launch_slices<4, 3, false>(a, p, (unsigned)blocks, s);
}

}  // namespace tbik
