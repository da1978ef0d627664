// The router of a mixture of experts: the k largest logits of each token, their weights, and the order in which products grouped
// by expert take the tokens.
//
// A token is one wavefront's work whatever the batch: each lane holds every 64th logit as a key that orders like it (NaN lowest), and
// k times the largest key is found with the row's data-parallel moves and the lowest index among its owners with ballots.  The
// order needs no sort: a token chooses an expert at most once, so a block of 64 tokens is one 64-bit mask per expert, and a
// choice's place is the expert's first row + what earlier blocks have + the bits below the token's in the mask.  Masks are
// joined with integer "or", counts are sums of integers: nothing depends on the order in which wavefronts run.
//
// Bound by launches and latency: 8191 tokens of 128 experts read 2 MB.  Up to 64 tokens are one workgroup and one launch; more are
// two launches, a block of 64 tokens each (select), then every block adds up the blocks' counts (a byte per expert and block) for itself (place).
#include "tbik_device.hpp"
#include "tbik_internal.hpp"

namespace tbik {

namespace {

constexpr int ROUTE_TOKENS = 64;           // of a block: bits of a mask
constexpr int ROUTE_WAVES = 16;

// Orders like the float; NaN below everything else, the two zeros equal.  0 is no float's key: a logit that has been chosen, or a lane
// without one.
__device__ __forceinline__ uint32_t key_of(float v) {
    const uint32_t b = __float_as_uint(v + 0.0f);
    if (v != v) return 1u;
    return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float logit_of(uint32_t key) {
    if (key <= 1u) return __uint_as_float(0x7fc00000u);
    return __uint_as_float((key & 0x80000000u) ? key & 0x7fffffffu : ~key);
}

template <int CTRL>
__device__ __forceinline__ uint32_t from_lane_in_row_u32(uint32_t v) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, false);
}
__device__ __forceinline__ uint32_t wave_max_u32(uint32_t v) {
    v = max(v, from_lane_in_row_u32<0xB1>(v));
    v = max(v, from_lane_in_row_u32<0x4E>(v));
    v = max(v, from_lane_in_row_u32<0x141>(v));
    v = max(v, from_lane_in_row_u32<0x140>(v));
    const uint32_t r0 = __builtin_amdgcn_readlane(v, 0), r1 = __builtin_amdgcn_readlane(v, 16), r2 = __builtin_amdgcn_readlane(v, 32), r3 = __builtin_amdgcn_readlane(v, 48);
    return max(max(r0, r1), max(r2, r3));
}

struct RouteParams {
    const void *logits;                    // [T, ldl]
    int64_t ldl;
    int dtype, T, E, k, renormalize;
    int32_t *experts;                      // [T, k]
    float *weights;                        // [T, k]
    int32_t *offsets;                      // [E + 1]
    int32_t *rows;                         // [T k]
    int32_t *slots;                        // [T, k]
    uint64_t *masks;                       // [blocks, E]
    uint8_t *counts;                       // [blocks, pitch]
    int pitch, blocks;
};

__device__ __forceinline__ float logit_at(const RouteParams &p, int64_t i) {
    if (p.dtype == TBIK_F32) return reinterpret_cast<const float *>(p.logits)[i];
    const uint16_t h = reinterpret_cast<const uint16_t *>(p.logits)[i];
    return p.dtype == TBIK_F16 ? (float)__builtin_bit_cast(_Float16, h) : bf16_bits_to_f32(h);
}

// A token's choices: lane j (j < k) gets expert and weight of choice j.  The weights: e^(l_j - l_0) over the sum of the chosen, ascending j, or
// over the sum of all experts (lane-wise chains in ascending expert order, then the tree over the lanes).
template <int PER_LANE>
__device__ __forceinline__ void choose(const RouteParams &p, int t, int lane, int *expert, float *weight) {
    uint32_t key[PER_LANE];
#pragma unroll
    for (int j = 0; j < PER_LANE; ++j) {
        const int e = j * 64 + lane;
        key[j] = e < p.E ? key_of(logit_at(p, (int64_t)t * p.ldl + e)) : 0u;
    }
    float all = 0.0f;
    uint32_t first = 0, mine = 0;
    int chosen = 0;
    for (int i = 0; i < p.k; ++i) {
        uint32_t best = key[0];
#pragma unroll
        for (int j = 1; j < PER_LANE; ++j) best = max(best, key[j]);
        best = wave_max_u32(best);
        if (i == 0) {
            first = best;
            if (!p.renormalize) {
#pragma unroll
                for (int j = 0; j < PER_LANE; ++j)
                    if (j * 64 + lane < p.E) all = all + expf(logit_of(key[j]) - logit_of(first));
                all = wave_tree_sum(all);
            }
        }
        int winner = -1;
#pragma unroll
        for (int j = 0; j < PER_LANE; ++j) {
            const uint64_t owners = __builtin_amdgcn_ballot_w64(key[j] == best);
            if (winner < 0 && owners) {
                const int at = __builtin_ctzll(owners);
                winner = j * 64 + at;
                if (lane == at) key[j] = 0u;
            }
        }
        if (lane == i) {
            mine = best;
            chosen = winner;
        }
    }
    const float top = logit_of(first);
    const float e = lane < p.k ? expf(logit_of(mine) - top) : 0.0f;
    float sum = all;
    if (p.renormalize) {
        sum = 0.0f;
        for (int i = 0; i < p.k; ++i) sum = sum + __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, e), i));
    }
    *weight = top == -__builtin_inff() ? 0.0f : e / sum;       // nothing to choose from: no weight
    *expert = chosen;
}

// ALONE: one block is the whole batch, and places its choices itself.
template <int PER_LANE, bool ALONE>
__global__ __launch_bounds__(64 * ROUTE_WAVES) void route_select_kernel(const RouteParams p) {
    __shared__ uint64_t mask[PER_LANE * 64];
    __shared__ int32_t first_row[ALONE ? PER_LANE * 64 : 1];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int t0 = blockIdx.x * ROUTE_TOKENS;
    const int tokens = min(ROUTE_TOKENS, p.T - t0);
    for (int e = threadIdx.x; e < PER_LANE * 64; e += 64 * ROUTE_WAVES) mask[e] = 0;
    __syncthreads();
    for (int i = wave; i < tokens; i += ROUTE_WAVES) {
        int expert;
        float weight;
        choose<PER_LANE>(p, t0 + i, lane, &expert, &weight);
        if (lane < p.k) {
            const int64_t at = (int64_t)(t0 + i) * p.k + lane;
            p.experts[at] = expert;
            p.weights[at] = weight;
            atomicOr(reinterpret_cast<unsigned long long *>(&mask[expert]), 1ull << i);
        }
    }
    __syncthreads();
    if constexpr (!ALONE) {
        for (int e = threadIdx.x; e < p.pitch; e += 64 * ROUTE_WAVES) {
            const uint64_t m = e < p.E ? mask[e] : 0;
            if (e < p.E) p.masks[(int64_t)blockIdx.x * p.E + e] = m;
            p.counts[(int64_t)blockIdx.x * p.pitch + e] = (uint8_t)__popcll(m);
        }
    } else {
        if (wave == 0) {                               // first rows: a scan over the experts
            int before = 0;
#pragma unroll
            for (int j = 0; j < PER_LANE; ++j) {
                const int e = j * 64 + lane, n = __popcll(mask[e]);
                int sum = n;
#pragma unroll
                for (int d = 1; d < 64; d *= 2) {
                    const int up = __shfl_up(sum, d);
                    if (lane >= d) sum += up;
                }
                first_row[e] = before + sum - n;
                if (e <= p.E) p.offsets[e] = before + sum - n;
                before += __builtin_amdgcn_readlane(sum, 63);
            }
            if (p.E == PER_LANE * 64 && lane == 0) p.offsets[p.E] = before;
        }
        __syncthreads();
        for (int c = threadIdx.x; c < tokens * p.k; c += 64 * ROUTE_WAVES) {
            const int i = c / p.k, e = p.experts[c];
            const int row = first_row[e] + __popcll(mask[e] & ((1ull << i) - 1));
            p.rows[row] = i;
            p.slots[c] = row;
        }
    }
}

constexpr int PLACE_THREADS = 512;

__global__ __launch_bounds__(PLACE_THREADS) void route_place_kernel(const RouteParams p) {
    extern __shared__ int32_t sums[];                  // [pitch] choices of all blocks, then [pitch] of the blocks before this one
    int32_t *const total = sums, *const before = sums + p.pitch;
    for (int e = threadIdx.x; e < 2 * p.pitch; e += PLACE_THREADS) sums[e] = 0;
    __syncthreads();
    // A thread adds up 16 experts' counts of every `step`-th block.
    const int chunks = p.pitch / 16, step = PLACE_THREADS / chunks;
    if ((int)threadIdx.x < step * chunks) {
        const int c = threadIdx.x % chunks, b0 = threadIdx.x / chunks;
        int all[16] = {}, early[16] = {};
        for (int b = b0; b < p.blocks; b += step) {
            const uint4 v = *reinterpret_cast<const uint4 *>(p.counts + (int64_t)b * p.pitch + c * 16);
            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int n = (w[i >> 2] >> (8 * (i & 3))) & 0xff;
                all[i] += n;
                early[i] += b < (int)blockIdx.x ? n : 0;
            }
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            if (all[i]) atomicAdd(&total[c * 16 + i], all[i]);
            if (early[i]) atomicAdd(&before[c * 16 + i], early[i]);
        }
    }
    __syncthreads();
    if (threadIdx.x < 64) {                            // first rows: a scan over the experts
        int ahead = 0;
        for (int e = threadIdx.x; e - (int)threadIdx.x < p.pitch; e += 64) {
            const int n = e < p.pitch ? total[e] : 0;
            int sum = n;
#pragma unroll
            for (int d = 1; d < 64; d *= 2) {
                const int up = __shfl_up(sum, d);
                if ((int)threadIdx.x >= d) sum += up;
            }
            if (blockIdx.x == 0 && e < p.E) p.offsets[e] = ahead + sum - n;
            if (e < p.pitch) before[e] += ahead + sum - n;
            ahead += __builtin_amdgcn_readlane(sum, 63);
        }
        if (blockIdx.x == 0 && threadIdx.x == 0) p.offsets[p.E] = ahead;
    }
    __syncthreads();
    const int t0 = blockIdx.x * ROUTE_TOKENS, tokens = min(ROUTE_TOKENS, p.T - t0);
    for (int c = threadIdx.x; c < tokens * p.k; c += PLACE_THREADS) {
        const int i = c / p.k;
        const int64_t at = (int64_t)t0 * p.k + c;
        const int e = p.experts[at];
        const int row = before[e] + __popcll(p.masks[(int64_t)blockIdx.x * p.E + e] & ((1ull << i) - 1));
        p.rows[row] = t0 + i;
        p.slots[at] = row;
    }
}

inline int route_blocks(int T) { return (int)(((int64_t)T + ROUTE_TOKENS - 1) / ROUTE_TOKENS); }
inline int route_pitch(int E) { return (E + 15) & ~15; }

template <bool ALONE>
void launch_select(const RouteParams &p, hipStream_t s) {
    const dim3 grid((unsigned)(ALONE ? 1 : p.blocks)), block(64 * ROUTE_WAVES);
    if (p.E <= 64) hipLaunchKernelGGL((route_select_kernel<1, ALONE>), grid, block, 0, s, p);
    else if (p.E <= 128) hipLaunchKernelGGL((route_select_kernel<2, ALONE>), grid, block, 0, s, p);
    else if (p.E <= 256) hipLaunchKernelGGL((route_select_kernel<4, ALONE>), grid, block, 0, s, p);
    else hipLaunchKernelGGL((route_select_kernel<8, ALONE>), grid, block, 0, s, p);
}

}  // namespace

size_t route_topk_workspace(int T, int E) {
    if (T <= ROUTE_TOKENS) return 0;
    return (size_t)route_blocks(T) * ((size_t)E * 8 + (size_t)route_pitch(E));
}

hipError_t launch_route_topk(const void *logits, int64_t ldl, int dtype, int T, int E, int k, int renormalize, int32_t *experts, float *weights,
                             int32_t *offsets, int32_t *rows, int32_t *slots, void *workspace, hipStream_t s) {
    RouteParams p{logits, ldl, dtype, T, E, k, renormalize, experts, weights, offsets, rows, slots, nullptr, nullptr, route_pitch(E), route_blocks(T)};
    if (T <= ROUTE_TOKENS) {
        launch_select<true>(p, s);
        return hipGetLastError();
    }
    p.counts = reinterpret_cast<uint8_t *>(workspace);
    p.masks = reinterpret_cast<uint64_t *>(p.counts + (int64_t)p.blocks * p.pitch);
    launch_select<false>(p, s);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(route_place_kernel, dim3((unsigned)p.blocks), dim3(PLACE_THREADS), 2 * p.pitch * sizeof(int32_t), s, p);
    return hipGetLastError();
}

}  // namespace tbik
