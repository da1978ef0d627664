// The router of a mixture of experts: the k largest logits of each token, their weights, and the order in which products grouped
// by expert take the tokens.
//
// A token is one wavefront's work whatever the batch: each lane holds every 64th logit as a key that orders like it (NaN lowest), largest first, and
// k times the largest of the lanes' first keys is found with data-parallel moves and its owner with a ballot.  The
// order needs no sort: a token chooses an expert at most once, so a block of up to 64 tokens is one 64-bit mask per expert, and a
// choice's place is the expert's first row + what earlier blocks have + the bits below the token's in the mask.  Masks are
// joined with integer "or", counts are sums of integers: nothing depends on the order in which wavefronts run.
//
// Bound by launches and latency: 8191 tokens of 128 experts read 2 MB.  Up to 64 tokens are one workgroup and one launch; more are
// two launches, a block of 32 tokens each (select), then every block adds up the blocks' counts (a byte per expert and block) for itself (place); what that
// reads grows with the square of the tokens, so above ROUTE_MANY blocks the counts are summed over chunks of blocks and the chunks scanned first (sum, scan).
// Measured, kernels: one token of 128 experts, 8 chosen, 3.0 us; 8191 tokens 8.7 us (select) and 4.5 (place).  Whole calls with and without the two extra
// launches: 16384 tokens of 128 experts 21.7 / 18.9 us, 32768 30.4 / 34.9 (of 8 experts 29.0 / 23.6); with them 65536 47 us, 1048576 537.  Of so many the
// instructions of the rounds are the bound (their bytes take some 130 us): a maximum over 64 lanes for each choice of each token.
#include "tbik_device.hpp"
#include "tbik_internal.hpp"

namespace tbik {

namespace {

constexpr int ROUTE_ALONE = 64;            // tokens of a block that is the whole batch: bits of a mask
constexpr int ROUTE_TOKENS = 32;           // of a block of many: 8192 tokens are a block for each compute unit
constexpr int TOKENS_PER_WAVE = 4;
constexpr int ROUTE_MANY = 1024;           // blocks
constexpr int ROUTE_CHUNK = 64;            // blocks of a chunk

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

// The largest of 64 lanes' values: within rows of 16 by shifts, then from row to row; lane 63 has it.  Six instructions and a move to a scalar register.
template <int CTRL>
__device__ __forceinline__ uint32_t max_with(uint32_t v) { return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, false)); }
__device__ __forceinline__ uint32_t wave_max_u32(uint32_t v) {
    v = max_with<0x111>(v);                            // row_shr 1, 2, 4, 8
    v = max_with<0x112>(v);
    v = max_with<0x114>(v);
    v = max_with<0x118>(v);
    v = max_with<0x142>(v);                            // row_bcast 15, 31
    v = max_with<0x143>(v);
    return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}

// Sums up to and with each lane's, and of all 64 in lane 63.
template <int CTRL, int ROWS>
__device__ __forceinline__ int plus(int v) { return v + __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xf, false); }
__device__ __forceinline__ int wave_scan(int v) {
    v = plus<0x111, 0xf>(v);                           // within rows of 16: row_shr 1, 2, 4, 8
    v = plus<0x112, 0xf>(v);
    v = plus<0x114, 0xf>(v);
    v = plus<0x118, 0xf>(v);
    v = plus<0x142, 0xa>(v);                           // row_bcast 15 to rows 1 and 3, 31 to rows 2 and 3
    return plus<0x143, 0xc>(v);
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
    int32_t *chunk_rows;                   // more than ROUTE_MANY blocks: [chunks + 1, pitch], choices of the chunks before, of all
    int chunks;
};

__device__ __forceinline__ uint32_t raw_logit(const RouteParams &p, int64_t i) {
    return p.dtype == TBIK_F32 ? reinterpret_cast<const uint32_t *>(p.logits)[i] : reinterpret_cast<const uint16_t *>(p.logits)[i];
}
__device__ __forceinline__ float logit_of_raw(uint32_t raw, int dtype) {
    return dtype == TBIK_F32 ? __uint_as_float(raw) : dtype == TBIK_F16 ? (float)__builtin_bit_cast(_Float16, (uint16_t)raw) : bf16_bits_to_f32(raw);
}

// The choices of TOKENS tokens, t[i] of them below p.T (the others repeat one): lane j (j < k) gets expert and weight of choice j.  The weights: e^(l_j - l_0)
// over the sum of the chosen, ascending j, or over the sum of all experts (lane-wise chains in ascending expert order, then the tree over the lanes).
// A token's rounds wait for each other, of the moves and ballots that each consists of; four tokens at once fill the gaps.
template <int PER_LANE, int TOKENS>
__device__ __forceinline__ void choose(const RouteParams &p, const int (&t)[TOKENS], int lane, int (&expert)[TOKENS], float (&weight)[TOKENS]) {
    // A lane's logits in falling order, the lower expert first among equals: a round looks at the lanes' first ones alone.
    uint32_t key[TOKENS][PER_LANE];
    int index[TOKENS][PER_LANE];
    // All loads before the first use (one branch by type around them; behind the last expert it is read once more).
    if (p.dtype == TBIK_F32) {
#pragma unroll
        for (int i = 0; i < TOKENS; ++i)
#pragma unroll
            for (int j = 0; j < PER_LANE; ++j) key[i][j] = reinterpret_cast<const uint32_t *>(p.logits)[(int64_t)t[i] * p.ldl + min(j * 64 + lane, p.E - 1)];
    } else {
#pragma unroll
        for (int i = 0; i < TOKENS; ++i)
#pragma unroll
            for (int j = 0; j < PER_LANE; ++j) key[i][j] = reinterpret_cast<const uint16_t *>(p.logits)[(int64_t)t[i] * p.ldl + min(j * 64 + lane, p.E - 1)];
    }
#pragma unroll
    for (int i = 0; i < TOKENS; ++i)
#pragma unroll
        for (int j = 0; j < PER_LANE; ++j) {
            const int e = j * 64 + lane;
            key[i][j] = e < p.E ? key_of(logit_of_raw(key[i][j], p.dtype)) : 0u;
            index[i][j] = e;
        }
#pragma unroll
    for (int i = 0; i < TOKENS; ++i)
#pragma unroll
        for (int n = 1; n < PER_LANE; ++n)
#pragma unroll
            for (int j = n; j > 0; --j) {              // into its place among the n before it
                const bool swap = key[i][j] > key[i][j - 1];
                const uint32_t high = swap ? key[i][j] : key[i][j - 1], low = swap ? key[i][j - 1] : key[i][j];
                const int first = swap ? index[i][j] : index[i][j - 1], second = swap ? index[i][j - 1] : index[i][j];
                key[i][j - 1] = high;
                key[i][j] = low;
                index[i][j - 1] = first;
                index[i][j] = second;
            }
    float all[TOKENS];
    uint32_t first[TOKENS], mine[TOKENS];
#pragma unroll
    for (int i = 0; i < TOKENS; ++i) {
        all[i] = 0.0f;
        first[i] = mine[i] = 0u;
        expert[i] = 0;
    }
    if (!p.renormalize) {                              // in ascending expert order, from memory once more
#pragma unroll
        for (int i = 0; i < TOKENS; ++i) {
            const float top = logit_of(wave_max_u32(key[i][0]));
#pragma unroll
            for (int j = 0; j < PER_LANE; ++j)
                if (j * 64 + lane < p.E) all[i] = all[i] + expf(logit_of_raw(raw_logit(p, (int64_t)t[i] * p.ldl + j * 64 + lane), p.dtype) - top);
            all[i] = wave_tree_sum(all[i]);
        }
    }
    for (int round = 0; round < p.k; ++round) {
        uint32_t best[TOKENS];
#pragma unroll
        for (int i = 0; i < TOKENS; ++i) best[i] = wave_max_u32(key[i][0]);
#pragma unroll
        for (int i = 0; i < TOKENS; ++i) {
            if (round == 0) first[i] = best[i];
            const uint64_t owners = __builtin_amdgcn_ballot_w64(key[i][0] == best[i]);
            uint64_t lowest = owners;                              // of several, those of the first block of 64 experts that has one
#pragma unroll
            for (int j = PER_LANE - 1; j > 0; --j) {
                const uint64_t low = owners & __builtin_amdgcn_ballot_w64(index[i][0] < 64 * j);
                lowest = low ? low : lowest;
            }
            const int at = __builtin_ctzll(lowest);
            const int winner = __builtin_amdgcn_readlane(index[i][0], at);
            if (lane == round) {
                mine[i] = best[i];
                expert[i] = winner;
            }
            const bool taken = lane == at;
#pragma unroll
            for (int j = 0; j < PER_LANE; ++j) {
                key[i][j] = taken ? (j + 1 < PER_LANE ? key[i][j + 1] : 0u) : key[i][j];
                if (j + 1 < PER_LANE) index[i][j] = taken ? index[i][j + 1] : index[i][j];
            }
        }
    }
#pragma unroll
    for (int i = 0; i < TOKENS; ++i) {
        const float top = logit_of(first[i]);
        const float e = lane < p.k ? expf(logit_of(mine[i]) - top) : 0.0f;
        float sum = all[i];
        if (p.renormalize) {
            sum = 0.0f;
            for (int j = 0; j < p.k; ++j) sum = sum + __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, e), j));
        }
        weight[i] = top == -__builtin_inff() ? 0.0f : e / sum;       // nothing to choose from: no weight
    }
}

// ALONE: one block is the whole batch, and places its choices itself.
template <int PER_LANE, bool ALONE>
__global__ __launch_bounds__(64 * (ALONE ? ROUTE_ALONE : ROUTE_TOKENS) / TOKENS_PER_WAVE) void route_select_kernel(const RouteParams p) {
    constexpr int BLOCK_TOKENS = ALONE ? ROUTE_ALONE : ROUTE_TOKENS, WAVES = BLOCK_TOKENS / TOKENS_PER_WAVE;
    __shared__ uint64_t mask[PER_LANE * 64];
    __shared__ int32_t first_row[ALONE ? PER_LANE * 64 : 1];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int t0 = blockIdx.x * BLOCK_TOKENS;
    const int tokens = min(BLOCK_TOKENS, p.T - t0);
    for (int e = threadIdx.x; e < PER_LANE * 64; e += 64 * WAVES) mask[e] = 0;
    __syncthreads();
    auto keep = [&](int i, int expert, float weight) __attribute__((always_inline)) {
        if (lane < p.k && i < tokens) {
            const int64_t at = (int64_t)(t0 + i) * p.k + lane;
            p.experts[at] = expert;
            p.weights[at] = weight;
            atomicOr(reinterpret_cast<unsigned long long *>(&mask[expert]), 1ull << i);
        }
    };
    if (tokens <= WAVES) {                             // one each: no gaps to fill
        if (wave < tokens) {
            int expert[1];
            float weight[1];
            choose<PER_LANE, 1>(p, {t0 + wave}, lane, expert, weight);
            keep(wave, expert[0], weight[0]);
        }
    } else {
        constexpr int TOKENS = PER_LANE < 8 ? TOKENS_PER_WAVE : ALONE ? 1 : 2;              // at once: what the registers hold
        for (int from = wave; from < tokens; from += TOKENS * WAVES) {
            int t[TOKENS], expert[TOKENS];
            float weight[TOKENS];
#pragma unroll
            for (int i = 0; i < TOKENS; ++i) t[i] = min(t0 + from + i * WAVES, p.T - 1);
            choose<PER_LANE, TOKENS>(p, t, lane, expert, weight);
#pragma unroll
            for (int i = 0; i < TOKENS; ++i) keep(from + i * WAVES, expert[i], weight[i]);
        }
    }
    __syncthreads();
    if constexpr (!ALONE) {
        for (int e = threadIdx.x; e < p.pitch; e += 64 * WAVES) {
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
                const int sum = wave_scan(n);
                first_row[e] = before + sum - n;
                if (e <= p.E) p.offsets[e] = before + sum - n;
                before += __builtin_amdgcn_readlane(sum, 63);
            }
            if (p.E == PER_LANE * 64 && lane == 0) p.offsets[p.E] = before;
        }
        __syncthreads();
        for (int c = threadIdx.x; c < tokens * p.k; c += 64 * WAVES) {
            const int i = c / p.k, e = p.experts[c];
            const int row = first_row[e] + __popcll(mask[e] & ((1ull << i) - 1));
            p.rows[row] = i;
            p.slots[c] = row;
        }
    }
}

constexpr int PLACE_THREADS = 512;

// Choices of a chunk of blocks, four experts a thread.
__global__ __launch_bounds__(kMaxGroups / 4) void route_sum_kernel(const RouteParams p) {
    const int quads = p.pitch / 4, c = threadIdx.x;
    if (c >= quads) return;
    const uint32_t *const counts = reinterpret_cast<const uint32_t *>(p.counts) + c;
    const int64_t b0 = (int64_t)blockIdx.x * ROUTE_CHUNK, b1 = min(b0 + ROUTE_CHUNK, (int64_t)p.blocks);
    uint32_t even = 0, odd = 0;                        // up to 32 a block: 64 do not overflow 16 bits
#pragma unroll 16
    for (int64_t b = b0; b < b1; ++b) {
        const uint32_t v = counts[b * quads];
        even += v & 0x00ff00ffu;
        odd += (v >> 8) & 0x00ff00ffu;
    }
    int32_t *const to = p.chunk_rows + (int64_t)blockIdx.x * p.pitch + c * 4;
    to[0] = even & 0xffffu;
    to[1] = odd & 0xffffu;
    to[2] = even >> 16;
    to[3] = odd >> 16;
}
// An expert a workgroup: the chunks' sums, 256 at a time, become those of the chunks before; behind the last, of all.
__global__ __launch_bounds__(256) void route_scan_kernel(const RouteParams p) {
    __shared__ int32_t wave_sum[4];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int32_t *const rows = p.chunk_rows + blockIdx.x;
    int before = 0;
    for (int from = 0; from < p.chunks; from += 256) {
        const int c = from + threadIdx.x;
        const int n = c < p.chunks ? rows[(int64_t)c * p.pitch] : 0, sum = wave_scan(n);
        if (lane == 63) wave_sum[wave] = sum;
        __syncthreads();
        int mine = before + sum - n;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            if (w < wave) mine += wave_sum[w];
            before += wave_sum[w];
        }
        if (c < p.chunks) rows[(int64_t)c * p.pitch] = mine;
        __syncthreads();
    }
    if (threadIdx.x == 0) rows[(int64_t)p.chunks * p.pitch] = before;
}

// MANY: the choices of the chunks before this block's, and of all, are known.
template <bool MANY>
__global__ __launch_bounds__(PLACE_THREADS) void route_place_kernel(const RouteParams p) {
    __shared__ int32_t total[kMaxGroups], before[kMaxGroups];      // choices of all blocks; of the blocks before this one, then first rows
    __shared__ int32_t part[2][PLACE_THREADS * 4];
    const int t0 = blockIdx.x * ROUTE_TOKENS, tokens = min(ROUTE_TOKENS, p.T - t0);
    const int64_t first = (int64_t)t0 * p.k;
    const uint64_t *const masks = p.masks + (int64_t)blockIdx.x * p.E;
    // The thread's first choice is on its way while the counts are added up.
    int e = 0;
    uint64_t m = 0;
    if ((int)threadIdx.x < tokens * p.k) {
        e = p.experts[first + threadIdx.x];
        m = masks[e];
    }
    // A thread adds up four experts' counts of every `step`-th block, two of them to a register (up to 32 a block: 2047 blocks do not overflow 16 bits).
    const int quads = p.pitch / 4, step = PLACE_THREADS / quads;
    if ((int)threadIdx.x < step * quads) {
        const int c = threadIdx.x % quads, own = threadIdx.x / quads;
        const int begin = MANY ? (int)blockIdx.x / ROUTE_CHUNK * ROUTE_CHUNK : 0, end = MANY ? (int)blockIdx.x : p.blocks;
        const uint32_t *const counts = reinterpret_cast<const uint32_t *>(p.counts) + c;
        int all[4] = {}, early[4] = {};
        for (int from = begin + own; from < end; from += 1000 * step) {
            uint32_t even[2] = {0, 0}, odd[2] = {0, 0};            // [earlier blocks, others]
            const int until = min(end, from + 1000 * step);
            for (int b0 = from; b0 < until; b0 += 8 * step) {
                uint32_t v[8];                                     // loads that do not wait for each other
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = b0 + i * step < until ? counts[(int64_t)(b0 + i * step) * quads] : 0u;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const bool ahead = b0 + i * step < (int)blockIdx.x;
                    even[0] += ahead ? v[i] & 0x00ff00ffu : 0u;
                    odd[0] += ahead ? (v[i] >> 8) & 0x00ff00ffu : 0u;
                    even[1] += v[i] & 0x00ff00ffu;
                    odd[1] += (v[i] >> 8) & 0x00ff00ffu;
                }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                early[i] += ((i & 1 ? odd[0] : even[0]) >> (i & 2 ? 16 : 0)) & 0xffffu;
                all[i] += ((i & 1 ? odd[1] : even[1]) >> (i & 2 ? 16 : 0)) & 0xffffu;
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            part[0][own * p.pitch + c * 4 + i] = all[i];
            part[1][own * p.pitch + c * 4 + i] = early[i];
        }
    }
    __syncthreads();
    for (int e = threadIdx.x; e < p.pitch; e += PLACE_THREADS) {
        int a = 0, b = 0;
        for (int i = 0; i < step; ++i) {
            a += part[0][i * p.pitch + e];
            b += part[1][i * p.pitch + e];
        }
        if constexpr (MANY) {
            a = p.chunk_rows[(int64_t)p.chunks * p.pitch + e];
            b += p.chunk_rows[(int64_t)(blockIdx.x / ROUTE_CHUNK) * p.pitch + e];
        }
        total[e] = a;
        before[e] = b;
    }
    __syncthreads();
    if (threadIdx.x < 64) {                            // first rows: a scan over the experts
        int ahead = 0;
        for (int e = threadIdx.x; e - (int)threadIdx.x < p.pitch; e += 64) {
            const int n = e < p.pitch ? total[e] : 0;
            const int sum = wave_scan(n);
            if (blockIdx.x == 0 && e < p.E) p.offsets[e] = ahead + sum - n;
            if (e < p.pitch) before[e] += ahead + sum - n;
            ahead += __builtin_amdgcn_readlane(sum, 63);
        }
        if (blockIdx.x == 0 && threadIdx.x == 0) p.offsets[p.E] = ahead;
    }
    __syncthreads();
    for (int c = threadIdx.x; c < tokens * p.k; c += PLACE_THREADS) {
        if (c >= PLACE_THREADS) {
            e = p.experts[first + c];
            m = masks[e];
        }
        const int i = c / p.k, row = before[e] + __popcll(m & ((1ull << i) - 1));
        p.rows[row] = t0 + i;
        p.slots[first + c] = row;
    }
}

inline int route_blocks(int T) { return (int)(((int64_t)T + ROUTE_TOKENS - 1) / ROUTE_TOKENS); }
inline int route_chunks(int T) { return (route_blocks(T) + ROUTE_CHUNK - 1) / ROUTE_CHUNK; }
inline int route_pitch(int E) { return (E + 15) & ~15; }

template <bool ALONE>
void launch_select(const RouteParams &p, hipStream_t s) {
    const dim3 grid((unsigned)(ALONE ? 1 : p.blocks)), block(64 * (ALONE ? ROUTE_ALONE : ROUTE_TOKENS) / TOKENS_PER_WAVE);
    if (p.E <= 64) hipLaunchKernelGGL((route_select_kernel<1, ALONE>), grid, block, 0, s, p);
    else if (p.E <= 128) hipLaunchKernelGGL((route_select_kernel<2, ALONE>), grid, block, 0, s, p);
    else if (p.E <= 256) hipLaunchKernelGGL((route_select_kernel<4, ALONE>), grid, block, 0, s, p);
    else hipLaunchKernelGGL((route_select_kernel<8, ALONE>), grid, block, 0, s, p);
}

}  // namespace

size_t route_topk_workspace(int T, int E) {
    if (T <= ROUTE_ALONE) return 0;
    const size_t sums = route_blocks(T) > ROUTE_MANY ? (size_t)(route_chunks(T) + 1) * route_pitch(E) * 4 : 0;
    return (size_t)route_blocks(T) * ((size_t)E * 8 + (size_t)route_pitch(E)) + sums;
}

hipError_t launch_route_topk(const void *logits, int64_t ldl, int dtype, int T, int E, int k, int renormalize, int32_t *experts, float *weights,
                             int32_t *offsets, int32_t *rows, int32_t *slots, void *workspace, hipStream_t s) {
    RouteParams p{logits, ldl, dtype, T, E, k, renormalize, experts, weights, offsets, rows, slots, nullptr, nullptr, route_pitch(E), route_blocks(T), nullptr,
                  route_chunks(T)};
    if (T <= ROUTE_ALONE) {
        launch_select<true>(p, s);
        return hipGetLastError();
    }
    p.counts = reinterpret_cast<uint8_t *>(workspace);
    p.masks = reinterpret_cast<uint64_t *>(p.counts + (int64_t)p.blocks * p.pitch);
    launch_select<false>(p, s);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (p.blocks <= ROUTE_MANY) {
        hipLaunchKernelGGL(route_place_kernel<false>, dim3((unsigned)p.blocks), dim3(PLACE_THREADS), 0, s, p);
        return hipGetLastError();
    }
    p.chunk_rows = reinterpret_cast<int32_t *>(p.masks + (int64_t)p.blocks * E);
    hipLaunchKernelGGL(route_sum_kernel, dim3((unsigned)p.chunks), dim3((unsigned)((p.pitch / 4 + 63) & ~63)), 0, s, p);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    hipLaunchKernelGGL(route_scan_kernel, dim3((unsigned)p.pitch), dim3(256), 0, s, p);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    hipLaunchKernelGGL(route_place_kernel<true>, dim3((unsigned)p.blocks), dim3(PLACE_THREADS), 0, s, p);
    return hipGetLastError();
}

}  // namespace tbik
