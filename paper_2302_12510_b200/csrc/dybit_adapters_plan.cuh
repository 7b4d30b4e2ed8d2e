// The plan of a batch: tokens grouped by adapter, and the lists of work that the adapter kernels walk.
//
// Group a < n holds the tokens of adapter a in their own order, group n those without an adapter.  Integer work only:
// one block counts and scans, then one block per group places its tokens by scanning the ids (T * (n + 1) comparisons
// from L2, a few microseconds for thousands of tokens and dozens of adapters; a plan is made once per batch and read
// by every projection of every layer).
#pragma once

#include "dybit_common.cuh"

namespace dybit {

constexpr int kPlanThreads = 1024;
constexpr int kChunkTokens = 512;            // of one adapter that a block of the gradient kernel sums up (longer sums: the tensor core's
                                             // cut-off additions show, over 1e-6 of the result for 1024 tokens of which 2 us are gained)

// A tile: up to 16, 32 or 64 tokens of one adapter.  `step` counts 16-token steps of assigned tokens.
struct AdapterTile { int adapter, start, count, step; };
// A chunk: kChunkTokens tokens of one adapter, or what is left of it: `rest` tokens from its start on.  `index` counts the
// chunks of the adapter; `partial` is the adapter's first slot among the chunks of adapters that have more than one.
struct AdapterChunk { int adapter, start, rest, step, index, partial, pad0, pad1; };

// Word offsets of a plan's parts for (T, n); the capacities bound what the device fills in.
struct PlanLayout {
    int64_t tiles_cap[3], chunks_cap, steps_cap, partials_cap;
    int64_t perm, offsets, tiles[3], chunks, words;
    __host__ __device__ static int64_t up4(int64_t v) { return (v + 3) / 4 * 4; }
    __host__ __device__ PlanLayout(int64_t T, int n) {
        const int64_t groups = T < n + 1 ? T : n + 1, adapters = T < n ? T : n;
        for (int i = 0; i < 3; ++i) tiles_cap[i] = T / (16 << i) + groups;
        steps_cap = T / 16 + adapters;
        chunks_cap = T / kChunkTokens + adapters;
        partials_cap = 2 * (T / kChunkTokens);          // an adapter with c >= 2 chunks has more than c/2 * kChunkTokens tokens
        int64_t w = 8;                                   // counts of tiles (three sizes), chunks; the rest spare
        perm = w;
        w = up4(w + T);
        offsets = w;                                     // per group: {first token, first tile of each size, first chunk, first partial} x (n + 2)
        w = up4(w + 6 * (int64_t)(n + 2));
        for (int i = 0; i < 3; ++i) {
            tiles[i] = w;
            w += 4 * tiles_cap[i];
        }
        chunks = w;
        w += 8 * chunks_cap;
        words = w;
    }
};

constexpr int kPlanColumns = 6;              // of the offsets table

__device__ __forceinline__ int plan_group(int id, int n) { return (unsigned)id < (unsigned)n ? id : n; }

__device__ __forceinline__ int plan_column(int col, int tokens, bool assigned) {
    if (col == 0) return tokens;
    if (col <= 3) return (tokens + (16 << (col - 1)) - 1) / (16 << (col - 1));
    const int chunks = assigned ? (tokens + kChunkTokens - 1) / kChunkTokens : 0;
    return col == 4 ? chunks : (chunks > 1 ? chunks : 0);
}

// One block: tokens of each group, then exclusive prefix sums of the six columns.
__global__ void __launch_bounds__(kPlanThreads) adapters_count_kernel(const int *__restrict__ ids, int64_t T, int n, int *plan) {
    extern __shared__ int s_bins[];                        // n + 1 counts
    __shared__ int s_warp[kPlanThreads / 32];
    pdl_enter();
    const PlanLayout L(T, n);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    for (int i = threadIdx.x; i <= n; i += kPlanThreads) s_bins[i] = 0;
    __syncthreads();
    for (int64_t t = threadIdx.x; t < T; t += kPlanThreads) atomicAdd(&s_bins[plan_group(ids[t], n)], 1);
    __syncthreads();
    const int per = (n + 1 + kPlanThreads - 1) / kPlanThreads, first = threadIdx.x * per;
    for (int col = 0; col < kPlanColumns; ++col) {
        int mine = 0;
        for (int i = first; i < first + per && i <= n; ++i) mine += plan_column(col, s_bins[i], i < n);
        int sum = mine;                                    // inclusive scan over the warp, then over the warps
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int o = __shfl_up_sync(0xffffffffu, sum, d);
            if (lane >= d) sum += o;
        }
        if (lane == 31) s_warp[warp] = sum;
        __syncthreads();
        int before = 0;
        for (int w = 0; w < warp; ++w) before += s_warp[w];
        int at = before + sum - mine;
        for (int i = first; i < first + per && i <= n; ++i) {
            plan[L.offsets + (int64_t)i * kPlanColumns + col] = at;
            at += plan_column(col, s_bins[i], i < n);
        }
        if (first <= n && first + per > n) {               // the thread of the last group also closes the table
            plan[L.offsets + (int64_t)(n + 1) * kPlanColumns + col] = at;
            if (col >= 1 && col <= 4) plan[col - 1] = at;
        }
        __syncthreads();
    }
}

// Block a: the tokens of group a in order, its tiles and its chunks.
__global__ void __launch_bounds__(kPlanThreads) adapters_place_kernel(const int *__restrict__ ids, int64_t T, int n, int *plan) {
    __shared__ int s_warp[kPlanThreads / 32];
    pdl_enter();
    const PlanLayout L(T, n);
    const int a = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int *off = plan + L.offsets + (int64_t)a * kPlanColumns;
    const int start = off[0], count = off[kPlanColumns] - start;
    if (count == 0) return;
    int *perm = plan + L.perm + start;
    int done = 0;
    for (int64_t t0 = 0; t0 < T && done < count; t0 += kPlanThreads) {
        const int64_t t = t0 + threadIdx.x;
        const bool is = t < T && plan_group(ids[t], n) == a;
        const unsigned votes = __ballot_sync(0xffffffffu, is);
        if (lane == 0) s_warp[warp] = __popc(votes);
        __syncthreads();
        int before = lane < warp ? s_warp[lane] : 0, all = s_warp[lane];
        before = __reduce_add_sync(0xffffffffu, before);
        all = __reduce_add_sync(0xffffffffu, all);
        const int at = done + before + __popc(votes & ((1u << lane) - 1u));
        if (is && DYBIT_CHECK(at < count && start + at < T, 0x70)) perm[at] = (int)t;
        done += all;
        __syncthreads();
    }
    const int step0 = off[1];                              // group n comes last: the tiles of 16 before it are the steps
    for (int i = 0; i < 3; ++i) {
        const int size = 16 << i, tiles = (count + size - 1) / size;
        AdapterTile *list = reinterpret_cast<AdapterTile *>(plan + L.tiles[i]) + off[1 + i];
        for (int k = threadIdx.x; k < tiles; k += kPlanThreads)
            if (DYBIT_CHECK(off[1 + i] + k < L.tiles_cap[i], 0x71)) list[k] = {a < n ? a : -1, start + k * size, min(size, count - k * size), step0 + k * (size / 16)};
    }
    if (a < n) {
        const int chunks = (count + kChunkTokens - 1) / kChunkTokens;
        AdapterChunk *list = reinterpret_cast<AdapterChunk *>(plan + L.chunks) + off[4];
        for (int k = threadIdx.x; k < chunks; k += kPlanThreads)
            if (DYBIT_CHECK(off[4] + k < L.chunks_cap, 0x72)) list[k] = {a, start + k * kChunkTokens, count - k * kChunkTokens, step0 + k * (kChunkTokens / 16), k, off[5], 0, 0};
    }
}

}  // namespace dybit

extern "C" {

size_t dybit_adapters_plan_bytes(int64_t T, int n_adapters) {
    if (T < 0 || T > 0x7fffffff / 2 || n_adapters < 1 || n_adapters > DYBIT_MAX_ADAPTERS) return 0;
    return (size_t)dybit::round_up(dybit::PlanLayout(T, n_adapters).words * 4, 16);
}

dybit_status dybit_adapters_plan(int64_t T, const int32_t *ids, int n_adapters, void *plan, size_t plan_bytes,
                                 void *stream) {
    using namespace dybit;
    const size_t need = dybit_adapters_plan_bytes(T, n_adapters);
    if (need == 0) return DYBIT_ERR_INVALID_ARG;
    if (plan == nullptr || (T > 0 && ids == nullptr)) return DYBIT_ERR_INVALID_ARG;
    if (!aligned(plan, 16) || !aligned(ids, 4)) return DYBIT_ERR_ALIGNMENT;
    if (plan_bytes < need) return DYBIT_ERR_WORKSPACE;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    launch_k(adapters_count_kernel, dim3(1), dim3(kPlanThreads), (size_t)(n_adapters + 1) * 4, s, ids, T, n_adapters,
             static_cast<int *>(plan));
    const dybit_status st = launch_status();
    if (st != DYBIT_OK || T == 0) return st;
    launch_k(adapters_place_kernel, dim3((unsigned)n_adapters + 1), dim3(kPlanThreads), 0, s, ids, T, n_adapters,
             static_cast<int *>(plan));
    return launch_status();
}

}  // extern "C"
