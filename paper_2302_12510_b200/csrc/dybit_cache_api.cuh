// Host side of the key-value cache: checks of arguments, sizes, launches.
#pragma once

#include <limits.h>

#include <type_traits>

#include "dybit_cache_prefill.cuh"

namespace dybit {

static dybit_status check_cache(const dybit_cache *c) {
    if (c == nullptr) return DYBIT_ERR_INVALID_ARG;
    if (c->pages < 0 || c->heads < 1 || c->dim < 1 || c->page < 1) return DYBIT_ERR_INVALID_ARG;
    if (c->dim % 16 != 0 || c->dim > kCacheMaxDim || (c->page != 16 && c->page != 32 && c->page != 64 && c->page != 128)) return DYBIT_ERR_UNSUPPORTED;
    if (c->heads > 4096 || c->pages > 0x7ffffffe / c->heads) return DYBIT_ERR_UNSUPPORTED;
    return DYBIT_OK;
}

// The cache's memory, which the plan does not look at.
static dybit_status check_cache_memory(const dybit_cache *c) {
    if (c->pages == 0) return DYBIT_OK;
    if (c->k_codes == nullptr || c->v_codes == nullptr || c->k_scales == nullptr || c->v_scales == nullptr) return DYBIT_ERR_INVALID_ARG;
    if (!aligned(c->k_codes, 16) || !aligned(c->v_codes, 16) || !aligned(c->k_scales, 4) || !aligned(c->v_scales, 4)) return DYBIT_ERR_ALIGNMENT;
    return DYBIT_OK;
}

static dybit_status check_batch(const dybit_cache *c, const dybit_cache_batch *b) {
    if (b == nullptr) return DYBIT_ERR_INVALID_ARG;
    if (b->sequences < 0 || b->tokens < 0 || b->max_new < 0 || b->q_heads < 1 || b->max_pages < 0 || b->window < 0 || b->table_stride < b->max_pages) return DYBIT_ERR_INVALID_ARG;
    if (b->q_heads % c->heads != 0) return DYBIT_ERR_INVALID_ARG;
    if (b->q_heads / c->heads > kCacheMaxGroup || b->sequences > (1 << 20) || b->tokens > (1 << 26)) return DYBIT_ERR_UNSUPPORTED;
    if (b->tokens * (int64_t)b->q_heads > (1 << 30) || (int64_t)b->max_pages * c->page > (1 << 26)) return DYBIT_ERR_UNSUPPORTED;
    return DYBIT_OK;
}

// The window as the kernels take it.  No sequence has more than 2^26 tokens, so one of 2^26 holds all of them; a longer one would
// pass 32 bits where it is taken from a position in front of the first.
static int window_or_none(int window) { return window > 0 && window < (1 << 26) ? window : INT_MAX; }

// Rows of a sequence that small tiles take, the others large ones: two tiles of 16, or four where the batch is small.  A large tile
// costs its keys the same however full it is, small ones each cost them; but a block of large tiles takes longer to begin and to
// end.  8 key heads of 4 queries, 4096 keys, small against large tiles: 16 sequences of 32 rows 97 : 113 us, of 48 rows 137 : 113 us, of 64
// rows 166 : 114 us; one sequence of 48 rows 27 : 44 us, of 64 rows 28 : 44 us.  Groups of 128 heads, one token of each of 64 sequences
// 160 : 74 us, of one 23 : 41 us: a small batch's single tokens take small tiles whatever their group.
constexpr int kSmallMost = 32, kSmallMostAlone = 64, kAloneRows = 2048;
static CacheShape cache_shape(const dybit_cache *c, const dybit_cache_batch *b) {
    CacheShape s = {};
    s.T = b->tokens;
    s.B = b->sequences;
    s.page = c->page;
    s.heads = c->heads;
    s.group = b->q_heads / c->heads;
    s.max_new = (int)std::min<int64_t>(b->max_new, b->tokens);
    s.max_pages = b->max_pages;
    s.small_tokens = b->tokens * b->q_heads <= kAloneRows ? std::max(1, kSmallMostAlone / s.group) : kSmallMost / s.group;
    s.causal = b->causal != 0;
    s.window = window_or_none(b->window);
    s.small_rows = (int64_t)s.max_new * s.group <= 8 ? 8 : kSmallRows;
    return s;
}

static dybit_status check_plan(const dybit_cache *c, const dybit_cache_batch *b, const void *plan) {
    dybit_status st = check_cache(c);
    if (st == DYBIT_OK) st = check_cache_memory(c);
    if (st == DYBIT_OK) st = check_batch(c, b);
    if (st != DYBIT_OK) return st;
    if (plan == nullptr || (b->table == nullptr && b->sequences > 0 && b->max_pages > 0)) return DYBIT_ERR_INVALID_ARG;
    return aligned(plan, 16) && aligned(b->table, 4) ? DYBIT_OK : DYBIT_ERR_ALIGNMENT;
}

static int log2_of(int v) {
    int s = 0;
    while ((1 << s) < v) ++s;
    return s;
}

// Tokens x heads x dim with unit inner stride.
static dybit_status check_heads(const void *x, dybit_dtype t, int64_t token, int64_t head, int64_t T, int heads, int dim) {
    if (x == nullptr) return DYBIT_ERR_INVALID_ARG;
    if ((heads > 1 && head < dim) || (T > 1 && token < dim)) return DYBIT_ERR_INVALID_ARG;
    return aligned(x, dtype_bytes(t)) ? DYBIT_OK : DYBIT_ERR_ALIGNMENT;
}
static bool heads_aligned(const void *x, dybit_dtype t, int64_t token, int64_t head, int bytes) {
    return aligned(x, bytes) && token * dtype_bytes(t) % bytes == 0 && head * dtype_bytes(t) % bytes == 0;
}

template <typename T, bool VEC>
static dybit_status launch_cache_write(const CacheWrite &p, int64_t items, int most, cudaStream_t s) {
    const int64_t tiles = items * 2 * p.heads;
    auto go = [&](auto kernel, int tiles_per_block) {
        const int64_t blocks = (tiles + tiles_per_block - 1) / tiles_per_block;
        if (blocks > kMaxGridX) return DYBIT_ERR_UNSUPPORTED;
        launch_k(kernel, dim3((unsigned)blocks), dim3(kCkptThreads), 0, s, p);
        return launch_status();
    };
    // warps to a page and head: as many as hold the new tokens of one in registers
    const int vectors = most * p.vpr;
    if (vectors <= 256) return go(cache_write_kernel<T, VEC, 1>, 8);
    if (vectors <= 512) return go(cache_write_kernel<T, VEC, 2>, 4);
    if (vectors <= 1024) return go(cache_write_kernel<T, VEC, 4>, 2);
    return go(cache_write_kernel<T, VEC, 8>, 1);
}

template <typename F>
static dybit_status with_type(dybit_dtype t, bool vec, F &&f) {
    switch (t) {
        case DYBIT_F32: return vec ? f.template operator()<float, true>() : f.template operator()<float, false>();
        case DYBIT_BF16: return vec ? f.template operator()<__nv_bfloat16, true>() : f.template operator()<__nv_bfloat16, false>();
        default: return vec ? f.template operator()<__half, true>() : f.template operator()<__half, false>();
    }
}

struct CacheWriteLauncher {
    const CacheWrite &p;
    int64_t items;
    int most;
    cudaStream_t s;
    template <typename T, bool VEC> dybit_status operator()() const { return launch_cache_write<T, VEC>(p, items, most, s); }
};
struct CacheReadLauncher {
    const CacheRead &p;
    int64_t items;
    int threads;
    cudaStream_t s;
    template <typename T, bool VEC> dybit_status operator()() const {
        const int64_t blocks = items * 2 * p.heads;
        if (blocks > kMaxGridX) return DYBIT_ERR_UNSUPPORTED;
        launch_k(cache_read_kernel<T, VEC>, dim3((unsigned)blocks), dim3((unsigned)threads), 0, s, p);
        return launch_status();
    }
};

// Codes [pages * heads][page][dim] of bytes, boxes of `rows` keys x DP bytes; what lies beyond dim reads as code 0.
static bool make_cache_map(CUtensorMap *map, const void *codes, const dybit_cache *c, int rows, int dp) {
    EncodeTiledFn fn = encode_tiled_fn();
    if (fn == nullptr) return false;
    cuuint64_t dims[3] = {(cuuint64_t)c->dim, (cuuint64_t)c->page, (cuuint64_t)(c->pages * c->heads)};
    cuuint64_t strides[2] = {(cuuint64_t)c->dim, (cuuint64_t)c->dim * c->page};
    cuuint32_t box[3] = {(cuuint32_t)dp, (cuuint32_t)rows, 1}, estr[3] = {1, 1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, const_cast<void *>(codes), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              dp == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Parts of the attention's workspace: outputs and {maximum, sum, exponent} of the parts of cut tiles.
struct CacheWorkspace {
    int64_t small_y, small_ml, large_y, large_ml, plan, bytes;
    CacheWorkspace(const CacheShape &s, int dim) {
        const CachePlanLayout L(s);
        int64_t at = 0;
        small_y = at, at += round_up((L.small_cap > 0 ? 2 * small_blocks(s.small_rows) : 0) * s.small_rows * (int64_t)dim * 4, 1024);
        small_ml = at, at += round_up((L.small_cap > 0 ? 2 * small_blocks(s.small_rows) : 0) * s.small_rows * 16, 1024);
        large_y = at, at += round_up((L.large_cap > 0 ? 2 * kLargeBlocks : 0) * kLargeRows * (int64_t)dim * 4, 1024);
        large_ml = at, at += round_up((L.large_cap > 0 ? 2 * kLargeBlocks : 0) * kLargeRows * 16, 1024);
        plan = at, at += round_up(L.words * 4, 1024);      // the work dealt out again, where a call masks otherwise than the plan
        bytes = at;
    }
};

template <typename T, int DP, int NQ, int BOX>
static dybit_status launch_cache_small(const CUtensorMap &mk, const CUtensorMap &mv, const CacheAttn &p, cudaStream_t s) {
    static std::atomic<int> ready[64];
    int dev = 0;
    DYBIT_CUDA_TRY(cudaGetDevice(&dev));
    if (dev < 0 || dev >= 64) return DYBIT_ERR_CUDA;
    if (ready[dev].load(std::memory_order_acquire) == 0) {
        DYBIT_CUDA_TRY(cudaFuncSetAttribute(cache_small_kernel<T, DP, NQ, BOX>, cudaFuncAttributeMaxDynamicSharedMemorySize, small_smem(8 * NQ)));
        ready[dev].store(1, std::memory_order_release);
    }
    launch_k(cache_small_kernel<T, DP, NQ, BOX>, dim3(148), dim3(32 * small_per_sm(8 * NQ)), small_smem(8 * NQ), s, mk, mv, p);
    return launch_status();
}

// The kernel that joins parts.  It asks for the split of L1 and shared memory that the attention kernels have: an SM has to run
// empty to change it.
template <typename T, int ROWS>
static dybit_status launch_cache_join(const CacheAttn &p, dim3 grid, cudaStream_t s) {
    static std::atomic<int> ready[64];
    int dev = 0;
    DYBIT_CUDA_TRY(cudaGetDevice(&dev));
    if (dev < 0 || dev >= 64) return DYBIT_ERR_CUDA;
    if (ready[dev].load(std::memory_order_acquire) == 0) {
        DYBIT_CUDA_TRY(cudaFuncSetAttribute(cache_join_kernel<T, ROWS>, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared));
        ready[dev].store(1, std::memory_order_release);
    }
    launch_k(cache_join_kernel<T, ROWS>, grid, dim3(256), 0, s, p);
    return launch_status();
}

template <typename T, int DP>
static dybit_status launch_cache_large(const dybit_cache *c, const CacheAttn &p, cudaStream_t s) {
    static std::atomic<int> ready[64];
    int dev = 0;
    DYBIT_CUDA_TRY(cudaGetDevice(&dev));
    if (dev < 0 || dev >= 64) return DYBIT_ERR_CUDA;
    if (ready[dev].load(std::memory_order_acquire) == 0) {
        DYBIT_CUDA_TRY(cudaFuncSetAttribute(cache_large_kernel<T, DP>, cudaFuncAttributeMaxDynamicSharedMemorySize, large_smem_bytes<DP>()));
        ready[dev].store(1, std::memory_order_release);
    }
    launch_k(cache_large_kernel<T, DP>, dim3(kLargeBlocks), dim3(kLgThreads), large_smem_bytes<DP>(), s, static_cast<const uint8_t *>(c->k_codes),
             static_cast<const uint8_t *>(c->v_codes), p);
    return launch_status();
}

template <typename T>
static dybit_status run_cache_attention(const dybit_cache *c, const CacheShape &shape, CacheAttn p, uint8_t *ws, const int *plan, cudaStream_t s) {
    const CachePlanLayout L(shape);
    const CacheWorkspace w(shape, c->dim);
    const int dp = c->dim <= 64 ? 64 : 128, box = c->page == 16 ? 16 : 32;
    CUtensorMap mk, mv;
    if (!make_cache_map(&mk, c->k_codes, c, box, dp) || !make_cache_map(&mv, c->v_codes, c, box, dp)) return DYBIT_ERR_CUDA;
    dybit_status st = DYBIT_OK;
    if ((p.causal != 0) != (shape.causal != 0) || p.window != shape.window) {
        CacheShape mine = shape;
        mine.causal = p.causal, mine.window = p.window;
        launch_k(cache_deal_kernel, dim3(L.large_cap > 0 ? 2 : 1), dim3(kCachePlanThreads), 0, s, mine, plan, reinterpret_cast<int *>(ws + w.plan));
        st = launch_status();
        if (st != DYBIT_OK) return st;
        plan = reinterpret_cast<const int *>(ws + w.plan);
    }
    CacheAttn small = p, large = p;
    small.tiles = reinterpret_cast<const CacheTile *>(plan + L.small);
    small.starts = reinterpret_cast<const CacheStart *>(plan + L.small_starts);
    small.joins = reinterpret_cast<const CacheJoin *>(plan + L.small_joins);
    small.counts = plan + kPlanSmall;
    small.part_y = reinterpret_cast<float *>(ws + w.small_y);
    small.part_ml = reinterpret_cast<float4 *>(ws + w.small_ml);
    large.tiles = reinterpret_cast<const CacheTile *>(plan + L.large);
    large.starts = reinterpret_cast<const CacheStart *>(plan + L.large_starts);
    large.joins = reinterpret_cast<const CacheJoin *>(plan + L.large_joins);
    large.counts = plan + kPlanLarge;
    large.part_y = reinterpret_cast<float *>(ws + w.large_y);
    large.part_ml = reinterpret_cast<float4 *>(ws + w.large_ml);
    if (L.large_cap > 0) {
        st = dp == 64 ? launch_cache_large<T, 64>(c, large, s) : launch_cache_large<T, 128>(c, large, s);
        if (st != DYBIT_OK) return st;
        small.beside = 1;
    }
    const bool few = shape.small_rows == 8;
    auto go = [&](auto d, auto q) {
        constexpr int DP = decltype(d)::value, NQ = decltype(q)::value;
        return box == 16 ? launch_cache_small<T, DP, NQ, 16>(mk, mv, small, s) : launch_cache_small<T, DP, NQ, 32>(mk, mv, small, s);
    };
    using one = std::integral_constant<int, 1>;
    using two = std::integral_constant<int, 2>;
    using d64 = std::integral_constant<int, 64>;
    using d128 = std::integral_constant<int, 128>;
    if (L.small_cap > 0) {
        st = dp == 64 ? (few ? go(d64(), one()) : go(d64(), two())) : (few ? go(d128(), one()) : go(d128(), two()));
        if (st != DYBIT_OK) return st;
    }
    if (L.large_cap > 0) {
        st = launch_cache_join<T, kLargeRows>(large, dim3(kLargeBlocks - 1, 8), s);
        if (st != DYBIT_OK) return st;
    }
    if (L.small_cap == 0) return DYBIT_OK;
    if (few) st = launch_cache_join<T, 8>(small, dim3(4 * 148), s);
    else st = launch_cache_join<T, kSmallRows>(small, dim3(4 * 148), s);
    return st;
}

}  // namespace dybit

extern "C" {

size_t dybit_cache_plan_bytes(const dybit_cache *cache, const dybit_cache_batch *batch) {
    using namespace dybit;
    if (check_cache(cache) != DYBIT_OK || check_batch(cache, batch) != DYBIT_OK) return 0;
    return (size_t)round_up(CachePlanLayout(cache_shape(cache, batch)).words * 4, 16);
}

dybit_status dybit_cache_plan(const dybit_cache *cache, const dybit_cache_batch *batch, const int32_t *starts, const int32_t *lengths, void *plan,
                              size_t plan_bytes, void *stream) {
    using namespace dybit;
    dybit_status st = check_cache(cache);
    if (st == DYBIT_OK) st = check_batch(cache, batch);
    if (st != DYBIT_OK) return st;
    if (plan == nullptr || (batch->sequences > 0 && (starts == nullptr || lengths == nullptr))) return DYBIT_ERR_INVALID_ARG;
    if (!aligned(plan, 16) || !aligned(starts, 4) || !aligned(lengths, 4)) return DYBIT_ERR_ALIGNMENT;
    if (plan_bytes < dybit_cache_plan_bytes(cache, batch)) return DYBIT_ERR_WORKSPACE;
    const CachePlanArgs a = {cache_shape(cache, batch), starts, lengths, static_cast<int *>(plan)};
    launch_k(cache_plan_kernel, dim3(1), dim3(kCachePlanThreads), 0, static_cast<cudaStream_t>(stream), a);
    return launch_status();
}

dybit_status dybit_cache_write(const dybit_cache *cache, const dybit_cache_batch *batch, const void *plan, const void *k, int64_t k_token_stride,
                               int64_t k_head_stride, const void *v, int64_t v_token_stride, int64_t v_head_stride, dybit_dtype t, int top,
                               void *stream) {
    using namespace dybit;
    dybit_status st = check_plan(cache, batch, plan);
    if (st != DYBIT_OK) return st;
    if (!dtype_ok(t) || top < 0 || top > 6) return DYBIT_ERR_INVALID_ARG;
    if (batch->tokens == 0 || batch->sequences == 0 || batch->max_new == 0) return DYBIT_OK;
    st = check_heads(k, t, k_token_stride, k_head_stride, batch->tokens, cache->heads, cache->dim);
    if (st == DYBIT_OK) st = check_heads(v, t, v_token_stride, v_head_stride, batch->tokens, cache->heads, cache->dim);
    if (st != DYBIT_OK) return st;
    const CacheShape shape = cache_shape(cache, batch);
    const CachePlanLayout L(shape);
    const int *words = static_cast<const int *>(plan);
    CacheWrite p = {};
    p.plan = words, p.items = reinterpret_cast<const CacheItem *>(words + L.items);
    p.table = batch->table, p.table_stride = batch->table_stride;
    p.pages = cache->pages, p.page = cache->page, p.heads = cache->heads, p.dim = cache->dim;
    p.vpr = cache->dim * dtype_bytes(t) / 16, p.vpr_mul = ((1 << 20) + p.vpr - 1) / p.vpr;
    p.x[0] = k, p.x[1] = v;
    p.token_stride[0] = k_token_stride, p.token_stride[1] = v_token_stride;
    p.head_stride[0] = k_head_stride, p.head_stride[1] = v_head_stride;
    p.codes[0] = static_cast<uint8_t *>(cache->k_codes), p.codes[1] = static_cast<uint8_t *>(cache->v_codes);
    p.scales[0] = cache->k_scales, p.scales[1] = cache->v_scales;
    p.top = top;
    const bool vec = heads_aligned(k, t, k_token_stride, k_head_stride, 16) && heads_aligned(v, t, v_token_stride, v_head_stride, 16);
    return with_type(t, vec, CacheWriteLauncher{p, L.items_cap, std::min(cache->page, shape.max_new), static_cast<cudaStream_t>(stream)});
}

dybit_status dybit_cache_read(const dybit_cache *cache, const dybit_cache_batch *batch, const void *plan, void *k, int64_t k_token_stride,
                              int64_t k_head_stride, void *v, int64_t v_token_stride, int64_t v_head_stride, dybit_dtype t, void *stream) {
    using namespace dybit;
    dybit_status st = check_plan(cache, batch, plan);
    if (st != DYBIT_OK) return st;
    if (!dtype_ok(t)) return DYBIT_ERR_INVALID_ARG;
    if (batch->tokens == 0 || batch->sequences == 0 || batch->max_new == 0) return DYBIT_OK;
    st = check_heads(k, t, k_token_stride, k_head_stride, batch->tokens, cache->heads, cache->dim);
    if (st == DYBIT_OK) st = check_heads(v, t, v_token_stride, v_head_stride, batch->tokens, cache->heads, cache->dim);
    if (st != DYBIT_OK) return st;
    const CacheShape shape = cache_shape(cache, batch);
    const CachePlanLayout L(shape);
    const int *words = static_cast<const int *>(plan);
    CacheRead p = {};
    p.plan = words, p.items = reinterpret_cast<const CacheItem *>(words + L.items);
    p.table = batch->table, p.table_stride = batch->table_stride;
    p.pages = cache->pages, p.page = cache->page, p.heads = cache->heads, p.dim = cache->dim;
    p.vpr = cache->dim * dtype_bytes(t) / 16, p.vpr_mul = ((1 << 20) + p.vpr - 1) / p.vpr;
    p.y[0] = k, p.y[1] = v, p.tokens = batch->tokens;
    p.token_stride[0] = k_token_stride, p.token_stride[1] = v_token_stride;
    p.head_stride[0] = k_head_stride, p.head_stride[1] = v_head_stride;
    p.codes[0] = static_cast<const uint8_t *>(cache->k_codes), p.codes[1] = static_cast<const uint8_t *>(cache->v_codes);
    p.scales[0] = cache->k_scales, p.scales[1] = cache->v_scales;
    const bool vec = heads_aligned(k, t, k_token_stride, k_head_stride, 16) && heads_aligned(v, t, v_token_stride, v_head_stride, 16);
    const int vectors = std::min(cache->page, shape.max_new) * p.vpr, threads = (int)std::min<int64_t>(kCkptThreads, round_up((vectors + 3) / 4, 32));
    return with_type(t, vec, CacheReadLauncher{p, L.items_cap, threads, static_cast<cudaStream_t>(stream)});
}

size_t dybit_cache_attention_workspace_bytes(const dybit_cache *cache, const dybit_cache_batch *batch) {
    using namespace dybit;
    if (check_cache(cache) != DYBIT_OK || check_batch(cache, batch) != DYBIT_OK) return 0;
    return (size_t)CacheWorkspace(cache_shape(cache, batch), cache->dim).bytes;
}

dybit_status dybit_cache_attention(const dybit_cache *cache, const dybit_cache_batch *batch, const void *plan, const void *q, dybit_dtype t,
                                   int64_t q_token_stride, int64_t q_head_stride, void *y, int64_t y_token_stride, int64_t y_head_stride, float *lse,
                                   float scale, int causal, int window, void *ws, size_t ws_bytes, void *stream) {
    using namespace dybit;
    dybit_status st = check_plan(cache, batch, plan);
    if (st != DYBIT_OK) return st;
    if (!dtype_ok(t) || window < 0 || (window > 0 && !causal) || !(scale >= 0.0f) || scale > 2.0e38f) return DYBIT_ERR_INVALID_ARG;
    if (t == DYBIT_F32) return DYBIT_ERR_UNSUPPORTED;
    if (batch->tokens == 0 || batch->sequences == 0 || batch->max_new == 0) return DYBIT_OK;
    st = check_heads(q, t, q_token_stride, q_head_stride, batch->tokens, batch->q_heads, cache->dim);
    if (st == DYBIT_OK) st = check_heads(y, t, y_token_stride, y_head_stride, batch->tokens, batch->q_heads, cache->dim);
    if (st != DYBIT_OK) return st;
    if (!aligned(lse, 4) || !aligned(ws, 1024)) return DYBIT_ERR_ALIGNMENT;
    if (ws == nullptr || ws_bytes < dybit_cache_attention_workspace_bytes(cache, batch)) return DYBIT_ERR_WORKSPACE;
    if (cache->pages == 0) return DYBIT_ERR_INVALID_ARG;
    CacheAttn p = {};
    p.table = batch->table, p.table_stride = batch->table_stride;
    p.pages = cache->pages, p.page_shift = log2_of(cache->page), p.heads = cache->heads, p.group = batch->q_heads / cache->heads, p.dim = cache->dim;
    p.k_scales = cache->k_scales, p.v_scales = cache->v_scales;
    p.q = q, p.q_token = q_token_stride, p.q_head = q_head_stride;
    p.y = y, p.y_token = y_token_stride, p.y_head = y_head_stride;
    p.lse = lse, p.tokens = batch->tokens;
    p.scale_log2 = scale * kLog2e;
    p.causal = causal != 0, p.window = window_or_none(window);
    p.q_vec = heads_aligned(q, t, q_token_stride, q_head_stride, 8), p.q_vec16 = heads_aligned(q, t, q_token_stride, q_head_stride, 16);
    p.y_vec = heads_aligned(y, t, y_token_stride, y_head_stride, 8), p.y_vec16 = heads_aligned(y, t, y_token_stride, y_head_stride, 16);
    const CacheShape shape = cache_shape(cache, batch);
    uint8_t *base = static_cast<uint8_t *>(ws);
    const int *words = static_cast<const int *>(plan);
    if (t == DYBIT_BF16) return run_cache_attention<__nv_bfloat16>(cache, shape, p, base, words, static_cast<cudaStream_t>(stream));
    return run_cache_attention<__half>(cache, shape, p, base, words, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
