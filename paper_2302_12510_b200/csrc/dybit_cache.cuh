// Key-value cache in signed 8-bit codes: its layout, the plan of a batch, the write of new tokens and the read-back.
//
// A pool of pages; a page holds `page` consecutive tokens of one sequence, head by head: codes
// [pages][heads][page][dim], so the tokens of one page and head are one run of bytes that the attention kernels fetch as
// they lie.  Keys and values have one power-of-two scale each per page and head: value = scale * value(code), and the
// scale 0 stands for a block in which every value is 0.
#pragma once

#include "dybit_row8.cuh"

namespace dybit {

// Barrier of the TPR threads that share tile `sub` of a block.
template <int TPR>
__device__ __forceinline__ void named_tile_sync(int sub) {
    asm volatile("bar.sync %0, %1;" ::"r"(1 + sub), "n"(TPR) : "memory");
}

constexpr int kCachePlanThreads = 1024;
constexpr int kSmallRows = 16;               // query rows (token x query head of one key head) of a small tile at most; half of them
                                             // where no sequence of the batch has more
constexpr int kLargeRows = 256;              // rows of a large tile: two accumulators of 128
constexpr int kSmallUnit = 64, kLargeUnit = 128;     // keys in which a split of the key axis is counted
// CTAs that the key axis is cut for.  Counted as the B200 has them, not asked of the device: the sizes of plans and
// workspaces depend on them and are the same wherever they are asked for.
constexpr int kSmallTarget = 148 * 3 * 2, kLargeTarget = 148;
constexpr int kSmallLeast = 4, kLargeLeast = 8;      // units that a split has at least

// New tokens of one sequence that go to one page (page < 0 for tokens in front of the sequence's first position).
struct CacheItem { int row, pos, count, seq; };
// A tile of query rows of one sequence, and one of the parts that its keys are cut into.
struct CacheTile { int row, n, len, seq, tile, split, splits, slot; };
// What one thread of the plan kernel knows of a sequence.
struct CacheSeq { int row, n, len, items, small_tiles, large_tiles; };

struct CacheShape {
    int64_t T;
    int B, page, heads, group, max_new, max_pages;
    int small_tokens;            // a sequence with more new tokens than this takes large tiles
    int small_rows;              // of a small tile: 8 or kSmallRows
};

// Word offsets of a plan's parts; the capacities bound what the device fills in.
struct CachePlanLayout {
    int64_t items_cap, small_cap, large_cap, small_slots, large_slots, small_comb_cap, large_comb_cap;
    int64_t items, small, large, small_comb, large_comb, words;
    __host__ __device__ static int64_t lesser(int64_t a, int64_t b) { return a < b ? a : b; }
    __host__ __device__ explicit CachePlanLayout(const CacheShape &s) {
        const int64_t T = s.T, B = s.B;
        items_cap = lesser(T, T / s.page + 3 * B);
        // new tokens that small tiles take: all of a sequence of at most small_tokens
        const int64_t few = s.small_tokens >= s.max_new ? T : lesser(T, B * (int64_t)s.small_tokens);
        const int64_t small_tiles = lesser(few * s.group, few * s.group / s.small_rows + B);
        const int64_t large_tiles = s.max_new > s.small_tokens ? lesser(T, T * s.group / kLargeRows + B) : 0;
        const int64_t small_parts = kSmallTarget / s.heads + 1, large_parts = kLargeTarget / s.heads + 1;
        small_cap = small_tiles + small_parts;
        large_cap = large_tiles > 0 ? large_tiles + large_parts : 0;
        small_slots = 2 * small_parts;
        large_slots = large_tiles > 0 ? 2 * large_parts : 0;
        small_comb_cap = lesser(small_tiles, small_parts);
        large_comb_cap = large_tiles > 0 ? lesser(large_tiles, large_parts) : 0;
        int64_t w = 16;                                  // counts: items, small, large, small_comb, large_comb; the rest spare
        items = w, w += 4 * items_cap;
        small = w, w += 8 * small_cap;
        large = w, w += 8 * large_cap;
        small_comb = w, w += 8 * small_comb_cap;
        large_comb = w, w += 8 * large_comb_cap;
        words = w;
    }
};

struct CachePlanArgs {
    CacheShape s;
    const int *starts, *lengths;
    int *plan;
};

__device__ __forceinline__ int cache_div_up(int a, int b) { return (a + b - 1) / b; }

__device__ __forceinline__ CacheSeq cache_seq(const CachePlanArgs &a, int b) {
    CacheSeq q;
    const int T = (int)a.s.T;
    const int lo = min(max(a.starts[b], 0), T), hi = min(max(a.starts[b + 1], lo), T);
    q.row = lo;
    q.n = min(hi - lo, a.s.max_new);
    q.len = (int)min((int64_t)max(a.lengths[b], 0), (int64_t)a.s.max_pages * a.s.page);
    const int outside = max(0, q.n - q.len), inside = q.n - outside, p0 = q.len - inside;
    q.items = cache_div_up(outside, a.s.page) + (inside > 0 ? (q.len - 1) / a.s.page - p0 / a.s.page + 1 : 0);
    const int rows = q.n * a.s.group;
    const bool small = q.n <= a.s.small_tokens;
    q.small_tiles = small ? cache_div_up(rows, a.s.small_rows) : 0;
    q.large_tiles = small ? 0 : cache_div_up(rows, kLargeRows);
    return q;
}

// Units of keys that a sequence's tiles are counted with; one at least, so that a tile without keys has a part that
// writes its zeros.
__device__ __forceinline__ int cache_units(int len, int unit) { return max(1, cache_div_up(len, unit)); }

// Sum over the block, the same for all threads.
__device__ __forceinline__ int64_t cache_block_sum(int64_t v, int64_t *s_warp) {
    for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) s_warp[threadIdx.x >> 5] = v;
    __syncthreads();
    int64_t all = 0;
    for (int w = 0; w < kCachePlanThreads / 32; ++w) all += s_warp[w];
    return all;
}

// Exclusive prefix sum over the block; *total receives the sum.
__device__ __forceinline__ int cache_block_scan(int v, int *s_warp, int *total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int sum = v;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int o = __shfl_up_sync(0xffffffffu, sum, d);
        if (lane >= d) sum += o;
    }
    __syncthreads();
    if (lane == 31) s_warp[warp] = sum;
    __syncthreads();
    const int mine = s_warp[lane], before = __reduce_add_sync(0xffffffffu, lane < warp ? mine : 0);
    *total = __reduce_add_sync(0xffffffffu, mine);
    return before + sum - v;
}

// One block.  The lists' capacities hold for starts that never decrease; entries beyond them (starts that do) are dropped,
// not written.  Integer work of B sequences: counts, the lengths of the parts, then the lists, a warp to a sequence.
__global__ void __launch_bounds__(kCachePlanThreads) cache_plan_kernel(const CachePlanArgs a) {
    __shared__ int64_t s_sum[kCachePlanThreads / 32];
    __shared__ int s_scan[kCachePlanThreads / 32];
    pdl_enter();
    const CachePlanLayout L(a.s);
    const int B = a.s.B, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int64_t small_units = 0, large_units = 0;
    for (int b = threadIdx.x; b < B; b += kCachePlanThreads) {
        const CacheSeq q = cache_seq(a, b);
        small_units += (int64_t)q.small_tiles * cache_units(q.len, kSmallUnit);
        large_units += (int64_t)q.large_tiles * cache_units(q.len, kLargeUnit);
    }
    small_units = cache_block_sum(small_units, s_sum);
    large_units = cache_block_sum(large_units, s_sum);
    // units of a part: the whole work over the CTAs that are to have some
    auto part = [&](int64_t units, int target, int least) {
        const int64_t parts = target / a.s.heads + 1;
        return (int)min((int64_t)1 << 30, max((int64_t)least, (units + parts - 1) / parts));
    };
    const int small_part = part(small_units, kSmallTarget, kSmallLeast), large_part = part(large_units, kLargeTarget, kLargeLeast);
    int at[7] = {0, 0, 0, 0, 0, 0, 0};                    // items, small, large, small_comb, large_comb, slots of small and large
    for (int b0 = 0; b0 < B; b0 += kCachePlanThreads) {
        const int b = b0 + threadIdx.x;
        CacheSeq q = {};
        if (b < B) q = cache_seq(a, b);
        const int sp = cache_div_up(cache_units(q.len, kSmallUnit), small_part), lp = cache_div_up(cache_units(q.len, kLargeUnit), large_part);
        const int count[7] = {q.items, q.small_tiles * sp, q.large_tiles * lp, sp > 1 ? q.small_tiles : 0, lp > 1 ? q.large_tiles : 0,
                              sp > 1 ? q.small_tiles * sp : 0, lp > 1 ? q.large_tiles * lp : 0};
        int first[7];
#pragma unroll
        for (int c = 0; c < 7; ++c) {
            int total;
            first[c] = at[c] + cache_block_scan(count[c], s_scan, &total);
            at[c] += total;
        }
        // the lists of these sequences, a warp to a sequence: lane k of the warp has what was counted for sequence k of its own
        for (int k = 0; k < 32; ++k) {
            const int seq = b0 + warp * 32 + k;
            if (seq >= B) break;
            auto of = [&](int v) { return __shfl_sync(0xffffffffu, v, k); };
            const int row = of(q.row), n = of(q.n), len = of(q.len), items = of(q.items), page = a.s.page;
            const int outside = max(0, n - len), p0 = len - (n - outside), out_items = cache_div_up(outside, page), i0 = of(first[0]);
            CacheItem *list = reinterpret_cast<CacheItem *>(a.plan + L.items) + i0;
            for (int i = lane; i < items; i += 32) {
                CacheItem it;
                if (i < out_items) {
                    it = {row + i * page, -1, min(page, outside - i * page), seq};
                } else {
                    const int j = p0 / page + (i - out_items), lo = max(p0, j * page), hi = (int)min((int64_t)len, (int64_t)(j + 1) * page);
                    it = {row + outside + lo - p0, lo, hi - lo, seq};
                }
                if ((unsigned)(i0 + i) < (uint64_t)L.items_cap) list[i] = it;
            }
            auto tiles = [&](int64_t list_at, int64_t cap, int64_t comb_at, int64_t comb_cap, int n_tiles, int parts, int t0, int c0, int slot0) {
                CacheTile *out = reinterpret_cast<CacheTile *>(a.plan + list_at) + t0, *comb = reinterpret_cast<CacheTile *>(a.plan + comb_at) + c0;
                for (int i = lane; i < n_tiles * parts; i += 32) {
                    // the last tile sees the most keys under a causal mask: it comes first
                    const int j = i / parts, split = i - j * parts, slot = parts > 1 ? slot0 + j * parts : -1;
                    const CacheTile t = {row, n, len, seq, n_tiles - 1 - j, split, parts, slot < 0 ? slot : slot + split};
                    if ((unsigned)(t0 + i) < (uint64_t)cap) out[i] = t;
                    if (split == 0 && parts > 1 && (unsigned)(c0 + j) < (uint64_t)comb_cap) comb[j] = t;
                }
            };
            tiles(L.small, L.small_cap, L.small_comb, L.small_comb_cap, of(q.small_tiles), of(sp), of(first[1]), of(first[3]), of(first[5]));
            tiles(L.large, L.large_cap, L.large_comb, L.large_comb_cap, of(q.large_tiles), of(lp), of(first[2]), of(first[4]), of(first[6]));
        }
    }
    if (threadIdx.x == 0) {
        const int64_t caps[5] = {L.items_cap, L.small_cap, L.large_cap, L.small_comb_cap, L.large_comb_cap};
#pragma unroll
        for (int c = 0; c < 5; ++c) a.plan[c] = (unsigned)at[c] < (uint64_t)caps[c] ? at[c] : (int)caps[c];
    }
}

// ------------------------------------------------------------------ write

struct CacheWrite {
    const int *plan;             // counts
    const CacheItem *items;
    const int *table;
    int64_t table_stride;
    int64_t pages;
    int page, heads, dim;
    int vpr, vpr_mul;            // 16-byte vectors of a row; i / vpr = i * vpr_mul >> 20 for i < 4096
    const void *x[2];            // keys, values
    int64_t token_stride[2], head_stride[2];
    uint8_t *codes[2];
    float *scales[2];
    int top;
};

// The page that holds position `pos` of a sequence, or -1.
__device__ __forceinline__ int64_t cache_page(const int *table, int64_t stride, int seq, int pos, int page, int64_t pages) {
    if (pos < 0) return -1;
    const int p = __ldg(table + seq * stride + pos / page);
    return (unsigned)p < (uint64_t)pages ? p : -1;
}

// W warps take the new tokens of one page and head, of the keys or of the values.  What fits 8 vectors per thread stays
// in registers between the maximum and the codes; the rest is read twice, the second time from the caches.
//   scale = the larger of what the page has and 2^(ceil(log2 amax) - top) of the new tokens
// Where a begun page's scale grows, its older codes are rounded once more at the new scale, a larger power of two.
template <typename T, bool VEC, int W>
__global__ void __launch_bounds__(kCkptThreads) cache_write_kernel(const CacheWrite p) {
    constexpr int E = 16 / (int)sizeof(T), NV = 8, TPR = W * 32;
    __shared__ unsigned s_best[8];
    pdl_enter();
    const int sub = threadIdx.x / TPR, t = threadIdx.x % TPR;
    const int64_t tile = (int64_t)blockIdx.x * (8 / W) + sub;
    const int item = (int)(tile / (2 * p.heads)), pair = (int)(tile - (int64_t)item * (2 * p.heads));
    if (item >= p.plan[0]) return;                         // all the warps of a tile
    const int kv = pair >= p.heads ? 1 : 0, head = pair - kv * p.heads;
    const CacheItem it = p.items[item];
    const int64_t page = cache_page(p.table, p.table_stride, it.seq, it.pos, p.page, p.pages);
    if (page < 0) return;
    const int off = it.pos & (p.page - 1), n_vec = it.count * p.vpr;
    const T *x = static_cast<const T *>(p.x[kv]) + it.row * p.token_stride[kv] + head * p.head_stride[kv];
    float *const scale_at = p.scales[kv] + page * p.heads + head;
    uint8_t *const block = p.codes[kv] + (page * p.heads + head) * ((int64_t)p.page * p.dim);
    auto load = [&](int i) {
        const int row = (int)(((unsigned)i * (unsigned)p.vpr_mul) >> 20), c = i - row * p.vpr;
        return load_row_vec<T, VEC>(x + row * p.token_stride[kv], c * E, p.dim);
    };
    uint4 v[NV];
    unsigned best = 0u;
#pragma unroll
    for (int i = 0; i < NV; ++i) v[i] = i * TPR + t < n_vec ? load(i * TPR + t) : make_uint4(0u, 0u, 0u, 0u);
    const float old = off > 0 ? *scale_at : 0.0f;
#pragma unroll
    for (int i = 0; i < NV; ++i) best = vec_absmax<T>(v[i], best);
    for (int i = NV * TPR + t; i < n_vec; i += TPR) best = vec_absmax<T>(load(i), best);
    best = absmax_as_f32<T>(best);
    auto block_max = [&](unsigned b) {
        b = __reduce_max_sync(0xffffffffu, b);
        if constexpr (W > 1) {
            if ((threadIdx.x & 31) == 0) s_best[threadIdx.x >> 5] = b;
            named_tile_sync<TPR>(sub);
#pragma unroll
            for (int w = 0; w < W; ++w) b = max(b, s_best[sub * W + w]);
        }
        return b;
    };
    best = block_max(best);
    const bool special = best >= 0x7f800000u;              // infinities or NaN: the maximum of the finite elements instead
    if (special) {
        float finite = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i) finite = vec_absmax_finite<T>(v[i], finite);
        for (int i = NV * TPR + t; i < n_vec; i += TPR) finite = vec_absmax_finite<T>(load(i), finite);
        if constexpr (W > 1) named_tile_sync<TPR>(sub);    // s_best is free again
        best = block_max(__float_as_uint(finite));
    }
    float scale = 0.0f, inv = 0.0f;
    if (best != 0u) pow2_scale(best, p.top, &scale, &inv);
    const bool grown = scale > old;
    if (!grown) {
        scale = old;
        inv = old > 0.0f ? __fdiv_rn(1.0f, old) : 0.0f;    // exact for a power of two
    }
    uint8_t *out = block + off * p.dim;
    auto store = [&](const uint4 &w, int i) {
        if (!DYBIT_CHECK((off + it.count) * p.dim <= p.page * p.dim && i * E < it.count * p.dim, 0x85)) return;
        if (special) store_vec_codes<T, true, true>(w, inv, out + i * E);
        else store_vec_codes<T, true, false>(w, inv, out + i * E);
    };
#pragma unroll
    for (int i = 0; i < NV; ++i)
        if (i * TPR + t < n_vec) store(v[i], i * TPR + t);
    for (int i = NV * TPR + t; i < n_vec; i += TPR) store(load(i), i);
    if (grown) {
        const float ratio = __fmul_rn(old, inv);           // a power of two of at most 1/2, or 0
        for (int i = t; i < off * p.dim / 16; i += TPR) {
            uint4 *at = reinterpret_cast<uint4 *>(block) + i;
            const uint4 c = *at;
            *at = make_uint4(encode4_8<true, false>(decode4<true>(c.x), ratio), encode4_8<true, false>(decode4<true>(c.y), ratio),
                             encode4_8<true, false>(decode4<true>(c.z), ratio), encode4_8<true, false>(decode4<true>(c.w), ratio));
        }
    }
    if (W > 1) named_tile_sync<TPR>(sub);                  // every thread of the tile has read the old scale
    if (t == 0 && (grown || off == 0)) *scale_at = scale;
}

// ------------------------------------------------------------------ read

struct CacheRead {
    const int *plan;
    const CacheItem *items;
    const int *table;
    int64_t table_stride;
    int64_t pages;
    int page, heads, dim;
    int vpr, vpr_mul;
    void *y[2];
    int64_t token_stride[2], head_stride[2];
    const uint8_t *codes[2];
    const float *scales[2];
};

// A block per page and head, of the keys or of the values: codes are fetched four vectors ahead, one vector of
// output each.  Tokens on pages that are not there read as zeros.
template <typename T, bool VEC>
__global__ void __launch_bounds__(kCkptThreads) cache_read_kernel(const CacheRead p) {
    constexpr int E = 16 / (int)sizeof(T), NV = 4;
    pdl_enter();
    const int item = (int)(blockIdx.x / (unsigned)(2 * p.heads)), pair = (int)(blockIdx.x - (unsigned)item * (2 * p.heads));
    if (item >= p.plan[0]) return;
    const int kv = pair >= p.heads ? 1 : 0, head = pair - kv * p.heads;
    const CacheItem it = p.items[item];
    const int64_t page = cache_page(p.table, p.table_stride, it.seq, it.pos, p.page, p.pages);
    const int n_vec = it.count * p.vpr;
    T *y = static_cast<T *>(p.y[kv]) + it.row * p.token_stride[kv] + head * p.head_stride[kv];
    const uint8_t *in = page < 0 ? nullptr : p.codes[kv] + ((page * p.heads + head) * p.page + (it.pos & (p.page - 1))) * (int64_t)p.dim;
    const float scale = page < 0 ? 0.0f : __ldg(p.scales[kv] + page * p.heads + head);
    for (int i0 = threadIdx.x; i0 < n_vec; i0 += NV * (int)blockDim.x) {
        uint2 w[NV];
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int i = i0 + j * (int)blockDim.x;
            w[j] = make_uint2(0u, 0u);
            if (i < n_vec && in != nullptr) {
                if constexpr (E == 4) w[j].x = __ldg(reinterpret_cast<const unsigned *>(in + i * E));
                else w[j] = __ldg(reinterpret_cast<const uint2 *>(in + i * E));
            }
        }
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int i = i0 + j * (int)blockDim.x;
            if (i >= n_vec) break;
            const int row = (int)(((unsigned)i * (unsigned)p.vpr_mul) >> 20), c = (i - row * p.vpr) * E;
            float f[E];
#pragma unroll
            for (int h = 0; h < E / 4; ++h) {
                const float4 d = decode4<true>(h == 0 ? w[j].x : w[j].y);
                f[4 * h] = __fmul_rn(d.x, scale), f[4 * h + 1] = __fmul_rn(d.y, scale);
                f[4 * h + 2] = __fmul_rn(d.z, scale), f[4 * h + 3] = __fmul_rn(d.w, scale);
            }
            T *dst = y + row * p.token_stride[kv] + c;
            if (!DYBIT_CHECK(c + E <= p.dim && row < it.count, 0x86)) continue;
            if constexpr (VEC) {
                uint4 o;
                if constexpr (E == 4) {
                    o = make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
                } else {
                    o = make_uint4(pack2<T>(f[0], f[1]), pack2<T>(f[2], f[3]), pack2<T>(f[4], f[5]), pack2<T>(f[6], f[7]));
                }
                *reinterpret_cast<uint4 *>(dst) = o;
            } else {
#pragma unroll
                for (int h = 0; h < E; ++h) dst[h] = from_f32<T>(f[h]);
            }
        }
    }
}

}  // namespace dybit
