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
constexpr int kSmallUnit = 64, kLargeUnit = 128;     // keys that work is counted in
// Blocks that the work of small and of large tiles is dealt out to: one resident wave.  Counted as the B200 has them, not asked of
// the device: the sizes of plans and workspaces depend on them and are the same wherever they are asked for.
constexpr int kLargeBlocks = 148;
// Small tiles' blocks are warps, as many to an SM as its registers hold.
__host__ __device__ constexpr int small_per_sm(int rows) { return rows == 8 ? 16 : 12; }
__host__ __device__ constexpr int small_blocks(int rows) { return 148 * small_per_sm(rows); }
// Units that a block has at least.  Fewer are no faster (4096 keys of one request, 1, 2 and 4 units of small tiles: 19.6, 19.7 and
// 26.4 us; four prompts of 300 tokens, 2, 4 and 8 units of large ones: 56, 56 and 63 us) and leave more parts to join.
constexpr int kSmallLeast = 2, kLargeLeast = 4;
// What a tile costs beside its keys, in units (none counted: 64 requests of 4000 keys 126.7 us, one unit 123.0).
constexpr int kTileUnits = 1;

// New tokens of one sequence that go to one page (pos < 0 for tokens in front of the sequence's first position).
struct CacheItem { int row, pos, count, seq; };
// A tile of query rows of one sequence: its number, its work and that of the tiles before it, in units, for each head.
struct CacheTile { int row, n, len, seq, tile, units; int64_t first; };
// Where a block starts in the work of all tiles and heads, head by head: `off` units into a tile, which it has a copy of.
struct CacheStart {
    int tile, head, off, pad;
    CacheTile t;
};
// A tile and head that several blocks work on: the first block that starts inside it, and the parts.
struct CacheJoin {
    CacheTile t;
    int head, first, parts, pad;
};
// What one thread of the plan kernel knows of a sequence.
struct CacheSeq { int row, n, len, items, small_tiles, large_tiles; };

struct CacheShape {
    int64_t T;
    int B, page, heads, group, max_new, max_pages;
    int small_tokens;            // a sequence with more new tokens than this takes large tiles
    int small_rows;              // of a small tile: 8 or kSmallRows
    int causal, window;          // how the calls mask; window INT_MAX for none
};

// Word offsets of a plan's parts; the capacities bound what the device fills in.
struct CachePlanLayout {
    int64_t items_cap, small_cap, large_cap;
    int64_t items, small, large, small_starts, large_starts, small_joins, large_joins, words;
    __host__ __device__ static int64_t lesser(int64_t a, int64_t b) { return a < b ? a : b; }
    __host__ __device__ explicit CachePlanLayout(const CacheShape &s) {
        const int64_t T = s.T, B = s.B;
        items_cap = lesser(T, T / s.page + 3 * B);
        // new tokens that small tiles take: all of a sequence of at most small_tokens
        const int64_t few = s.small_tokens >= s.max_new ? T : lesser(T, B * (int64_t)s.small_tokens);
        small_cap = lesser(few * s.group, few * s.group / s.small_rows + B);
        large_cap = s.max_new > s.small_tokens ? lesser(T, T * s.group / kLargeRows + B) : 0;
        int64_t w = 16;                                  // counts: items; tiles, blocks and joins, of small and of large; the rest spare
        items = w, w += 4 * items_cap;
        small = w, w += 8 * small_cap;
        large = w, w += 8 * large_cap;
        small_starts = w, w += 12 * (small_blocks(s.small_rows) + 1);
        large_starts = w, w += large_cap > 0 ? 12 * (kLargeBlocks + 1) : 0;
        small_joins = w, w += 12 * (small_blocks(s.small_rows) - 1);
        large_joins = w, w += large_cap > 0 ? 12 * (kLargeBlocks - 1) : 0;
        words = w;
    }
};

constexpr int kPlanSmall = 1, kPlanLarge = 5;        // where a plan has their four counts
// Joins of more parts than these are listed from the end of the list: a block to a row instead of a warp (one request of 65,000 keys).
constexpr int kFewParts = 8;

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
    // Tokens beyond max_new, or beyond the table's last page, are left out as if the sequence ended in front of them: its other
    // tokens keep their positions.  (len may then be negative, where every row that is left lies in front of position 0.)
    const int len = max(a.lengths[b], 0);
    const int beyond = min(hi - lo, max(hi - lo - a.s.max_new, max(0, len - a.s.max_pages * a.s.page)));
    q.row = lo;
    q.n = hi - lo - beyond;
    q.len = len - beyond;
    const int outside = min(q.n, max(0, q.n - q.len)), inside = q.n - outside, p0 = q.len - inside;
    q.items = cache_div_up(outside, a.s.page) + (inside > 0 ? (q.len - 1) / a.s.page - p0 / a.s.page + 1 : 0);
    const int rows = q.n * a.s.group;
    const bool small = q.n <= a.s.small_tokens;
    q.small_tiles = small ? cache_div_up(rows, a.s.small_rows) : 0;
    q.large_tiles = small ? 0 : cache_div_up(rows, kLargeRows);
    return q;
}

// Units of work of a tile's rows r0 .. r0 + rows - 1: its keys under the mask that is expected; one at least, so that a tile
// without keys has a block that writes its zeros.
__device__ __forceinline__ int cache_units(const CacheShape &s, const CacheSeq &q, int r0, int rows, int unit) {
    if (!s.causal) return max(1, cache_div_up(q.len, unit)) + kTileUnits;
    const int p0 = q.len - q.n, lo = max(0, p0 + r0 / s.group + 1 - min(s.window, 0x3fffffff)), hi = p0 + min(q.n - 1, (r0 + rows - 1) / s.group) + 1;
    return (hi <= lo ? 1 : cache_div_up(hi, unit) - lo / unit) + kTileUnits;
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

// Shared memory of the kernels that are one block.
constexpr int kDealTiles = 2048;             // tiles whose prefix sums are searched in shared memory; more are searched in the plan
union CachePlanShared {
    struct { CacheSeq q; int first[3]; } seqs[kCachePlanThreads];
    struct {
        int64_t first[kDealTiles];
        short head[small_blocks(8) + 1];
        int tile[small_blocks(8) + 1], off[small_blocks(8) + 1];
    } deal;
};

// One block.  The work of n tiles, for each head, dealt out evenly: `out` gets the tiles with their work, and with what comes before
// them, under the shape's mask.  counts: tiles, blocks that have some work, joins of few parts and of many.
__device__ __forceinline__ void cache_deal(const CacheShape &s, const CacheTile *tiles, CacheTile *out, int n, CacheStart *starts, CacheJoin *joins, bool large,
                                           int *counts, int *s_scan, CachePlanShared &sh) {
    const int rows = large ? kLargeRows : s.small_rows, unit = large ? kLargeUnit : kSmallUnit;
    int64_t units = 0;
    for (int i0 = 0; i0 < n; i0 += kCachePlanThreads) {
        const int i = i0 + threadIdx.x;
        CacheTile t = {};
        if (i < n) {
            t = tiles[i];
            const CacheSeq q = {t.row, t.n, t.len, 0, 0, 0};
            t.units = cache_units(s, q, t.tile * rows, rows, unit);
        }
        int total;
        t.first = units + cache_block_scan(t.units, s_scan, &total);
        if (i < n) out[i] = t;
        if (i < n && i < kDealTiles) sh.deal.first[i] = t.first;
        units += total;
    }
    __syncthreads();
    if (n == 0) {
        if (threadIdx.x == 0) counts[0] = counts[1] = counts[2] = counts[3] = 0;
        return;
    }
    const int64_t work = units * s.heads;
    const int blocks = (int)min((int64_t)(large ? kLargeBlocks : small_blocks(s.small_rows)), max((int64_t)1, work / (large ? kLargeLeast : kSmallLeast)));
    for (int c = threadIdx.x; c <= blocks; c += kCachePlanThreads) {
        const int64_t g = c < blocks ? work / blocks * c + work % blocks * c / blocks : work;
        const int head = (int)(g / units);
        const int64_t r = g - (int64_t)head * units;
        int lo = 0, hi = n - 1;                            // the last tile whose work starts at or before r
        while (lo < hi) {
            const int mid = (lo + hi + 1) / 2;
            if ((n <= kDealTiles ? sh.deal.first[mid] : out[mid].first) <= r) lo = mid;
            else hi = mid - 1;
        }
        const CacheTile t = out[lo];
        const int off = (int)(r - t.first);
        if (DYBIT_CHECK(c <= (large ? kLargeBlocks : small_blocks(s.small_rows)) && head <= s.heads, 0x8b)) starts[c] = {lo, head, off, 0, t};
        sh.deal.tile[c] = lo, sh.deal.head[c] = (short)head, sh.deal.off[c] = off;
    }
    __syncthreads();
    int n_joins[2] = {0, 0};
    const int last = (large ? kLargeBlocks : small_blocks(s.small_rows)) - 2;
    for (int c0 = 1; c0 < blocks; c0 += kCachePlanThreads) {
        const int c = c0 + threadIdx.x;
        int parts = 0;
        auto same = [&](int i) { return sh.deal.tile[i] == sh.deal.tile[c] && sh.deal.head[i] == sh.deal.head[c]; };
        if (c < blocks && sh.deal.off[c] > 0 && (!same(c - 1) || sh.deal.off[c - 1] == 0)) {
            int lo = c, hi = blocks - 1;                   // the last block that starts inside, too: starts go up
            while (lo < hi) {
                const int mid = (lo + hi + 1) / 2;
                if (same(mid)) lo = mid;
                else hi = mid - 1;
            }
            parts = lo - c + 2;                            // those and the block before
        }
#pragma unroll
        for (int many = 0; many < 2; ++many) {
            const bool is = parts > 0 && (parts > kFewParts && !large) == (many != 0);
            int total;
            const int at = n_joins[many] + cache_block_scan(is ? 1 : 0, s_scan, &total);
            const int to = many ? last - at : at;
            if (is && DYBIT_CHECK(to >= 0 && to <= last, 0x8c)) joins[to] = {out[sh.deal.tile[c]], sh.deal.head[c], c, parts, 0};
            n_joins[many] += total;
        }
    }
    if (threadIdx.x == 0) counts[0] = n, counts[1] = blocks, counts[2] = n_joins[0], counts[3] = n_joins[1];
}

// The plan's work dealt out again for calls that mask otherwise than it expects: block 0 the small tiles', block 1 the large ones'.
// to: counts, tiles and starts as in the plan.
__global__ void __launch_bounds__(kCachePlanThreads) cache_deal_kernel(const CacheShape s, const int *plan, int *to) {
    __shared__ int s_scan[kCachePlanThreads / 32];
    __shared__ CachePlanShared sh;
    pdl_enter();
    const CachePlanLayout L(s);
    const bool large = blockIdx.x != 0;
    const int64_t tiles = large ? L.large : L.small, starts = large ? L.large_starts : L.small_starts, joins = large ? L.large_joins : L.small_joins;
    const int counts = large ? kPlanLarge : kPlanSmall;
    cache_deal(s, reinterpret_cast<const CacheTile *>(plan + tiles), reinterpret_cast<CacheTile *>(to + tiles), plan[counts],
               reinterpret_cast<CacheStart *>(to + starts), reinterpret_cast<CacheJoin *>(to + joins), large, to + counts, s_scan, sh);
}

// One block.  The lists' capacities hold for starts that never decrease; entries beyond them (starts that do) are dropped,
// not written.  Integer work of B sequences: counts and the lists, a warp to a sequence; then the blocks' starts.  Some kilobytes: bound by
// the block's barriers and searches, 10 us for a few sequences, 22 for 64 (2368 starts, each found by bisection).
__global__ void __launch_bounds__(kCachePlanThreads) cache_plan_kernel(const CachePlanArgs a) {
    __shared__ int s_scan[kCachePlanThreads / 32];
    __shared__ CachePlanShared sh;
    pdl_enter();
    const CachePlanLayout L(a.s);
    const int B = a.s.B, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int at[3] = {0, 0, 0};                                // items, small and large tiles
    for (int b0 = 0; b0 < B; b0 += kCachePlanThreads) {
        const int b = b0 + threadIdx.x;
        CacheSeq q = {};
        if (b < B) q = cache_seq(a, b);
        const int count[3] = {q.items, q.small_tiles, q.large_tiles};
        int first[3];
#pragma unroll
        for (int c = 0; c < 3; ++c) {
            int total;
            first[c] = at[c] + cache_block_scan(count[c], s_scan, &total);
            at[c] += total;
        }
        __syncthreads();
        sh.seqs[threadIdx.x] = {q, {first[0], first[1], first[2]}};
        __syncthreads();
        // a warp to a sequence
        for (int k = warp; k < kCachePlanThreads && b0 + k < B; k += kCachePlanThreads / 32) {
            const int seq = b0 + k;
            const CacheSeq m = sh.seqs[k].q;
            const int i0 = sh.seqs[k].first[0];
            const int page = a.s.page, outside = min(m.n, max(0, m.n - m.len)), p0 = m.len - (m.n - outside), out_items = cache_div_up(outside, page);
            CacheItem *list = reinterpret_cast<CacheItem *>(a.plan + L.items) + i0;
            for (int i = lane; i < m.items; i += 32) {
                CacheItem it;
                if (i < out_items) {
                    it = {m.row + i * page, -1, min(page, outside - i * page), seq};
                } else {
                    const int j = p0 / page + (i - out_items), lo = max(p0, j * page), hi = (int)min((int64_t)m.len, (int64_t)(j + 1) * page);
                    it = {m.row + outside + lo - p0, lo, hi - lo, seq};
                }
                if ((unsigned)(i0 + i) < (uint64_t)L.items_cap) list[i] = it;
            }
            auto tiles = [&](int64_t list_at, int64_t cap, int n_tiles, int t0) {
                CacheTile *out = reinterpret_cast<CacheTile *>(a.plan + list_at) + t0;
                for (int i = lane; i < n_tiles; i += 32)
                    if ((unsigned)(t0 + i) < (uint64_t)cap) out[i] = {m.row, m.n, m.len, seq, i, 0, 0};
            };
            tiles(L.small, L.small_cap, m.small_tiles, sh.seqs[k].first[1]);
            tiles(L.large, L.large_cap, m.large_tiles, sh.seqs[k].first[2]);
        }
    }
    const int64_t caps[3] = {L.items_cap, L.small_cap, L.large_cap};
#pragma unroll
    for (int c = 0; c < 3; ++c) at[c] = (unsigned)at[c] < (uint64_t)caps[c] ? at[c] : (int)caps[c];
    __syncthreads();
    CacheTile *small = reinterpret_cast<CacheTile *>(a.plan + L.small), *large = reinterpret_cast<CacheTile *>(a.plan + L.large);
    if (threadIdx.x == 0) a.plan[0] = at[0];
    cache_deal(a.s, small, small, at[1], reinterpret_cast<CacheStart *>(a.plan + L.small_starts), reinterpret_cast<CacheJoin *>(a.plan + L.small_joins), false,
               a.plan + kPlanSmall, s_scan, sh);
    __syncthreads();
    cache_deal(a.s, large, large, at[2], reinterpret_cast<CacheStart *>(a.plan + L.large_starts), reinterpret_cast<CacheJoin *>(a.plan + L.large_joins), true,
               a.plan + kPlanLarge, s_scan, sh);
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
// Four prompts of 2048 tokens, 8 heads of 128 in bf16 (50 MB): 16.6 us, floor 7.7.  Bound by latency: 74 registers leave a third of
// the warps, issue 53 %, DRAM 23 %.
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
    if constexpr (W > 1) named_tile_sync<TPR>(sub);        // every thread of the tile has read the old scale
    else __syncwarp();
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
    int64_t tokens;
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
            if (!DYBIT_CHECK(c + E <= p.dim && row < it.count && it.row >= 0 && it.row + row < p.tokens, 0x86)) continue;
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
