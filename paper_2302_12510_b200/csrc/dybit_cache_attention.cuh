// Attention over the 8-bit cache.
//
//     x[i][j] = scale * q_i . k_j  (keys j that row i sees),   y_i = sum_j softmax_j(x[i]) v_j,   k_j = s_K(page) * value(code)
//
// Rows are (new token, query head) pairs of one key head: the heads of a group share every key that is fetched.  Two
// kernels: this one for tiles of 8 or 16 rows, bound by the one pass over the codes, and dybit_cache_prefill.cuh for
// tiles of 256 rows, bound by the tensor cores.
//
// Launches of a call that do not need one another run side by side as far as there is room: a kernel waits for what came before the
// call's first kernel through that one (which lets its successor start only behind its own wait), and for its neighbour before it
// ends, so that the end of the last one is the end of all.  (Blocks of the two kinds of tiles do not share an SM: 55,296 and 64,512 or
// 65,536 registers.  Small tiles begin where a block of large ones has ended or has no work.)
//
// What both have in common.  The running maximum of a row goes over x + log2 of the values' scale (base 2), so
//     p'_j = 2^(x_j + e_j - m),   e_j = log2 s_V(page) - E0
// is at most a small constant and the second product takes the bare values of the codes, exact in f16 (seven significant
// bits), with p' rounded to f16: half a step is 2^-11 of it, that of an f16 output.  (Below 2^-14 of the row's largest, 2^-25 of that.
// On prompts and decode steps outputs in f16 are 2.5e-4 from the formula, where fp32 probabilities give 2.0e-4; in bf16 the
// outputs' own rounding, 1.6e-3, hides it.)  The sum of the probabilities is
//     l = sum_j p'_j * 2^-e_j    in fp32, one product per page,
// and y = 2^E0 * (sum_j p'_j value_j) / l.  E0 is the exponent of one of the first pages of a part that a row of the tile
// sees: a page that all rows have slid past may hold anything.  The maximum is raised only when it would grow by more than 2^8 (p'
// stays below that, far from f16's end), so the accumulators are hardly ever rescaled.
#pragma once

#include "dybit_cache.cuh"
#include "dybit_wait.cuh"

namespace dybit {

__device__ __forceinline__ void enter_beside(int beside) {
    if (!beside) asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}
__device__ __forceinline__ void leave_beside(int beside) {
    if (beside) asm volatile("griddepcontrol.wait;" ::: "memory");
}

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kRaise = 8.0f;
constexpr int kCacheMaxDim = 128, kCacheMaxGroup = 128;

struct CacheAttn {
    const int *counts;           // of the plan: tiles, blocks, joins of few parts and of many
    const CacheTile *tiles;
    const CacheStart *starts;
    const CacheJoin *joins;
    const int *table;
    int64_t table_stride;
    int64_t pages;
    int page_shift, heads, group, dim;
    const float *k_scales, *v_scales;
    const void *q;
    int64_t q_token, q_head;
    void *y;
    int64_t y_token, y_head;
    float *lse;                  // [T][query heads], or null
    float scale_log2;            // softmax scale * log2(e)
    int causal, window;          // window: keys that a row sees, its own the last; INT_MAX for all
    float *part_y;               // [slot][rows][dim]: sums of the parts of tiles that several blocks work on
    float4 *part_ml;             // [slot][rows]: {m + E0, l, E0, -}
    int q_vec, q_vec16, y_vec, y_vec16;  // rows can be moved in pieces of 8 (16) bytes
    int beside;                  // this launch may run beside the one before it, whose own wait covers what both read
    int64_t tokens;              // rows of q and y
};

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Four codes of a word as two pairs of 16-bit numbers, the codes of bytes 0 and 2 and those of bytes 1 and 3: decode2 of
// dybit_code8.cuh, for f16 as well (1024 + c is exact there, and the patterns add up to 36 << 10).  What contracts or carries
// the codes is free to take every other one, and so no byte permutation spreads them (132 us with one, 127 without, for a pass over
// 524 MB of codes).
__device__ __forceinline__ __half2 as_half2(unsigned w) { return *reinterpret_cast<const __half2 *>(&w); }
__device__ __forceinline__ unsigned half2_bits(__half2 v) { return *reinterpret_cast<const unsigned *>(&v); }
// codes in bytes 0 and 2 of w, their signs at bits 15 and 31 of s
template <typename T> __device__ __forceinline__ unsigned decode_pair(unsigned w, unsigned s);
template <> __device__ __forceinline__ unsigned decode_pair<__half>(unsigned w, unsigned s) {
    const __half2 h = as_half2((w & 0x007f007fu) | 0x64006400u);
    const unsigned g = half2_bits(__hfma2(h, as_half2(0xbc00bc00u), as_half2(0x64806480u)));           // 1152 - h = 128 - c
    const __half2 curve = as_half2(0x90009000u - g);
    const __half2 above = __hfma2_relu(h, as_half2(0xa000a000u), as_half2(0x48404840u));               // max(0, 8.5 - h / 128)
    return half2_bits(__hsub2(curve, above)) | (s & 0x80008000u);
}
template <> __device__ __forceinline__ unsigned decode_pair<__nv_bfloat16>(unsigned w, unsigned s) {
    const __nv_bfloat162 h = as_bf162((w & 0x007f007fu) | 0x43004300u);
    const unsigned g = as_u32(__hfma2(h, as_bf162(0xbf80bf80u), as_bf162(0x43804380u)));               // 256 - h = 128 - c
    const __nv_bfloat162 curve = as_bf162(0x82008200u - g);
    const __nv_bfloat162 above = __hfma2_relu(h, as_bf162(0xbc00bc00u), as_bf162(0x3fc03fc0u));        // max(0, 1.5 - h / 128)
    return as_u32(__hsub2(curve, above)) | (s & 0x80008000u);
}
template <typename T>
__device__ __forceinline__ void decode_word(unsigned w, unsigned &even, unsigned &odd) {
    even = decode_pair<T>(w, w << 8);
    odd = decode_pair<T>(w >> 8, w);
}

// Two query elements, infinities as NaN (x * 0 + x; exact for every other number): a row with one then has NaN for every score and is NaN
// itself.  Infinite scores would look like scores of keys that are not there.
template <typename T> __device__ __forceinline__ unsigned nan_for_infinity(unsigned w) {
    if constexpr (__is_same(T, __half)) return half2_bits(__hfma2(as_half2(w), as_half2(0u), as_half2(w)));
    else return as_u32(__hfma2(as_bf162(w), as_bf162(0u), as_bf162(w)));
}

// d (16 x 8, fp32) += a (16 x 16) * b (16 x 8) on the legacy tensor path: sixteen rows of codes against eight queries.
template <typename T>
__device__ __forceinline__ void mma_16816(float (&d)[4], unsigned a0, unsigned a1, unsigned a2, unsigned a3, const unsigned (&b)[2]) {
    if constexpr (__is_same(T, __half)) {
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b[0]), "r"(b[1]));
    } else {
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b[0]), "r"(b[1]));
    }
}

// An 8 x 8 matrix of 16-bit elements, two to a lane, with rows and columns exchanged.
__device__ __forceinline__ unsigned transpose8(unsigned a) {
    unsigned d;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
    return d;
}

// Row r of a sequence: its token's position, and which keys [lo, hi) it sees.  Rows that are not there see none.
struct RowKeys { int lo, hi; };
__device__ __forceinline__ RowKeys row_keys(const CacheAttn &p, const CacheTile &t, int r) {
    RowKeys k = {0, 0};
    const int token = r / p.group;
    if (token >= t.n) return k;
    const int pos = t.len - t.n + token;
    k.hi = p.causal ? max(0, pos + 1) : t.len;
    k.lo = p.window == 0x7fffffff ? 0 : max(0, pos + 1 - p.window);
    return k;
}

// A part of a tile: units from .. to - 1 of its work, for one key head.  slot < 0: the whole tile.
struct CachePart {
    CacheTile tile;
    int head, from, to, slot;
};

// Where a block is in the work.
struct CachePlace { int tile, head, off; };
__device__ __forceinline__ CachePlace cache_place(const CacheStart &s) { return {s.tile, s.head, s.off}; }

// The next part of a block's share, which ends at `end`; false where there is none.  part.tile is the tile at `at` already.  A part
// that starts inside a tile is the block's first, one that ends inside a tile its last: two slots to a block are enough.
__device__ __forceinline__ bool cache_next(const CacheAttn &p, int block, CachePlace &at, const CachePlace &end, int n_tiles, CachePart &part) {
    if (at.head > end.head || (at.head == end.head && (at.tile > end.tile || (at.tile == end.tile && at.off >= end.off)))) return false;
    part.head = at.head;
    part.from = at.off;
    part.to = at.head == end.head && at.tile == end.tile ? min(end.off, part.tile.units) : part.tile.units;
    part.slot = part.from == 0 && part.to == part.tile.units ? -1 : 2 * block + (part.from == 0 ? 1 : 0);
    at.off = 0;
    if (++at.tile == n_tiles) at.tile = 0, ++at.head;
    return true;
}

// The keys [first, last) of a part of a tile whose rows are r0 .. r0 + rows - 1, in units of `unit` keys.
struct KeyRange { int first, last; };
__device__ __forceinline__ KeyRange part_keys(const CacheAttn &p, const CachePart &part, int r0, int rows, int unit) {
    const CacheTile &t = part.tile;
    const RowKeys a = row_keys(p, t, r0), z = row_keys(p, t, min(r0 + rows, t.n * p.group) - 1);
    KeyRange k = {0, 0};
    if (z.hi <= a.lo) return k;                            // positions grow with the row
    const int u0 = a.lo / unit, u1 = cache_div_up(z.hi, unit), n = u1 - u0;
    k.first = (u0 + (int)((int64_t)n * part.from / t.units)) * unit;
    k.last = (u0 + (int)((int64_t)n * part.to / t.units)) * unit;
    return k;
}

// y of row r, elements d .. d + 3, from the sums at maximum m (relative to the exponent e0), and its logarithm of the sum.
template <typename T>
__device__ __forceinline__ void store_attention_row(const CacheAttn &p, const CacheTile &tile, int head, int r, int d, const float4 &s, float l,
                                                    float m, float e0) {
    const int token = r / p.group, h = head * p.group + (r - token * p.group);
    // a row that sees no key: zeros (and minus infinity)
    const float inv = l == 0.0f ? 0.0f : __fdiv_rn(1.0f, l), up = __uint_as_float((unsigned)((int)e0 + 127) << 23);
    T *y = static_cast<T *>(p.y) + (tile.row + token) * p.y_token + h * p.y_head + d;
    const float f0 = s.x * inv * up, f1 = s.y * inv * up, f2 = s.z * inv * up, f3 = s.w * inv * up;
    if (!DYBIT_CHECK(token < tile.n && tile.row >= 0 && tile.row + token < p.tokens && d + 4 <= p.dim, 0x87)) return;
    if (p.y_vec) {
        *reinterpret_cast<uint2 *>(y) = make_uint2(pack2<T>(f0, f1), pack2<T>(f2, f3));
    } else {
        y[0] = from_f32<T>(f0), y[1] = from_f32<T>(f1), y[2] = from_f32<T>(f2), y[3] = from_f32<T>(f3);
    }
    if (d == 0 && p.lse != nullptr)
        p.lse[(int64_t)(tile.row + token) * (p.heads * p.group) + h] = l == 0.0f ? -INFINITY : (m + __log2f(l)) * kLn2;
}

// ------------------------------------------------------------------ tiles of 8 or 16 rows

constexpr int kSmSegment = 1024;             // keys whose page numbers and scales are held in shared memory at a time
constexpr int kSmBytes = 4096;               // codes of the keys (of the values) that a warp takes at a time
__host__ __device__ constexpr int small_smem(int rows) { return small_per_sm(rows) * 2 * kSmBytes + 1024; }

// Two 16 x 16 matrices of bytes in shared memory, transposed: lane 4 * g + t gets the bytes 4t .. 4t + 3 of column g (r0; second
// matrix r2) and of column g + 8 (r1, r3).  Lanes 0 .. 15 give the rows of the first matrix, the others those of the second.
__device__ __forceinline__ void ldmatrix_b8_trans(uint32_t addr, unsigned &r0, unsigned &r1, unsigned &r2, unsigned &r3) {
    asm volatile("ldmatrix.sync.aligned.m16n16.x2.trans.shared.b8 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r0), "=r"(r1), "=r"(r2), "=r"(r3)
                 : "r"(addr)
                 : "memory");
}

// What the score and value loops need of the keys of a box.
struct alignas(32) KeyBlock {
    float c, e, f;               // x's factor, values' exponent, 2^-e
    int y, z, zv;                // token in the page, page * heads + head of keys and of values: the TMA's coordinates
};

// Every warp has a share of its own, 32 keys (heads of up to 64: 64) to a round; a tile that is cut is joined afterwards.  The TMA
// fills a buffer for keys and one for values; both are read into registers at once and filled again while their codes are worked
// on.  Shares are equal; a scheduler favours its older warps, so the last of its warps works alone for a while.  Shares by age and a
// pause for warps that are ahead gained nothing.
// Both products have the codes as their left operand, sixteen rows of them, and 8 * NQ query rows as their right one:
//     S^T = K Q^T (keys x rows),   Y^T += V^T P^T (head elements x rows)
// so that an instruction takes twice the codes that it would with the queries on the left.  A stage is read straight into
// the fragments: contractions over head elements and over keys may run in any order.  Of K a lane takes 16 consecutive codes of
// two neighbouring keys, of V, which the instruction wants with keys side by side, four keys of a head element, by a
// transposing load of bytes; the keys of both products are numbered by what that load gives (row i of the two halves of 16 keys is
// key 2i and key 2i + 1).  Bound by instruction issue, then by HBM: 64 requests of 4000 keys take 88 M warp instructions, 57 M of them to decode
// (7 to a pair of codes), at 74 % of the issue slots 122 us where the codes' bytes take 80.
// BOX: keys of a TMA box, 32 or, on pages of 16 tokens, 16.
template <typename T, int DP, int NQ, int BOX>
__global__ void __launch_bounds__(32 * small_per_sm(8 * NQ), 1)
cache_small_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const CacheAttn p) {
    constexpr int KS = DP / 16;                            // matrix instructions along a head
    constexpr int ROWS = 8 * NQ, WARPS = small_per_sm(ROWS), KEYS = kSmBytes / DP, BL = KEYS / 16, NB = KEYS / BOX;      // blocks of 16 keys, boxes
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    __shared__ KeyBlock s_blocks[WARPS][kSmSegment / BOX];
    __shared__ uint64_t s_full[WARPS][2];
    __shared__ uint32_t s_abort;

    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    KeyBlock *const s_block = s_blocks[warp];
    uint64_t *const k_full = &s_full[warp][0], *const v_full = &s_full[warp][1];
    if (lane == 0) {
        mbar_init(k_full, 1);
        mbar_init(v_full, 1);
        if (warp == 0) s_abort = 0;
        fence_mbar_init();
    }
    if (threadIdx.x == 0) {
        prefetch_tensormap(&map_k);
        prefetch_tensormap(&map_v);
    }
    __syncthreads();
    enter_beside(p.beside);
    const int block = warp * (int)gridDim.x + (int)blockIdx.x, n_tiles = __ldg(p.counts), n_blocks = __ldg(p.counts + 1);
    CachePart part;
    part.tile = p.starts[block].t;
    CachePlace at = cache_place(p.starts[block]);
    const CachePlace end = cache_place(p.starts[block + 1]);
    if (block >= n_blocks) {
        leave_beside(p.beside);
        return;
    }
    uint8_t *ks = smem + warp * (2 * kSmBytes), *vs = ks + kSmBytes;
    uint32_t it = 0;                                       // rounds so far
    bool ok = true;

    while (ok && cache_next(p, block, at, end, n_tiles, part)) {
        const CacheTile &tile = part.tile;
        const int head = part.head, r0 = tile.tile * ROWS, rows = min(ROWS, tile.n * p.group - r0);
        const KeyRange range = part_keys(p, part, r0, ROWS, KEYS);
        const int *table = p.table + tile.seq * p.table_stride;
        // this lane's scores are those of rows 8 * q + 2t and 8 * q + 2t + 1
        RowKeys seen[NQ][2];
#pragma unroll
        for (int q = 0; q < NQ; ++q)
#pragma unroll
            for (int h = 0; h < 2; ++h) seen[q][h] = row_keys(p, tile, r0 + 8 * q + 2 * t + h);
        // keys between these two are seen by every row that is there
        const int all_lo = row_keys(p, tile, r0 + rows - 1).lo, all_hi = row_keys(p, tile, r0).hi;

        // queries as right-hand fragments: row 8 * q + g; k index 2t, 2t+1 (8+2t, 8+2t+1) of step j is head element
        // 16 * (t + 4 * (j / 4)) + 4 * (j % 4) + 0, 2 (1, 3)
        unsigned qf[NQ][KS][2];
#pragma unroll
        for (int q = 0; q < NQ; ++q) {
            const int r = r0 + 8 * q + g, token = r / p.group, h = head * p.group + (r - token * p.group);
            const T *row = 8 * q + g < rows ? static_cast<const T *>(p.q) + (tile.row + token) * p.q_token + h * p.q_head : nullptr;
#pragma unroll
            for (int j = 0; j < KS; ++j) {
                const int d = 16 * (t + 4 * (j / 4)) + 4 * (j % 4);
                uint2 v = make_uint2(0u, 0u);
                if (row != nullptr && d < p.dim) {
                    if (p.q_vec) {
                        v = __ldg(reinterpret_cast<const uint2 *>(row + d));
                    } else {
                        T e[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) e[i] = row[d + i];
                        memcpy(&v, e, 8);
                    }
                }
                v.x = nan_for_infinity<T>(v.x), v.y = nan_for_infinity<T>(v.y);
                qf[q][j][0] = __byte_perm(v.x, v.y, 0x5410), qf[q][j][1] = __byte_perm(v.x, v.y, 0x7632);
            }
        }

        float e0 = 0.0f;                                   // exponent of the value scale of the first keys that are seen
        // output i: head elements 16i + g (o[0], o[1]) and 16i + g + 8 (o[2], o[3]) of rows 8q + 2t and 8q + 2t + 1
        float o[NQ][KS][4], m[NQ][2], l[NQ][2];
#pragma unroll
        for (int q = 0; q < NQ; ++q) {
#pragma unroll
            for (int i = 0; i < KS; ++i) o[q][i][0] = o[q][i][1] = o[q][i][2] = o[q][i][3] = 0.0f;
            m[q][0] = m[q][1] = -INFINITY;
            l[q][0] = l[q][1] = 0.0f;
        }
        for (int seg = range.first; seg < range.last && ok; seg += kSmSegment) {
            const int seg_end = min(range.last, seg + kSmSegment);
            __syncwarp();
            const int boxes = (seg_end - seg) / BOX, none = (int)(p.pages * p.heads);      // a coordinate outside the pool reads as zeros
            auto box_of = [&](int i) {
                const int key = seg + BOX * i;
                const int pg = i < boxes && key < tile.len ? __ldg(table + (key >> p.page_shift)) : -1;
                return (unsigned)pg < (uint64_t)p.pages ? (int)((int64_t)pg * p.heads + head) : none;
            };
            int z = box_of(lane);
            if (lane < NB) {                               // the first keys are on their way before anything else is known
                if (lane == 0) mbar_arrive_expect_tx(k_full, kSmBytes);
                __syncwarp((1u << NB) - 1u);
                tma_load_3d(ks + lane * BOX * DP, &map_k, 0, (seg + BOX * lane) & ((1 << p.page_shift) - 1), z, k_full);
            }
            __syncwarp();
            for (int i0 = 0; i0 < boxes; i0 += 32) {
                const int i = i0 + lane;
                KeyBlock b = {0.0f, -INFINITY, 0.0f, (seg + BOX * i) & ((1 << p.page_shift) - 1), z, none};      // not there: seen by no row
                float vs = 0.0f;
                if (z != none) {
                    vs = __ldg(p.v_scales + z);
                    b.c = __ldg(p.k_scales + z) * p.scale_log2;
                    b.zv = vs > 0.0f ? z : none;
                }
                const float e = vs > 0.0f ? (float)((int)((__float_as_uint(vs) >> 23) & 255u) - 127) : 0.0f;
                if (i0 == 0 && seg == range.first) {
                    // of the first round's boxes the one with the first key that all rows see, or else the last, which some row sees
                    int at = 0;
#pragma unroll
                    for (int k = 1; k < NB; ++k) at += all_lo >= seg + k * BOX ? 1 : 0;
                    e0 = __shfl_sync(0xffffffffu, e, at);
                }
                if (z != none) {
                    b.e = vs > 0.0f ? e - e0 : 0.0f;
                    b.f = __uint_as_float((unsigned)(127 - max(-126, min(126, (int)b.e))) << 23);
                }
                if (i < boxes) s_block[i] = b;
                z = box_of(i + 32);
            }
            __syncwarp();
            const int rounds = (seg_end - seg) / KEYS;
            auto fetch = [&](int i, bool values) {         // one lane
                uint64_t *bar = values ? v_full : k_full;
                mbar_arrive_expect_tx(bar, kSmBytes);
#pragma unroll
                for (int b = 0; b < NB; ++b) {
                    const KeyBlock &k = s_block[NB * i + b];
                    tma_load_3d((values ? vs : ks) + b * BOX * DP, values ? &map_v : &map_k, 0, k.y, values ? k.zv : k.z, bar);
                }
            };
            if (lane == 0) fetch(0, true);
            __syncwarp();
            for (int i = 0; i < rounds; ++i, ++it) {
                const bool more = lane == 0 && i + 1 < rounds;
                ok = __all_sync(0xffffffffu, wait_bounded(k_full, it & 1u, &s_abort, 0x81));
                if (!ok) break;
                // keys 2g and 2g + 1 of each block; a fragment is 16 codes
                uint4 w[BL][2][DP / 64];
#pragma unroll
                for (int b = 0; b < BL; ++b)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const int row = b * 16 + 2 * g + h;
                        if constexpr (DP == 128) {
                            w[b][h][0] = *reinterpret_cast<const uint4 *>(ks + row * 128 + ((t ^ (row & 7)) << 4));
                            w[b][h][1] = *reinterpret_cast<const uint4 *>(ks + row * 128 + (((t + 4) ^ (row & 7)) << 4));
                        } else {
                            w[b][h][0] = *reinterpret_cast<const uint4 *>(ks + row * 64 + ((t ^ ((row >> 1) & 3)) << 4));
                        }
                    }
                __syncwarp();
                if (more) fetch(i + 1, false);
                // x[b][q][0], [1]: key 2g of block b, rows 8q + 2t and 8q + 2t + 1; [2], [3]: key 2g + 1
                float x[BL][NQ][4];
#pragma unroll
                for (int b = 0; b < BL; ++b) {
#pragma unroll
                    for (int q = 0; q < NQ; ++q) x[b][q][0] = x[b][q][1] = x[b][q][2] = x[b][q][3] = 0.0f;
#pragma unroll
                    for (int j = 0; j < KS; ++j) {
                        unsigned c[2];
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const uint4 &q4 = w[b][h][j / 4];
                            c[h] = j % 4 == 0 ? q4.x : j % 4 == 1 ? q4.y : j % 4 == 2 ? q4.z : q4.w;
                        }
                        unsigned a0, a1, a2, a3;
                        decode_word<T>(c[0], a0, a2);
                        decode_word<T>(c[1], a1, a3);
#pragma unroll
                        for (int q = 0; q < NQ; ++q) mma_16816<T>(x[b][q], a0, a1, a2, a3, qf[q][j]);
                    }
                }
                const int first = seg + KEYS * i;
                const bool edge = first < all_lo || first + KEYS > all_hi;
                // scores in base 2 are x * c + e; the factor is not negative: the largest product has the largest score
                float c[BL], e[BL], f[BL], top[NQ][2];
#pragma unroll
                for (int b = 0; b < BL; ++b) {
                    const float4 kb = *reinterpret_cast<const float4 *>(&s_block[NB * i + b * 16 / BOX]);
                    c[b] = kb.x, e[b] = kb.y, f[b] = kb.z;
                    if (edge) {
                        const int ka = first + b * 16 + 2 * g;
#pragma unroll
                        for (int q = 0; q < NQ; ++q)
#pragma unroll
                            for (int k = 0; k < 4; ++k) {
                                const int key = ka + (k >> 1);
                                const bool is = key >= seen[q][k & 1].lo && key < seen[q][k & 1].hi;
                                x[b][q][k] = is ? __fmaf_rn(x[b][q][k], c[b], e[b]) : -INFINITY;
                            }
                        c[b] = 1.0f, e[b] = 0.0f;
                    }
#pragma unroll
                    for (int q = 0; q < NQ; ++q)
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const float a = __fmaf_rn(fmaxf(x[b][q][h], x[b][q][2 + h]), c[b], e[b]);
                            top[q][h] = b == 0 ? a : fmaxf(top[q][h], a);
                        }
                }
                bool raise = false;
#pragma unroll
                for (int q = 0; q < NQ; ++q) raise |= top[q][0] > m[q][0] + kRaise || top[q][1] > m[q][1] + kRaise;
                if (__any_sync(0xffffffffu, raise)) {
#pragma unroll
                    for (int q = 0; q < NQ; ++q)
#pragma unroll
                        for (int h = 0; h < 2; ++h) {          // the row's maximum over the eight lanes that share it
                            float a = top[q][h];
#pragma unroll
                            for (int d = 4; d < 32; d <<= 1) a = fmaxf(a, __shfl_xor_sync(0xffffffffu, a, d));
                            const float n = fmaxf(m[q][h], a), s = m[q][h] == n ? 1.0f : ex2(m[q][h] - n);
                            m[q][h] = n;
                            l[q][h] *= s;
#pragma unroll
                            for (int d = 0; d < KS; ++d) o[q][d][h] *= s, o[q][d][2 + h] *= s;
                        }
                }
                unsigned pf[BL][NQ][2];
#pragma unroll
                for (int q = 0; q < NQ; ++q) {
                    const float u0 = m[q][0] == -INFINITY ? 0.0f : m[q][0], u1 = m[q][1] == -INFINITY ? 0.0f : m[q][1];
#pragma unroll
                    for (int b = 0; b < BL; ++b) {
                        float(&v)[4] = x[b][q];
                        const float s0 = e[b] - u0, s1 = e[b] - u1;
                        v[0] = ex2(__fmaf_rn(v[0], c[b], s0)), v[1] = ex2(__fmaf_rn(v[1], c[b], s1));
                        v[2] = ex2(__fmaf_rn(v[2], c[b], s0)), v[3] = ex2(__fmaf_rn(v[3], c[b], s1));
                        l[q][0] = __fmaf_rn(v[0] + v[2], f[b], l[q][0]);
                        l[q][1] = __fmaf_rn(v[1] + v[3], f[b], l[q][1]);
                        // keys x rows -> rows x keys
                        pf[b][q][0] = transpose8(pack_f16(v[0], v[1]));
                        pf[b][q][1] = transpose8(pack_f16(v[2], v[3]));
                    }
                }
                ok = __all_sync(0xffffffffu, wait_bounded(v_full, it & 1u, &s_abort, 0x8a));
                if (!ok) break;
                unsigned z[BL][KS][2];                     // four keys of head elements 16j + g and 16j + g + 8
#pragma unroll
                for (int b = 0; b < BL; ++b) {
                    const int row = b * 16 + (lane & 15);
#pragma unroll
                    for (int j = 0; j < KS; j += 2)
                        ldmatrix_b8_trans(smem_u32(vs) + row * DP + (((j + (lane >> 4)) ^ (DP == 128 ? row & 7 : (row >> 1) & 3)) << 4), z[b][j][0], z[b][j][1],
                                          z[b][j + 1][0], z[b][j + 1][1]);
                }
                __syncwarp();
                if (more) fetch(i + 1, true);
#pragma unroll
                for (int b = 0; b < BL; ++b)
#pragma unroll
                    for (int j = 0; j < KS; ++j) {
                        unsigned a0, a1, a2, a3;
                        decode_word<__half>(z[b][j][0], a0, a2);
                        decode_word<__half>(z[b][j][1], a1, a3);
#pragma unroll
                        for (int q = 0; q < NQ; ++q) mma_16816<__half>(o[q][j], a0, a1, a2, a3, pf[b][q]);
                    }
            }
        }
        if (!ok) {                                             // copies in flight land before the block's memory is given up
            for (int i = 0; i < 64; ++i) __nanosleep(2000);
        }

        // through shared memory, so that a lane has four elements of a row side by side
#pragma unroll
        for (int q = 0; q < NQ; ++q)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) l[q][h] += __shfl_xor_sync(0xffffffffu, l[q][h], d);
        constexpr int LD = DP + 4;
        float *const all = reinterpret_cast<float *>(ks), *const stats = all + 8 * LD;
        const int vecs = p.dim / 4;
#pragma unroll
        for (int q = 0; q < NQ; ++q) {
            if (q * 8 >= rows) break;
            __syncwarp();
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float *row = all + (2 * t + h) * LD + g;
#pragma unroll
                for (int i = 0; i < KS; ++i) row[16 * i] = o[q][i][h], row[16 * i + 8] = o[q][i][2 + h];
                if (g == 0) stats[2 * (2 * t + h)] = m[q][h], stats[2 * (2 * t + h) + 1] = l[q][h];
            }
            __syncwarp();
            for (int i = lane; i < 8 * vecs; i += 32) {
                const int lr = i / vecs, d = (i - lr * vecs) * 4, r = q * 8 + lr;
                if (r >= rows) break;
                const float4 v = *reinterpret_cast<const float4 *>(all + lr * LD + d);
                const float top = stats[2 * lr], sum = stats[2 * lr + 1];
                if (part.slot >= 0) {
                    if (!DYBIT_CHECK(part.slot < 2 * small_blocks(ROWS) && r < ROWS && d + 4 <= p.dim, 0x8d)) continue;
                    const int64_t to = (int64_t)part.slot * ROWS + r;
                    *reinterpret_cast<float4 *>(p.part_y + to * p.dim + d) = v;
                    if (d == 0) p.part_ml[to] = make_float4(top + e0, sum, e0, 0.0f);
                } else {
                    store_attention_row<T>(p, tile, head, r0 + r, d, v, sum, top, e0);
                }
            }
        }
        part.tile = p.tiles[at.tile];
        fence_proxy_async_smem();                          // the buffers are the TMA's again
        __syncwarp();
    }
    leave_beside(p.beside);
}

// ------------------------------------------------------------------ parts of a tile, joined

// Where element d of row r of a large tile's part lies: rows of 32 side by side, four elements each, as the threads that hold them
// write them.
__device__ __forceinline__ int64_t large_part_at(int64_t r, int d, int dim) { return ((r >> 5) * (dim / 4) + d / 4) * 128 + (r & 31) * 4; }

// Joins the parts of tiles at their common maximum.  part_ml.x is a part's maximum with its exponent in it, so that parts whose
// values have other scales compare.  Small tiles of few parts take a warp each, those of many a block of eight warps to a row.  Large
// tiles: a lane to a row, blockIdx.y a group of 32 rows, the warps share the head's elements.  Bound by latency: eight parts of a
// warp are on their way at once (with four warps and four parts one request of 65,000 keys took 80 us, of 4096 keys 19.7; now 59 and
// 17.6).
struct JoinSum { float4 s; float m, l; };

// l counts in the first part's exponent already
__device__ __forceinline__ void join_add(JoinSum &a, float m, float l, const float4 &s) {
    const float top = fmaxf(a.m, m), f = a.m == -INFINITY ? 0.0f : ex2(a.m - top), w = m == -INFINITY ? 0.0f : ex2(m - top);
    a.s.x = a.s.x * f + s.x * w, a.s.y = a.s.y * f + s.y * w, a.s.z = a.s.z * f + s.z * w, a.s.w = a.s.w * f + s.w * w;
    a.l = a.l * f + l * w;
    a.m = top;
}

template <int ROWS>
__device__ __forceinline__ int64_t join_row(const CacheJoin &j, int k, int r) {
    // slots of the parts: the second one of the block before, then the first ones of the blocks that start in the tile
    return (int64_t)(k == 0 ? 2 * j.first - 1 : 2 * (j.first + k - 1)) * ROWS + r;
}

// Parts first, first + step ... of elements d .. d + 3 of row r, AHEAD of them on their way at once; e: the first part's exponent.
template <int ROWS, int AHEAD>
__device__ __forceinline__ JoinSum join_parts(const CacheAttn &p, const CacheJoin &j, int r, int d, int first, int step, float e) {
    JoinSum a = {make_float4(0.f, 0.f, 0.f, 0.f), -INFINITY, 0.0f};
#pragma unroll AHEAD
    for (int k = first; k < j.parts; k += step) {
        const int64_t at = join_row<ROWS>(j, k, r);
        const float4 ml = __ldcg(p.part_ml + at);
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        if (d < p.dim) v = __ldcg(reinterpret_cast<const float4 *>(p.part_y + (ROWS == kLargeRows ? large_part_at(at, d, p.dim) : at * p.dim + d)));
        join_add(a, ml.x, ml.y * ex2(e - ml.z), v);
    }
    return a;
}

template <typename T, int ROWS>
__global__ void __launch_bounds__(256) cache_join_kernel(const CacheAttn p) {
    __shared__ float4 s_sum[8][kCacheMaxDim / 4];
    __shared__ float2 s_ml[8];
    enter_beside(p.beside);
    const int few = __ldg(p.counts + 2), many = __ldg(p.counts + 3), lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    auto rows_of = [&](const CacheJoin &j) { return min(ROWS, j.t.n * p.group - j.t.tile * ROWS); };
    auto store = [&](const CacheJoin &j, int r, int d, const JoinSum &a, float e) {
        if (d < p.dim) store_attention_row<T>(p, j.t, j.head, j.t.tile * ROWS + r, d, a.s, a.l, a.m - e, e);
    };
    if constexpr (ROWS == kLargeRows) {
        for (int i = blockIdx.x; i < few; i += gridDim.x) {
            const CacheJoin j = p.joins[i];
            const int r = blockIdx.y * 32 + lane;
            if (r < rows_of(j)) {
                const float e = __ldcg(p.part_ml + join_row<ROWS>(j, 0, r)).z;
#pragma unroll 2
                for (int d = warp * 4; d < p.dim; d += 32) store(j, r, d, join_parts<ROWS, 4>(p, j, r, d, 0, 1, e), e);
            }
        }
    } else {
        // a tile's rows go to as many blocks (warps) as there are
        const int blocks = many > 0 ? min(ROWS, max(1, (int)gridDim.x / many)) : 1;
        for (int i = blockIdx.x; i < blocks * many; i += gridDim.x) {
            const CacheJoin j = p.joins[small_blocks(ROWS) - 2 - i / blocks];
            for (int r = i % blocks; r < rows_of(j); r += blocks) {
                const float e = __ldcg(p.part_ml + join_row<ROWS>(j, 0, r)).z;
                JoinSum a = join_parts<ROWS, 8>(p, j, r, lane * 4, warp, 8, e);
                s_sum[warp][lane] = a.s;
                if (lane == 0) s_ml[warp] = make_float2(a.m, a.l);
                __syncthreads();
                if (warp == 0) {
#pragma unroll
                    for (int w = 1; w < 8; ++w) join_add(a, s_ml[w].x, s_ml[w].y, s_sum[w][lane]);
                    store(j, r, lane * 4, a, e);
                }
                __syncthreads();
            }
        }
        const int warps = few > 0 ? min(ROWS, max(1, 8 * (int)gridDim.x / few)) : 1;
        for (int i = blockIdx.x + warp * gridDim.x; i < warps * few; i += 8 * gridDim.x) {
            const CacheJoin j = p.joins[i / warps];
            const int rows = rows_of(j);
#pragma unroll 2
            for (int r = i % warps; r < rows; r += warps) {
                const float e = __ldcg(p.part_ml + join_row<ROWS>(j, 0, r)).z;
                store(j, r, lane * 4, join_parts<ROWS, 4>(p, j, r, lane * 4, 0, 1, e), e);
            }
        }
    }
    leave_beside(p.beside);
}

}  // namespace dybit
