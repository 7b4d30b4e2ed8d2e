// Attention over the 8-bit cache.
//
//     x[i][j] = scale * q_i . k_j  (keys j that row i sees),   y_i = sum_j softmax_j(x[i]) v_j,   k_j = s_K(page) * value(code)
//
// Rows are (new token, query head) pairs of one key head: the heads of a group share every key that is fetched.  Two
// kernels: this one for tiles of up to 16 rows, bound by the one pass over the codes, and dybit_cache_prefill.cuh for
// tiles of 256 rows, bound by the tensor cores.
//
// What both have in common.  The running maximum of a row goes over x + log2 of the values' scale (base 2), so
//     p'_j = 2^(x_j + e_j - m),   e_j = log2 s_V(page) - E0
// is at most a small constant and the second product takes the bare values of the codes, exact in f16 (seven significant
// bits), with p' rounded to f16: 2^-12 of it, as fine as f16 outputs need.  The sum of the probabilities is
//     l = sum_j p'_j * 2^-e_j    in fp32, one product per page,
// and y = 2^E0 * (sum_j p'_j value_j) / l.  E0 is the exponent of the first page that a part looks at.  The maximum is
// raised only when it would grow by more than 2^8 (p' stays below that, far from f16's end), so the accumulators are
// hardly ever rescaled.
#pragma once

#include "dybit_cache.cuh"
#include "dybit_wait.cuh"

namespace dybit {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kRaise = 8.0f;

struct CacheAttn {
    const int *plan;             // counts
    const CacheTile *tiles, *comb;
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
    float *part_y;               // [slot][head][rows][dim] of parts
    float4 *part_ml;             // [slot][head][rows]: {m + E0, l, E0, -}
    int q_vec, q_vec16, y_vec;   // rows can be moved in pieces of 8 (16) bytes
};

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Two codes as a pair of f16 numbers: decode2 in f16 (1024 + c is exact, and the patterns add up to 36 << 10).
__device__ __forceinline__ __half2 as_half2(unsigned w) { return *reinterpret_cast<const __half2 *>(&w); }
__device__ __forceinline__ unsigned half2_bits(__half2 v) { return *reinterpret_cast<const unsigned *>(&v); }
__device__ __forceinline__ unsigned decode2_f16(unsigned w) {
    const __half2 h = as_half2((w & 0x007f007fu) | 0x64006400u);
    const unsigned g = half2_bits(__hfma2(h, as_half2(0xbc00bc00u), as_half2(0x64806480u)));           // 1152 - h = 128 - c
    const __half2 curve = as_half2(0x90009000u - g);
    const __half2 above = __hfma2_relu(h, as_half2(0xa000a000u), as_half2(0x48404840u));               // max(0, 8.5 - h / 128)
    return half2_bits(__hsub2(curve, above)) | (w & 0x80008000u);
}
template <typename T> __device__ __forceinline__ unsigned decode_pair(unsigned w);
template <> __device__ __forceinline__ unsigned decode_pair<__nv_bfloat16>(unsigned w) { return decode2<true>(w); }
template <> __device__ __forceinline__ unsigned decode_pair<__half>(unsigned w) { return decode2_f16(w); }

template <typename T>
__device__ __forceinline__ void mma_16816(float (&d)[4], const unsigned (&a)[4], unsigned b0, unsigned b1) {
    if constexpr (__is_same(T, __half)) {
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    } else {
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    }
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

// The keys [first, last) of this part of a tile whose rows are r0 .. r1 - 1, in units of `unit` keys.
struct KeyRange { int first, last; };
__device__ __forceinline__ KeyRange tile_keys(const CacheAttn &p, const CacheTile &t, int r0, int rows, int unit) {
    const RowKeys a = row_keys(p, t, r0), z = row_keys(p, t, min(r0 + rows, t.n * p.group) - 1);
    KeyRange k = {0, 0};
    if (z.hi <= a.lo) return k;                            // positions grow with the row
    const int u0 = a.lo / unit, u1 = cache_div_up(z.hi, unit), n = u1 - u0;
    k.first = (u0 + (int)((int64_t)n * t.split / t.splits)) * unit;
    k.last = (u0 + (int)((int64_t)n * (t.split + 1) / t.splits)) * unit;
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
    if (!DYBIT_CHECK(token < tile.n && d + 4 <= p.dim, 0x87)) return;
    if (p.y_vec) {
        *reinterpret_cast<uint2 *>(y) = make_uint2(pack2<T>(f0, f1), pack2<T>(f2, f3));
    } else {
        y[0] = from_f32<T>(f0), y[1] = from_f32<T>(f1), y[2] = from_f32<T>(f2), y[3] = from_f32<T>(f3);
    }
    if (d == 0 && p.lse != nullptr)
        p.lse[(int64_t)(tile.row + token) * (p.heads * p.group) + h] = l == 0.0f ? -INFINITY : (m + __log2f(l)) * kLn2;
}

// ------------------------------------------------------------------ tiles of 16 rows

constexpr int kSmThreads = 128, kSmWarps = 4;
constexpr int kSmKeys = 32;                  // keys of a stage: two boxes of 16
constexpr int kSmStages = 2;
constexpr int kSmSegment = 4096;             // keys whose page numbers and scales are held in shared memory at a time

template <int DP> __host__ __device__ constexpr int small_stage_bytes() { return 2 * kSmKeys * DP; }
template <int DP> __host__ __device__ constexpr int small_smem_bytes() { return kSmWarps * kSmStages * small_stage_bytes<DP>() + 1024; }

// What the score and value loops need of 16 keys.
struct KeyBlock { float c, e, f; int z, zv; };   // x's factor, values' exponent, 2^-e; coordinates page * heads + head of keys and values

// Four warps share a part's keys, 32 at a time each, with a ring of their own that the TMA fills; they meet at the end.
// A stage is read straight into the fragments of mma.sync: the contraction over head elements and the one over keys may
// run in any order, so a lane takes 16 consecutive codes of its key, and the keys of a block are ordered so that the
// swizzled reads of a quarter warp hit different banks (key_row).  Bound by HBM, then by instruction issue: a pair of
// codes takes 7 instructions and there is little else.
template <typename T, int DP>
__global__ void __launch_bounds__(kSmThreads, 3)
cache_small_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const CacheAttn p) {
    constexpr int KS = DP / 16;                            // matrix instructions along a head
    constexpr int X = DP / 8;                              // head elements of a lane's value column, and n-tiles of the output
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    __shared__ KeyBlock s_block[kSmSegment / 16];
    __shared__ uint64_t s_full[kSmWarps][kSmStages];
    __shared__ uint32_t s_abort;
    __shared__ float s_m[kSmWarps][16], s_l[kSmWarps][16];

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int item = (int)(blockIdx.x / (unsigned)p.heads), head = (int)(blockIdx.x - (unsigned)item * (unsigned)p.heads);
    if (threadIdx.x == 0) {
        for (int w = 0; w < kSmWarps; ++w)
            for (int s = 0; s < kSmStages; ++s) mbar_init(&s_full[w][s], 1);
        s_abort = 0;
        fence_mbar_init();
        prefetch_tensormap(&map_k);
        prefetch_tensormap(&map_v);
    }
    pdl_enter();
    if (item >= p.plan[1]) return;
    const CacheTile tile = p.tiles[item];
    const int r0 = tile.tile * kSmallRows, rows = min(kSmallRows, tile.n * p.group - r0);
    const KeyRange range = tile_keys(p, tile, r0, kSmallRows, kSmKeys);
    const int *table = p.table + tile.seq * p.table_stride;
    const RowKeys k0 = row_keys(p, tile, r0 + g), k1 = row_keys(p, tile, r0 + g + 8);
    // keys between these two are seen by every row that is there
    const int all_lo = row_keys(p, tile, r0 + rows - 1).lo, all_hi = row_keys(p, tile, r0).hi;

    // queries as fragments: k index 2t, 2t+1 (8+2t, 8+2t+1) of step j is element 16 * (t + 4 * (j / 4)) + 4 * (j % 4) + 0, 1 (2, 3)
    unsigned qf[KS][4];
    {
        const int ra = r0 + g, rb = ra + 8;
        auto row_at = [&](int r) {
            const int token = r / p.group, h = head * p.group + (r - token * p.group);
            return static_cast<const T *>(p.q) + (tile.row + token) * p.q_token + h * p.q_head;
        };
        const T *qa = g < rows ? row_at(ra) : nullptr, *qb = g + 8 < rows ? row_at(rb) : nullptr;
        auto four = [&](const T *q, int d) {
            uint2 v = make_uint2(0u, 0u);
            if (q != nullptr && d < p.dim) {
                if (p.q_vec) {
                    v = __ldg(reinterpret_cast<const uint2 *>(q + d));
                } else {
                    T e[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) e[i] = q[d + i];
                    memcpy(&v, e, 8);
                }
            }
            return v;
        };
#pragma unroll
        for (int j = 0; j < KS; ++j) {
            const int d = 16 * (t + 4 * (j / 4)) + 4 * (j % 4);
            const uint2 a = four(qa, d), b = four(qb, d);
            qf[j][0] = a.x, qf[j][1] = b.x, qf[j][2] = a.y, qf[j][3] = b.y;
        }
    }

    // exponent of the first page's value scale
    float e0 = 0.0f;
    if (range.last > range.first) {
        const int pg = __ldg(table + (range.first >> p.page_shift));
        const float s = (unsigned)pg < (uint64_t)p.pages ? __ldg(p.v_scales + (int64_t)pg * p.heads + head) : 0.0f;
        e0 = s > 0.0f ? (float)((int)((__float_as_uint(s) >> 23) & 255u) - 127) : 0.0f;
    }

    uint8_t *ring = smem + warp * (kSmStages * small_stage_bytes<DP>());
    float o[X][4];
#pragma unroll
    for (int i = 0; i < X; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.0f;
    float m0 = -INFINITY, m1 = -INFINITY, l0 = 0.0f, l1 = 0.0f;
    // n index g of a block of eight keys is key key_row(g): two neighbours lie four (DP 64: an odd number of) rows apart and
    // the rows of the even ones differ above their lowest bit, which makes both kinds of reads free of bank conflicts
    auto key_row = [](int i) {
        if constexpr (DP == 128) {
            const int h = i >> 1;
            return (2 * h + (h >> 1)) ^ ((i & 1) << 2);
        } else {
            const int h = i >> 1, even = (h & 1) | ((h & 2) << 1);
            return (i & 1) ? (even ^ 3) : even;
        }
    };
    const int kr = key_row(g), kv0 = key_row(2 * t), kv1 = key_row(2 * t + 1);
    uint32_t it = 0;                                       // stages used by this warp so far
    bool ok = true;

    for (int seg = range.first; seg < range.last; seg += kSmSegment) {
        const int seg_end = min(range.last, seg + kSmSegment);
        if (__syncthreads_and(ok) == 0) break;             // a wait that ran out ends the loop for all four warps
        for (int i = threadIdx.x; i < (seg_end - seg) / 16; i += kSmThreads) {
            const int key = seg + 16 * i;
            const int pg = key < tile.len ? __ldg(table + (key >> p.page_shift)) : -1;
            const int none = (int)(p.pages * p.heads);     // a coordinate outside the pool reads as zeros
            KeyBlock b = {0.0f, -INFINITY, 0.0f, none, none};                    // not there: seen by no row
            if ((unsigned)pg < (uint64_t)p.pages) {
                b.z = (int)((int64_t)pg * p.heads + head);
                const float ks = __ldg(p.k_scales + b.z), vs = __ldg(p.v_scales + b.z);
                b.c = ks * p.scale_log2;
                b.zv = vs > 0.0f ? b.z : none;
                b.e = vs > 0.0f ? (float)((int)((__float_as_uint(vs) >> 23) & 255u) - 127) - e0 : 0.0f;
                b.f = __uint_as_float((unsigned)(127 - max(-126, min(126, (int)b.e))) << 23);
            }
            s_block[i] = b;
        }
        __syncthreads();
        const int n_tiles = (seg_end - seg) / kSmKeys;
        auto fetch = [&](int i, uint32_t stage) {          // one lane
            uint8_t *dst = ring + stage * small_stage_bytes<DP>();
            uint64_t *bar = &s_full[warp][stage];
            mbar_arrive_expect_tx(bar, small_stage_bytes<DP>());
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const int z = s_block[2 * i + b].z, zv = s_block[2 * i + b].zv, y = (seg + kSmKeys * i + 16 * b) & ((1 << p.page_shift) - 1);
                tma_load_3d(dst + b * 16 * DP, &map_k, 0, y, z, bar);
                tma_load_3d(dst + (kSmKeys + b * 16) * DP, &map_v, 0, y, zv, bar);
            }
        };
        if (lane == 0) {
#pragma unroll
            for (int s = 0; s < kSmStages; ++s)
                if (warp + s * kSmWarps < n_tiles) fetch(warp + s * kSmWarps, (it + s) % kSmStages);
        }
        __syncwarp();
        for (int i = warp; i < n_tiles; i += kSmWarps, ++it) {
            const uint32_t stage = it % kSmStages;
            ok = __all_sync(0xffffffffu, wait_bounded(&s_full[warp][stage], (it / kSmStages) & 1u, &s_abort, 0x81));
            if (!ok) break;
            const uint8_t *ks = ring + stage * small_stage_bytes<DP>(), *vs = ks + kSmKeys * DP;
            const KeyBlock b0 = s_block[2 * i], b1 = s_block[2 * i + 1];
            float x[4][4];
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                const int row = n * 8 + kr;
                uint4 w[DP / 64];
                if constexpr (DP == 128) {
                    w[0] = *reinterpret_cast<const uint4 *>(ks + row * 128 + ((t ^ (row & 7)) << 4));
                    w[1] = *reinterpret_cast<const uint4 *>(ks + row * 128 + (((t + 4) ^ (row & 7)) << 4));
                } else {
                    w[0] = *reinterpret_cast<const uint4 *>(ks + row * 64 + ((t ^ ((row >> 1) & 3)) << 4));
                }
                x[n][0] = x[n][1] = x[n][2] = x[n][3] = 0.0f;
#pragma unroll
                for (int j = 0; j < KS; ++j) {
                    const uint4 &q4 = w[j / 4];
                    const unsigned c = j % 4 == 0 ? q4.x : j % 4 == 1 ? q4.y : j % 4 == 2 ? q4.z : q4.w;
                    mma_16816<T>(x[n], qf[j], decode_pair<T>(__byte_perm(c, 0u, 0x1100)), decode_pair<T>(__byte_perm(c, 0u, 0x3322)));
                }
            }
            // x[n][0], x[n][1]: row g, keys key_row(2t), key_row(2t + 1) of block n; x[n][2], x[n][3]: row g + 8
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                const float c = n < 2 ? b0.c : b1.c, e = n < 2 ? b0.e : b1.e;
#pragma unroll
                for (int k = 0; k < 4; ++k) x[n][k] = __fmaf_rn(x[n][k], c, e);
            }
            const int first = seg + kSmKeys * i;
            if (first < all_lo || first + kSmKeys > all_hi) {
#pragma unroll
                for (int n = 0; n < 4; ++n) {
                    const int ka = first + n * 8 + kv0, kb = first + n * 8 + kv1;
                    if (ka < k0.lo || ka >= k0.hi) x[n][0] = -INFINITY;
                    if (kb < k0.lo || kb >= k0.hi) x[n][1] = -INFINITY;
                    if (ka < k1.lo || ka >= k1.hi) x[n][2] = -INFINITY;
                    if (kb < k1.lo || kb >= k1.hi) x[n][3] = -INFINITY;
                }
            }
            float a0 = x[0][0], a1 = x[0][2];
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                a0 = fmaxf(a0, fmaxf(x[n][0], x[n][1]));
                a1 = fmaxf(a1, fmaxf(x[n][2], x[n][3]));
            }
#pragma unroll
            for (int d = 1; d < 4; d <<= 1) {
                a0 = fmaxf(a0, __shfl_xor_sync(0xffffffffu, a0, d));
                a1 = fmaxf(a1, __shfl_xor_sync(0xffffffffu, a1, d));
            }
            if (__any_sync(0xffffffffu, a0 > m0 + kRaise || a1 > m1 + kRaise)) {
                const float n0 = fmaxf(m0, a0), n1 = fmaxf(m1, a1);
                const float f0 = m0 == n0 ? 1.0f : ex2(m0 - n0), f1 = m1 == n1 ? 1.0f : ex2(m1 - n1);
                m0 = n0, m1 = n1;
                l0 *= f0, l1 *= f1;
#pragma unroll
                for (int d = 0; d < X; ++d) o[d][0] *= f0, o[d][1] *= f0, o[d][2] *= f1, o[d][3] *= f1;
            }
            const float u0 = m0 == -INFINITY ? 0.0f : m0, u1 = m1 == -INFINITY ? 0.0f : m1;
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                unsigned pf[4];
                float s0 = 0.0f, s1 = 0.0f;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    float(&v)[4] = x[2 * b + h];
                    v[0] = ex2(v[0] - u0), v[1] = ex2(v[1] - u0), v[2] = ex2(v[2] - u1), v[3] = ex2(v[3] - u1);
                    s0 += v[0] + v[1];
                    s1 += v[2] + v[3];
                    pf[2 * h] = pack_f16(v[0], v[1]);
                    pf[2 * h + 1] = pack_f16(v[2], v[3]);
                }
                const float f = b == 0 ? b0.f : b1.f;
                l0 = __fmaf_rn(s0, f, l0), l1 = __fmaf_rn(s1, f, l1);
                const int ra = b * 16 + kv0, rb = b * 16 + kv1;
                if constexpr (DP == 128) {
                    uint4 v[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int row = (k & 1 ? rb : ra) + (k >> 1) * 8;
                        v[k] = *reinterpret_cast<const uint4 *>(vs + row * 128 + ((g ^ (row & 7)) << 4));
                    }
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        unsigned c[4];
#pragma unroll
                        for (int k = 0; k < 4; ++k) c[k] = w == 0 ? v[k].x : w == 1 ? v[k].y : w == 2 ? v[k].z : v[k].w;
#pragma unroll
                        for (int y = 0; y < 4; ++y) {
                            const unsigned sel = 0x4400u + 0x1111u * y;
                            mma_16816<__half>(o[4 * w + y], pf, decode2_f16(__byte_perm(c[0], c[1], sel)), decode2_f16(__byte_perm(c[2], c[3], sel)));
                        }
                    }
                } else {
                    uint2 v[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int row = (k & 1 ? rb : ra) + (k >> 1) * 8;
                        v[k] = *reinterpret_cast<const uint2 *>(vs + row * 64 + (((g >> 1) ^ ((row >> 1) & 3)) << 4) + (g & 1) * 8);
                    }
#pragma unroll
                    for (int w = 0; w < 2; ++w) {
                        unsigned c[4];
#pragma unroll
                        for (int k = 0; k < 4; ++k) c[k] = w == 0 ? v[k].x : v[k].y;
#pragma unroll
                        for (int y = 0; y < 4; ++y) {
                            const unsigned sel = 0x4400u + 0x1111u * y;
                            mma_16816<__half>(o[4 * w + y], pf, decode2_f16(__byte_perm(c[0], c[1], sel)), decode2_f16(__byte_perm(c[2], c[3], sel)));
                        }
                    }
                }
            }
            __syncwarp();
            if (lane == 0 && i + kSmStages * kSmWarps < n_tiles) fetch(i + kSmStages * kSmWarps, stage);
        }
    }
    if (!ok) {                                             // copies in flight land before the block's memory is given up
        for (int i = 0; i < 64; ++i) __nanosleep(2000);
    }

    // the four warps' parts: maxima first, then the sums at the common maximum
#pragma unroll
    for (int d = 1; d < 4; d <<= 1) {
        l0 += __shfl_xor_sync(0xffffffffu, l0, d);
        l1 += __shfl_xor_sync(0xffffffffu, l1, d);
    }
    if (t == 0) {
        s_m[warp][g] = m0, s_m[warp][g + 8] = m1;
        s_l[warp][g] = l0, s_l[warp][g + 8] = l1;
    }
    __syncthreads();
    auto common = [&](int r) {
        float m = s_m[0][r];
#pragma unroll
        for (int w = 1; w < kSmWarps; ++w) m = fmaxf(m, s_m[w][r]);
        return m;
    };
    constexpr int LD = DP + 4;
    float *sum = reinterpret_cast<float *>(smem) + warp * 8 * LD;
    const int vecs = p.dim / 4;
#pragma unroll
    for (int half = 0; half < 2; ++half) {                 // rows 0 .. 7, then 8 .. 15: the ring holds one half of four warps
        if (half * 8 >= rows) break;
        const float m = common(g + 8 * half), mine = half == 0 ? m0 : m1;
        const float f = mine == -INFINITY ? 0.0f : ex2(mine - m);
        if (half == 1) __syncthreads();
#pragma unroll
        for (int i = 0; i < X; i += 4) {
            *reinterpret_cast<float4 *>(sum + g * LD + 2 * t * X + i) =
                make_float4(o[i][2 * half] * f, o[i + 1][2 * half] * f, o[i + 2][2 * half] * f, o[i + 3][2 * half] * f);
            *reinterpret_cast<float4 *>(sum + g * LD + (2 * t + 1) * X + i) =
                make_float4(o[i][2 * half + 1] * f, o[i + 1][2 * half + 1] * f, o[i + 2][2 * half + 1] * f, o[i + 3][2 * half + 1] * f);
        }
        __syncthreads();
        for (int i = threadIdx.x; i < 8 * vecs; i += kSmThreads) {
            const int lr = i / vecs, d = (i - lr * vecs) * 4, r = half * 8 + lr;
            if (r >= rows) break;
            float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
            float l = 0.0f;
            const float mr = common(r);
#pragma unroll
            for (int w = 0; w < kSmWarps; ++w) {
                const float4 v = *reinterpret_cast<const float4 *>(reinterpret_cast<float *>(smem) + (w * 8 + lr) * LD + d);
                s.x += v.x, s.y += v.y, s.z += v.z, s.w += v.w;
                l += s_m[w][r] == -INFINITY ? s_l[w][r] : s_l[w][r] * ex2(s_m[w][r] - mr);
            }
            if (tile.splits > 1) {
                const int64_t at = ((int64_t)tile.slot * p.heads + head) * kSmallRows + r;
                *reinterpret_cast<float4 *>(p.part_y + at * p.dim + d) = s;
                if (d == 0) p.part_ml[at] = make_float4(mr + e0, l, e0, 0.0f);
            } else {
                store_attention_row<T>(p, tile, head, r0 + r, d, s, l, mr, e0);
            }
        }
    }
}

// ------------------------------------------------------------------ parts of a tile, joined

// Sixteen rows of a tile and one key head: the parts at their common maximum.  part_ml.x is a part's maximum with its
// exponent in it, so that parts whose values have other scales compare.
template <typename T, int ROWS>
__global__ void __launch_bounds__(128) cache_join_kernel(const CacheAttn p) {
    pdl_enter();
    const int item = (int)(blockIdx.x / (unsigned)p.heads), head = (int)(blockIdx.x - (unsigned)item * (unsigned)p.heads);
    if (item >= p.plan[ROWS == kSmallRows ? 3 : 4]) return;
    const CacheTile tile = p.comb[item];
    const int r0 = blockIdx.y * 16, rows = min(ROWS, tile.n * p.group - tile.tile * ROWS), vecs = p.dim / 4;
    const int64_t step = (int64_t)p.heads * ROWS;
    for (int i = threadIdx.x; i < 16 * vecs; i += 128) {
        const int r = r0 + i / vecs, d = (i - i / vecs * vecs) * 4;
        if (r >= rows) break;
        const int64_t at = ((int64_t)tile.slot * p.heads + head) * ROWS + r;
        const float4 *ml = p.part_ml + at;
        const float *y = p.part_y + at * p.dim + d;
        float m = -INFINITY;
#pragma unroll 8
        for (int k = 0; k < tile.splits; ++k) m = fmaxf(m, __ldcg(ml + k * step).x);
        const float e = ml->z;
        float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
        float l = 0.0f;
#pragma unroll 8
        for (int k = 0; k < tile.splits; ++k) {
            const float4 a = __ldcg(ml + k * step), v = __ldcg(reinterpret_cast<const float4 *>(y + k * step * p.dim));
            const float w = a.x == -INFINITY ? 0.0f : ex2(a.x - m);
            s.x += v.x * w, s.y += v.y * w, s.z += v.z * w, s.w += v.w * w;
            l += (a.x == -INFINITY ? a.y : a.y * w) * ex2(e - a.z);
        }
        store_attention_row<T>(p, tile, head, tile.tile * ROWS + r, d, s, l, m - e, e);
    }
}

}  // namespace dybit
