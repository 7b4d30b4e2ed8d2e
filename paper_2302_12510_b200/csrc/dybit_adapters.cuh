// Low-rank adapters of many requests beside a shared projection, and their gradients.
//
//   forward    V_t = A_a x_t,             y_t  = base_t   + sum_r alpha_a V_t[r] B_a[r]
//   backward   U_t = alpha_a B_a dY_t,    dX_t = dXbase_t + sum_r U_t[r] A_a[r],
//              dA_a = sum_t U_t^T x^_t,   dB_a = sum_t alpha_a V_t^T dY_t
// With both factors rank-major the two lines that map tokens to tokens are one operator with the factors exchanged
// (adapter_tokens_kernel); the two gradients are one more (adapter_grad_kernel).
//
// All of it is bound by memory: a token costs 4 R multiplications per element read, R = 8 .. 128.  The products run on
// mma.sync, which takes its operands from registers: a tcgen05 tile would have to stage every element in shared memory
// (and the codes once more as bf16) for 128 x 8..64 outputs, and its 128 rows would be mostly empty in a decode step.
#pragma once

#include "dybit_adapters_plan.cuh"
#include "dybit_checkpoint.cuh"
#include "dybit_code8.cuh"
#include "dybit_sm100.cuh"

namespace dybit {

using namespace sm100;

// ------------------------------------------------------------------ matrix instructions on registers

template <typename TW>
__device__ __forceinline__ void mma16(float (&c)[4], unsigned a0, unsigned a1, unsigned a2, unsigned a3, unsigned b0, unsigned b1) {
    if constexpr (sizeof(TW) == 2 && __is_same(TW, __half)) {
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                     : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    } else {
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                     : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    }
}

__device__ __forceinline__ void mma8_tf32(float (&c)[4], unsigned a0, unsigned a1, unsigned a2, unsigned a3, unsigned b0, unsigned b1) {
    asm("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// What is left of x after its leading part `head`; nothing of an infinity (whose difference would be NaN).
__device__ __forceinline__ float rest_of(float x, float head) {
    return fabsf(x) == __uint_as_float(0x7f800000u) ? 0.0f : __fsub_rn(x, head);
}
// The nearest number of eleven significant bits (tf32); the largest fp32 numbers, whose nearest is an infinity, are cut off.
__device__ __forceinline__ float round_tf32(float x) {
    unsigned r;
    asm("cvt.rna.tf32.f32 %0, %1;" : "=r"(r) : "f"(x));
    const float cut = __uint_as_float(__float_as_uint(x) & 0xffffe000u);
    return fabsf(x) > 3.4e38f && fabsf(x) < __uint_as_float(0x7f800000u) ? cut : __uint_as_float(r);
}
__device__ __forceinline__ float top16(float x) { return __uint_as_float(__float_as_uint(x) & 0xffff0000u); }

// Two fp32 numbers as three pairs of bf16 whose sums they are (down to bf16's smallest numbers): eight significand bits cut
// off, the 16 that are left rounded to eight, and what that leaves, of either sign, which has no more than eight.
__device__ __forceinline__ void split3(float x, float y, unsigned &hi, unsigned &mid, unsigned &lo) {
    hi = __byte_perm(__float_as_uint(x), __float_as_uint(y), 0x7632);
    const float x1 = rest_of(x, top16(x)), y1 = rest_of(y, top16(y));
    mid = pack_bf16(x1, y1);
    lo = pack_bf16(__fsub_rn(x1, __uint_as_float(mid << 16)), __fsub_rn(y1, top16(__uint_as_float(mid))));
}

// ------------------------------------------------------------------ tokens -> tokens

struct AdapterTokens {
    const void *x;               // tokens x K
    int64_t ldx;
    const void *w1, *w2;         // n x R x K, n x R x N
    const float *alpha;
    const int *plan;
    const void *base;
    int64_t ldbase;
    void *y;
    int64_t ldy;
    float *v_out;                // forward: tokens x R, or null
    int64_t T, K, N;
    int n, R;
    int64_t perm_at, tiles_at;   // word offsets in the plan
    int64_t tiles_cap, steps_cap;                // what the plan's list and the fragments' buffers hold (range checks)
    int fast;                    // all rows start where vectors can be moved: 16 bytes in x and w1, four elements in w2, base and y
    int wide;                    // 16-bit y: rows of base and y start on 16-byte boundaries and hold whole vectors
    // backward: fragments for adapter_grad_kernel
    const float *v_in;
    const float *scales;
    int64_t scale_stride;
    uint4 *frag_u, *frag_v;
};

// A lane's sixteen elements of a 64-column block of a row, as raw words, zeros from column K on.  The order of columns
// inside a sum is free as long as both operands take the same: lane q takes runs of G elements, four lanes side by side
// (column (4i + q) * G + j of the block), with G the elements of x in 16 bytes.  FAST: rows start on 16-byte boundaries and
// hold whole runs.  Otherwise (G = 1) element loads without branches, so that all of them are in flight together.
template <typename T, int G, bool FAST>
__device__ __forceinline__ void load16(unsigned (&w)[4 * sizeof(T)], const T *row, int block, int q, int K) {
    if constexpr (FAST) {
        constexpr int kWords = G * (int)sizeof(T) / 4;         // of a run: 4, or 2 for a 16-bit factor beside an fp32 x
#pragma unroll
        for (int i = 0; i < 16 / G; ++i) {
            const int c = block * 64 + (4 * i + q) * G;
            if constexpr (kWords == 4) {
                const uint4 v = c < K ? __ldg(reinterpret_cast<const uint4 *>(row + c)) : make_uint4(0u, 0u, 0u, 0u);
                w[4 * i] = v.x;
                w[4 * i + 1] = v.y;
                w[4 * i + 2] = v.z;
                w[4 * i + 3] = v.w;
            } else {
                const uint2 v = c < K ? __ldg(reinterpret_cast<const uint2 *>(row + c)) : make_uint2(0u, 0u);
                w[2 * i] = v.x;
                w[2 * i + 1] = v.y;
            }
        }
    } else {
        T e[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int c = block * 64 + 4 * i + q;
            const T v = row[min(c, K - 1)];
            e[i] = c < K ? v : from_f32<T>(0.0f);
        }
#pragma unroll
        for (int i = 0; i < 4 * (int)sizeof(T); ++i) w[i] = reinterpret_cast<const unsigned *>(e)[i];
    }
}

// Four consecutive elements of a row, raw.
template <typename T> struct Quad { unsigned w[sizeof(T)]; };
template <typename T>
__device__ __forceinline__ Quad<T> zero_quad() {
    Quad<T> o;
#pragma unroll
    for (int j = 0; j < (int)sizeof(T); ++j) o.w[j] = 0u;
    return o;
}
// FAST: rows start on boundaries of four elements and hold whole quads.
template <typename T, bool FAST>
__device__ __forceinline__ Quad<T> load_quad(const T *row, int c, int cols) {
    Quad<T> o = zero_quad<T>();
    if constexpr (FAST) {
        if (c < cols) {
            if constexpr (sizeof(T) == 4) {
                const uint4 v = *reinterpret_cast<const uint4 *>(row + c);
                o.w[0] = v.x, o.w[1] = v.y, o.w[2] = v.z, o.w[3] = v.w;
            } else {
                const uint2 v = *reinterpret_cast<const uint2 *>(row + c);
                o.w[0] = v.x, o.w[1] = v.y;
            }
        }
    } else {
        T e[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const T v = row[min(c + j, cols - 1)];
            e[j] = c + j < cols ? v : from_f32<T>(0.0f);
        }
#pragma unroll
        for (int j = 0; j < (int)sizeof(T); ++j) o.w[j] = reinterpret_cast<const unsigned *>(e)[j];
    }
    return o;
}
template <typename T, bool FAST>
__device__ __forceinline__ void store_quad(T *row, int c, int cols, const float4 f) {
    if constexpr (FAST) {
        if (c < cols && DYBIT_CHECK(c + 4 <= cols, 0x78)) {
            if constexpr (sizeof(T) == 4) *reinterpret_cast<float4 *>(row + c) = f;
            else *reinterpret_cast<uint2 *>(row + c) = make_uint2(pack2<T>(f.x, f.y), pack2<T>(f.z, f.w));
        }
    } else {
        const float e[4] = {f.x, f.y, f.z, f.w};
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (c + j < cols) row[c + j] = from_f32<T>(e[j]);
    }
}
template <typename T>
__device__ __forceinline__ float4 quad_floats(const Quad<T> &v) {
    if constexpr (sizeof(T) == 4) {
        return make_float4(__uint_as_float(v.w[0]), __uint_as_float(v.w[1]), __uint_as_float(v.w[2]), __uint_as_float(v.w[3]));
    } else {
        const float2 a = unpack2<T>(v.w[0]), b = unpack2<T>(v.w[1]);
        return make_float4(a.x, a.y, b.x, b.y);
    }
}

template <typename T>
__device__ __forceinline__ void store4(T *row, int64_t c, int64_t cols, bool vec, const float4 f) {
    if (vec && c + 4 <= cols) {
        if constexpr (sizeof(T) == 4) *reinterpret_cast<float4 *>(row + c) = f;
        else *reinterpret_cast<uint2 *>(row + c) = make_uint2(pack2<T>(f.x, f.y), pack2<T>(f.z, f.w));
        return;
    }
    const float e[4] = {f.x, f.y, f.z, f.w};
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (c + j < cols) row[c + j] = from_f32<T>(e[j]);
}

__device__ __forceinline__ float4 ld_cluster_f4(uint32_t addr) {
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
__device__ __forceinline__ uint32_t cluster_nctarank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire;" ::: "memory"); }

// Fragments of a 16 (ranks) x 16 (tokens) block for adapter_grad_kernel: lane (g, q) of the reader takes ranks g, g + 8
// and tokens q, 4 + q, 8 + q, 12 + q; three uint4 (leading, middle and last bf16 parts) of 32 lanes follow one another.
__device__ __forceinline__ void store_fragment(uint4 *frag, int lane, const float (&f0)[4], const float (&f1)[4]) {
    uint4 part[3];
    split3(f0[0], f0[1], part[0].x, part[1].x, part[2].x);
    split3(f1[0], f1[1], part[0].y, part[1].y, part[2].y);
    split3(f0[2], f0[3], part[0].z, part[1].z, part[2].z);
    split3(f1[2], f1[3], part[0].w, part[1].w, part[2].w);
#pragma unroll
    for (int i = 0; i < 3; ++i) frag[i * 32 + lane] = part[i];
}

constexpr int kTokWarps = 8;
constexpr int kTokThreads = kTokWarps * 32;
constexpr int kMaxClusterCtas = 8;

template <int RT, int MT>
struct TokSmem {
    static constexpr int kTile = 16 * MT * RT;                 // floats of one token tile of V
    static constexpr int kFrag = MT * (RT / 16) * 4 * 128;     // words of its fragments for the second product (at most four parts)
    static constexpr int kWords = kTokWarps * kTile > kFrag ? kTokWarps * kTile : kFrag;       // the warps' sums make room for them
    static constexpr int kBytes = (kWords + kTile + (16 * MT * RT)) * 4;
};

// One cluster per tile of up to 16 * MT tokens of one adapter.  Its CTAs share the columns of x in the first product
// and those of y in the second; in between they sum up their parts of V through distributed shared memory.  RT is the
// rank rounded up (16, 32, 64, 128); ranks and columns that are missing are zeros, tokens that are missing repeat the
// tile's first one and are not stored.
//
// First product: a warp takes 64 columns at a time.  Lane (g = lane / 4, q = lane % 4) loads sixteen columns of token rows
// g, g + 8 and of factor rows g (+ 8 per n-tile) straight from memory and uses them as the four K = 16 slices of the
// fragment layout.
// Second product: V, scaled by alpha, enters it as an fp32 number whatever the type of y: three bf16 numbers that hold all
// of it, for f16 factors two tf32 numbers rounded to nearest (off by at most 2^-24 of V, as an fp32 number is itself).
// They are kept in shared memory as fragments.  The 64 columns of a warp are dealt to fragment columns so that a lane ends
// up with 16 bytes of consecutive ones and four lanes with 64.  The base is added to the finished sum by an fp32 addition
// rounded to nearest (in the accumulators the tensor core would cut it off).  It is fetched while the products run; one of 16
// bits in a tile of several slices, where a warp has many steps, a step ahead (8192 tokens bf16, four slices: 45.5 us; tiles of
// one slice are better off without the second set of registers: 256 tokens of 64 adapters 8.3 us, with it 8.8).
template <typename TX, typename TW, typename TY, int RT, int MT, bool BWD, bool FAST>
__global__ void __launch_bounds__(kTokThreads, RT <= 32 ? 2 : 1) adapter_tokens_kernel(const AdapterTokens p) {
    constexpr int NT = RT / 8, RB = RT / 16, TM = 16 * MT, XW = 4 * (int)sizeof(TX);
    constexpr int XB = sizeof(TX) == 4 || RT > 16 ? 1 : (MT < 2 ? MT : 2);     // 16-token slices whose loads are in flight together
    constexpr int WB = NT < 8 ? NT : 8;                                        // n-tiles of the factor in registers
    constexpr bool kBf16 = __is_same(TW, __nv_bfloat16);
    constexpr bool kHoldB = RT <= 32;                                          // the second factor stays in registers across slices
    constexpr int PARTS = kBf16 ? 3 : 4;                                       // fragments per 16 ranks
    constexpr int BREGS = kBf16 ? 2 : 4;                                       // registers of the second factor per n-tile and 16 ranks
    using Smem = TokSmem<RT, MT>;
    extern __shared__ __align__(16) float smem_f[];
    float *s_warp = smem_f;                                    // [warps][TM][RT]
    unsigned *s_frag = reinterpret_cast<unsigned *>(smem_f);   // the same words later: [MT][RB][PARTS][lane][4]
    float *s_part = smem_f + Smem::kWords;                     // [TM][RT], read by the whole cluster
    float *s_v = s_part + Smem::kTile;                         // [TM][RT]: alpha V (backward)
    __shared__ int s_token[TM];
    pdl_enter();
    const int cs = (int)cluster_nctarank(), rank = (int)cluster_ctarank();
    const int tile_id = (int)blockIdx.x / cs;
    constexpr int kList = MT == 1 ? 0 : (MT == 2 ? 1 : 2);
    if (tile_id >= p.plan[kList] || !DYBIT_CHECK(tile_id < p.tiles_cap, 0x73)) return;       // the whole cluster
    const AdapterTile tile = reinterpret_cast<const AdapterTile *>(p.plan + p.tiles_at)[tile_id];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
    const int R = p.R, K = (int)p.K, N = (int)p.N;
    if (!DYBIT_CHECK(tile.adapter < p.n && tile.start >= 0 && tile.count >= 1 && tile.count <= TM && (int64_t)tile.start + tile.count <= p.T, 0x74)) return;
    if (threadIdx.x < TM) s_token[threadIdx.x] = p.plan[p.perm_at + tile.start + ((int)threadIdx.x < tile.count ? (int)threadIdx.x : 0)];
    __syncthreads();
#ifdef DYBIT_DEBUG_BOUNDS
    if (__syncthreads_or(threadIdx.x < TM && !DYBIT_CHECK((unsigned)s_token[threadIdx.x] < p.T, 0x75))) return;      // the whole cluster: all see the same
#endif

    const int rblocks = tile.adapter >= 0 ? (R + 15) / 16 : 0;
    const TW *w2 = static_cast<const TW *>(p.w2) + (int64_t)max(tile.adapter, 0) * R * N;
    const int groups = (N + 63) / 64;
    // n-tile j = jh * 4 + jl, fragment column 2q' + b stands for column jh * 32 + b * 16 + q' * 4 + jl (y of 32 bits) or
    // b * 32 + q' * 8 + jh * 4 + jl (16 bits)
    constexpr bool kWide = sizeof(TY) == 2;
    constexpr int kJh = kWide ? 4 : 32, kCb = kWide ? 32 : 16, kCq = kWide ? 8 : 4;
    const int gcol = (g & 1) * kCb + (g >> 1) * kCq;           // the lane's columns as fragment column g: + jh * kJh + jl
    unsigned bq[kHoldB ? RB : 1][8][BREGS];                    // [16 ranks][n-tile jh * 4 + jl][fragment registers]
    auto load_b = [&](unsigned (&o)[8][BREGS], int rb, int n0) {
        // bf16: ranks 2q, 2q + 1, 2q + 8, 2q + 9 in pairs; f16: ranks q, q + 4, q + 8, q + 12 as floats
#pragma unroll
        for (int jh = 0; jh < 2; ++jh) {
            Quad<TW> r[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int rank_row = rb * 16 + (kBf16 ? 2 * q + (i & 1) + 8 * (i >> 1) : q + 4 * i);
                r[i] = rank_row < R ? load_quad<TW, FAST>(w2 + (int64_t)rank_row * N, n0 + jh * kJh + gcol, N) : zero_quad<TW>();
            }
#pragma unroll
            for (int jl = 0; jl < 4; ++jl) {
                if constexpr (kBf16) {
                    o[jh * 4 + jl][0] = __byte_perm(r[0].w[jl / 2], r[1].w[jl / 2], jl % 2 ? 0x7632 : 0x5410);
                    o[jh * 4 + jl][1] = __byte_perm(r[2].w[jl / 2], r[3].w[jl / 2], jl % 2 ? 0x7632 : 0x5410);
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float2 f = unpack2<TW>(r[i].w[jl / 2]);
                        o[jh * 4 + jl][i] = __float_as_uint(jl % 2 ? f.y : f.x);
                    }
                }
            }
        }
    };
    auto load_group = [&](int gi) {
        if constexpr (kHoldB) {
#pragma unroll
            for (int rb = 0; rb < RB; ++rb)
                if (rb < rblocks) load_b(bq[rb], rb, gi * 64);
        }
    };
    const int g_first = rank * kTokWarps + warp, g_step = cs * kTokWarps;

    if (tile.adapter >= 0) {
        // ---- V = x A^T over this CTA's columns, this warp's blocks of 64
        const TW *w1 = static_cast<const TW *>(p.w1) + (int64_t)tile.adapter * R * K;
        const int blocks = (K + 63) / 64, per = (blocks + cs - 1) / cs;
        const int last = min(blocks, (rank + 1) * per);
        float acc[MT][NT][4];
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[m][j][i] = 0.0f;
        for (int b = rank * per + warp; b < last; b += kTokWarps) {
#pragma unroll
            for (int j0 = 0; j0 < NT; j0 += WB) {
                unsigned w[WB][8];
#pragma unroll
                for (int j = 0; j < WB; ++j) {                 // (a missing rank reads row 0: its column of V is not used)
                    const int r = (j0 + j) * 8 + g;
                    load16<TW, 16 / (int)sizeof(TX), FAST>(w[j], w1 + (int64_t)(r < R ? r : 0) * K, b, q, K);
                }
#pragma unroll
                for (int m0 = 0; m0 < MT; m0 += XB) {
                    if (m0 * 16 >= tile.count) break;
                    unsigned x[XB][2][XW];
#pragma unroll
                    for (int m = 0; m < XB; ++m)
#pragma unroll
                        for (int h = 0; h < 2; ++h)
                            load16<TX, 16 / (int)sizeof(TX), FAST>(x[m][h], static_cast<const TX *>(p.x) + (int64_t)s_token[(m0 + m) * 16 + 8 * h + g] * p.ldx, b, q, K);
#pragma unroll
                    for (int m = 0; m < XB; ++m) {
                        const unsigned (&x0)[XW] = x[m][0], (&x1)[XW] = x[m][1];
#pragma unroll
                        for (int s = 0; s < 4; ++s) {
                            if constexpr (sizeof(TX) == 2) {
#pragma unroll
                                for (int j = 0; j < WB; ++j)
                                    mma16<TW>(acc[m0 + m][j0 + j], x0[2 * s], x1[2 * s], x0[2 * s + 1], x1[2 * s + 1], w[j][2 * s], w[j][2 * s + 1]);
                            } else {
                                unsigned a[4][3];
                                split3(__uint_as_float(x0[4 * s]), __uint_as_float(x0[4 * s + 1]), a[0][0], a[0][1], a[0][2]);
                                split3(__uint_as_float(x1[4 * s]), __uint_as_float(x1[4 * s + 1]), a[1][0], a[1][1], a[1][2]);
                                split3(__uint_as_float(x0[4 * s + 2]), __uint_as_float(x0[4 * s + 3]), a[2][0], a[2][1], a[2][2]);
                                split3(__uint_as_float(x1[4 * s + 2]), __uint_as_float(x1[4 * s + 3]), a[3][0], a[3][1], a[3][2]);
#pragma unroll
                                for (int i = 2; i >= 0; --i)
#pragma unroll
                                    for (int j = 0; j < WB; ++j)
                                        mma16<TW>(acc[m0 + m][j0 + j], a[0][i], a[1][i], a[2][i], a[3][i], w[j][2 * s], w[j][2 * s + 1]);
                            }
                        }
                    }
                }
            }
        }
        // ---- the second product's first operands are on their way while V is summed up
        if (g_first < groups) load_group(g_first);
        // ---- sum over the warps, then over the cluster
        float *mine = s_warp + warp * Smem::kTile;
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                *reinterpret_cast<float2 *>(mine + (m * 16 + g) * RT + j * 8 + 2 * q) = make_float2(acc[m][j][0], acc[m][j][1]);
                *reinterpret_cast<float2 *>(mine + (m * 16 + g + 8) * RT + j * 8 + 2 * q) = make_float2(acc[m][j][2], acc[m][j][3]);
            }
        __syncthreads();
        for (int i = threadIdx.x; i < Smem::kTile / 4; i += kTokThreads) {
            float4 s = reinterpret_cast<const float4 *>(s_warp)[i];
#pragma unroll
            for (int w = 1; w < kTokWarps; ++w) {
                const float4 o = reinterpret_cast<const float4 *>(s_warp + w * Smem::kTile)[i];
                s.x += o.x;
                s.y += o.y;
                s.z += o.z;
                s.w += o.w;
            }
            reinterpret_cast<float4 *>(s_part)[i] = s;
        }
        cluster_arrive();
        cluster_wait();
        const float alpha = p.alpha != nullptr ? __ldg(p.alpha + tile.adapter) : 1.0f;
        for (int i = threadIdx.x; i < Smem::kTile / 4; i += kTokThreads) {
            const uint32_t here = smem_u32(s_part + 4 * i);
            float4 part[kMaxClusterCtas];
#pragma unroll
            for (int c = 0; c < kMaxClusterCtas; ++c)
                if (c < cs) part[c] = ld_cluster_f4(mapa_u32(here, (uint32_t)c));
            float4 s = part[0];
#pragma unroll
            for (int c = 1; c < kMaxClusterCtas; ++c)
                if (c < cs) {
                    s.x += part[c].x;
                    s.y += part[c].y;
                    s.z += part[c].z;
                    s.w += part[c].w;
                }
            const int row = 4 * i / RT, r = 4 * i % RT;
            if (!BWD && p.v_out != nullptr && rank == 0 && row < tile.count && r < R)
                *reinterpret_cast<float4 *>(p.v_out + (int64_t)s_token[row] * R + r) = s;
            if (r >= R) s = make_float4(0.f, 0.f, 0.f, 0.f);
            const float v[4] = {alpha * s.x, alpha * s.y, alpha * s.z, alpha * s.w};
            if (BWD) *reinterpret_cast<float4 *>(s_v + row * RT + r) = make_float4(v[0], v[1], v[2], v[3]);
            unsigned *frag = s_frag + ((row / 16) * RB + r / 16) * (PARTS * 128);
            if constexpr (kBf16) {
                // register (row & 8) / 8 + 2 * (r & 8) / 8 of lane 4 * (row % 8) + (r % 8) / 2
#pragma unroll
                for (int j = 0; j < 4; j += 2) {
                    unsigned part3[3];
                    split3(v[j], v[j + 1], part3[0], part3[1], part3[2]);
                    unsigned *at = frag + ((row & 7) * 4 + ((r + j) & 7) / 2) * 4 + ((row >> 3) & 1) + 2 * ((r >> 3) & 1);
#pragma unroll
                    for (int c = 0; c < PARTS; ++c) at[c * 128] = part3[c];
                }
            } else {
                // part 2 * (slice of 8 ranks) + (0: leading, 1: rest); register (row & 8) / 8 + 2 * (r & 4) / 4 of lane 4 * (row % 8) + r % 4
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float hi = round_tf32(v[j]);
                    unsigned *at = frag + ((r >> 3) & 1) * 256 + ((row & 7) * 4 + j) * 4 + ((row >> 3) & 1) + 2 * ((r >> 2) & 1);
                    at[0] = __float_as_uint(hi);
                    at[128] = __float_as_uint(round_tf32(rest_of(v[j], hi)));
                }
            }
        }
        cluster_arrive();                                      // (waited for before the CTA leaves)
        __syncthreads();
        if constexpr (BWD) {
            // fragments of U (times the row's scale) and of alpha V for the other gradients, dealt out over the cluster
            const int steps = (tile.count + 15) / 16, mtr = (R + 15) / 16, half_items = steps * mtr;
            for (int i = rank + cs * warp; i < 2 * half_items; i += cs * kTokWarps) {
                const bool is_u = i < half_items;
                const int k = is_u ? i : i - half_items, st = k / mtr, m = k % mtr;
                float f[2][4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int row = st * 16 + 4 * e + q;
                    const int64_t t = s_token[row];
                    const float factor = is_u ? __ldg(p.scales + t * p.scale_stride) : alpha;
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const int r = m * 16 + g + 8 * h;
                        float v = 0.0f;
                        if (row < tile.count && r < R) v = factor * (is_u ? s_v[row * RT + r] : __ldg(p.v_in + t * R + r));
                        f[h][e] = v;
                    }
                }
                if (DYBIT_CHECK(tile.step >= 0 && tile.step + st < p.steps_cap, 0x76))
                    store_fragment((is_u ? p.frag_u : p.frag_v) + ((int64_t)(tile.step + st) * mtr + m) * 96, lane, f[0], f[1]);
            }
        }
    } else if (!BWD && p.v_out != nullptr && rank == 0) {
        for (int i = threadIdx.x; i < tile.count * R; i += kTokThreads) p.v_out[(int64_t)s_token[i / R] * R + i % R] = 0.0f;
    }

    // ---- y = base + V B over this CTA's groups of 64 columns
    constexpr bool kBaseAhead = sizeof(TY) == 2 && MT > 1;
    const bool wide_rows = p.wide != 0;
    Quad<TY> base[2][4];                                       // [row][jh * 2 + b]
    auto load_base = [&](int n0, int m) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const TY *row = static_cast<const TY *>(p.base) + (int64_t)s_token[m * 16 + g + 8 * h] * p.ldbase;
            if (p.base == nullptr) {
#pragma unroll
                for (int i = 0; i < 4; ++i) base[h][i] = zero_quad<TY>();
            } else if constexpr (kWide && FAST) {              // two quads side by side in one load
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    const int c = n0 + b * kCb + q * kCq;
                    if (wide_rows) {
                        const uint4 v = c < N ? *reinterpret_cast<const uint4 *>(row + c) : make_uint4(0u, 0u, 0u, 0u);
                        base[h][b].w[0] = v.x, base[h][b].w[1] = v.y, base[h][2 + b].w[0] = v.z, base[h][2 + b].w[1] = v.w;
                    } else {
                        base[h][b] = load_quad<TY, FAST>(row, c, N);
                        base[h][2 + b] = load_quad<TY, FAST>(row, c + kJh, N);
                    }
                }
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) base[h][i] = load_quad<TY, FAST>(row, n0 + (i >> 1) * kJh + (i & 1) * kCb + q * kCq, N);
            }
        }
    };
    if (kBaseAhead && g_first < groups) load_base(g_first * 64, 0);
    for (int gi = g_first; gi < groups; gi += g_step) {
        const int n0 = gi * 64;
        if (gi != g_first) load_group(gi);
#pragma unroll 1
        for (int m = 0; m < MT; ++m) {
            if (m * 16 >= tile.count) break;
            if (!kBaseAhead) load_base(n0, m);
            Quad<TY> mine[2][4];                               // 16 bits: this step's base, while the next one is on its way
            if constexpr (kBaseAhead) {
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int i = 0; i < 4; ++i) mine[h][i] = base[h][i];
                if (m + 1 < MT && (m + 1) * 16 < tile.count) load_base(n0, m + 1);
                else if (gi + g_step < groups) load_base((gi + g_step) * 64, 0);
            }
            float acc[8][4];
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[j][i] = -0.0f;   // (a token without an adapter keeps its base bit for bit)
            auto ranks16 = [&](const unsigned (&b)[8][BREGS], int rb) {
                const uint4 *frag = reinterpret_cast<const uint4 *>(s_frag + (m * RB + rb) * (PARTS * 128)) + lane;
                uint4 a[PARTS];
#pragma unroll
                for (int c = 0; c < PARTS; ++c) a[c] = frag[c * 32];
#pragma unroll
                for (int c = PARTS - 1; c >= 0; --c)
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        if constexpr (kBf16) mma16<__nv_bfloat16>(acc[j], a[c].x, a[c].y, a[c].z, a[c].w, b[j][0], b[j][1]);
                        else mma8_tf32(acc[j], a[c].x, a[c].y, a[c].z, a[c].w, b[j][2 * (c / 2)], b[j][2 * (c / 2) + 1]);
                    }
            };
            if constexpr (kHoldB) {
#pragma unroll
                for (int rb = 0; rb < RB; ++rb)
                    if (rb < rblocks) ranks16(bq[rb], rb);
            } else {
#pragma unroll 1
                for (int rb = 0; rb < rblocks; ++rb) {
                    load_b(bq[0], rb, n0);
                    ranks16(bq[0], rb);
                }
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if (m * 16 + g + 8 * h >= tile.count) continue;
                TY *row = static_cast<TY *>(p.y) + (int64_t)s_token[m * 16 + g + 8 * h] * p.ldy;
                float4 o[4];                                   // [jh * 2 + b]
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int j = (i >> 1) * 4, k = 2 * h + (i & 1);
                    const float4 f = quad_floats<TY>(kBaseAhead ? mine[h][i] : base[h][i]);
                    o[i] = make_float4(__fadd_rn(f.x, acc[j][k]), __fadd_rn(f.y, acc[j + 1][k]), __fadd_rn(f.z, acc[j + 2][k]),
                                       __fadd_rn(f.w, acc[j + 3][k]));
                }
                if constexpr (kWide && FAST) {
                    if (wide_rows) {
#pragma unroll
                        for (int b = 0; b < 2; ++b) {
                            const int c = n0 + b * kCb + q * kCq;
                            if (c < N && DYBIT_CHECK(c + 8 <= N, 0x77))
                                *reinterpret_cast<uint4 *>(row + c) = make_uint4(pack2<TY>(o[b].x, o[b].y), pack2<TY>(o[b].z, o[b].w),
                                                                                 pack2<TY>(o[2 + b].x, o[2 + b].y), pack2<TY>(o[2 + b].z, o[2 + b].w));
                        }
                        continue;
                    }
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) store_quad<TY, FAST>(row, n0 + (i >> 1) * kJh + (i & 1) * kCb + q * kCq, N, o[i]);
            }
        }
    }
    if (tile.adapter >= 0) cluster_wait();                     // the others may still read this CTA's part of V
}

// ------------------------------------------------------------------ gradients of the factors

enum class GradSrc { CodesSigned, CodesUnsigned, Bf16, F32 };

struct AdapterGradSide {
    const void *src;             // tokens x cols: codes or dY
    int64_t ld;                  // elements (bytes for codes)
    int64_t cols;
    const uint4 *frag;           // fragments of the left operand, by step
    float *out;                  // n x R x cols
    float *partial;              // partial slots x R x cols
    int vec;
};
struct AdapterGrad {
    AdapterGradSide side[2];     // 0: dA from the codes, 1: dB from dY
    const int *plan;
    int64_t T;
    int n, R;
    int64_t perm_at, chunks_at, offsets_at;      // word offsets in the plan
    int64_t steps_cap, partials_cap;             // what the fragments' and the partial sums' buffers hold (range checks)
    int blocks0;                 // blocks along x that belong to side 0
    int wc;                      // groups of 64 columns per block: 1, 2 or 4; the other warps share the tokens
    int chunk_slots;             // blocks along y that take chunks; n more look after adapters without tokens
};

// Eight columns of one token row as raw words: columns 8g .. 8g+7 of the warp's 64, for fp32 4g .. 4g+3 and 32 more.
template <GradSrc S> struct SrcWords { static constexpr int n = S == GradSrc::F32 ? 8 : (S == GradSrc::Bf16 ? 4 : 2); };
template <GradSrc S>
struct SrcRing {
    static constexpr int kElem = S == GradSrc::F32 ? 4 : (S == GradSrc::Bf16 ? 2 : 1);
    static constexpr int kPitch = 64 * kElem + 32;             // bytes of a row: the reads below meet no bank twice
    static constexpr int kStage = 16 * kPitch;
    static constexpr int kStages = S == GradSrc::F32 ? 3 : 4;
    static constexpr int kBytes = kTokWarps * kStages * kStage;
};
template <GradSrc S>
__device__ __forceinline__ void read_src8(unsigned (&w)[SrcWords<S>::n], const uint8_t *row, int g) {
    if constexpr (S == GradSrc::F32) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint4 v = *reinterpret_cast<const uint4 *>(row + g * 16 + i * 128);
            w[4 * i] = v.x, w[4 * i + 1] = v.y, w[4 * i + 2] = v.z, w[4 * i + 3] = v.w;
        }
    } else if constexpr (S == GradSrc::Bf16) {
        const uint4 v = *reinterpret_cast<const uint4 *>(row + g * 16);
        w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
    } else {
        const uint2 v = *reinterpret_cast<const uint2 *>(row + g * 8);
        w[0] = v.x, w[1] = v.y;
    }
}
// The same from memory where the row may be missing, end before the 64 columns or start anywhere: zeros for what is not there.
template <GradSrc S>
__device__ __forceinline__ void load_src8_any(unsigned (&w)[SrcWords<S>::n], const uint8_t *row, bool there, int64_t c0, int g, int64_t cols) {
    constexpr int W = SrcWords<S>::n;
    if constexpr (W == 2) {                                    // rows of codes are padded to 16: eight are always there
        w[0] = w[1] = 0u;
        if (there && c0 + 8 * g < cols) {
            const uint2 v = __ldg(reinterpret_cast<const uint2 *>(row + c0 + 8 * g));
            w[0] = v.x, w[1] = v.y;
        }
    } else {
        using T = typename Elem<S == GradSrc::F32 ? DYBIT_F32 : DYBIT_BF16>::type;
        T e[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int64_t c = c0 + (S == GradSrc::F32 ? j / 4 * 32 + 4 * g + j % 4 : 8 * g + j);
            const T v = reinterpret_cast<const T *>(row)[c < cols ? c : cols - 1];
            e[j] = there && c < cols ? v : from_f32<T>(0.0f);
        }
#pragma unroll
        for (int i = 0; i < W; ++i) w[i] = reinterpret_cast<const unsigned *>(e)[i];
    }
}

// Column j (0 .. 7) of two token rows as pairs of bf16: the number of parts it takes to hold them exactly.
template <GradSrc S> struct SrcParts { static constexpr int n = S == GradSrc::F32 ? 3 : 1; };
template <GradSrc S>
__device__ __forceinline__ void src_pair(unsigned (&o)[SrcParts<S>::n], const unsigned (&a)[SrcWords<S>::n], const unsigned (&b)[SrcWords<S>::n], int j) {
    if constexpr (S == GradSrc::F32) {
        split3(__uint_as_float(a[j]), __uint_as_float(b[j]), o[0], o[1], o[2]);
    } else if constexpr (S == GradSrc::Bf16) {
        o[0] = __byte_perm(a[j / 2], b[j / 2], j % 2 ? 0x7632 : 0x5410);
    } else {
        const unsigned w = __byte_perm(a[j / 4], b[j / 4], 0x4400u + (unsigned)(j % 4) * 0x1111u);   // code j of a twice, code j of b twice
        o[0] = decode2<S == GradSrc::CodesSigned>(w);
    }
}

// A pair of bf16 with zeros in the place of infinities and NaN.
__device__ __forceinline__ unsigned finite_pair(unsigned w) {
    return ((w & 0x7f80u) == 0x7f80u ? 0u : w & 0xffffu) | ((w & 0x7f800000u) == 0x7f800000u ? 0u : w & 0xffff0000u);
}

// acc += left (16 * MR ranks x 16 tokens) * src (16 tokens x 64 columns).  The products of two lower parts whose sum of places is
// above 2 are left out: each is below 2^-23 of the whole product, and since the last part has either sign they do not add up
// to a bias (a product's own rounding in fp32 is 2^-24).  The products that go into one accumulator follow each other at a
// distance: a matrix instruction takes dozens of clocks.
// APART: an infinity would meet the other side's lower parts as well, which may be 0, and 0 * infinity is NaN.  Leading parts
// that are not finite are multiplied with leading parts only (the lower parts of an infinity are 0).
template <GradSrc S, int MR, bool APART>
__device__ __forceinline__ void grad_multiply(float (&acc)[MR][8][4], const unsigned (&x)[4][SrcWords<S>::n], const uint4 (&f)[MR][3]) {
    constexpr int P = SrcParts<S>::n, JG = P == 1 ? 8 : 4;
#pragma unroll
    for (int j0 = 0; j0 < 8; j0 += JG) {
        unsigned b0[JG][P], b1[JG][P];
#pragma unroll
        for (int j = 0; j < JG; ++j) {
            src_pair<S>(b0[j], x[0], x[1], j0 + j);
            src_pair<S>(b1[j], x[2], x[3], j0 + j);
        }
#pragma unroll
        for (int i = 2; i >= 0; --i)
#pragma unroll
            for (int k = P - 1; k >= 0; --k)
#pragma unroll
                for (int m = 0; m < MR; ++m)
#pragma unroll
                    for (int j = 0; j < JG; ++j) {
                        if (i + k > 2) continue;
                        uint4 l = f[m][i];
                        unsigned r0 = b0[j][k], r1 = b1[j][k];
                        if (APART && i == 0 && k > 0) l = make_uint4(finite_pair(l.x), finite_pair(l.y), finite_pair(l.z), finite_pair(l.w));
                        if (APART && i > 0 && k == 0) r0 = finite_pair(r0), r1 = finite_pair(r1);
                        mma16<__nv_bfloat16>(acc[m][j0 + j], l.x, l.y, l.z, l.w, r0, r1);
                    }
    }
}

// Rows `row`, 4 + row, 8 + row, 12 + row of a chunk from memory.
template <GradSrc S>
__device__ __forceinline__ void load_step_any(unsigned (&x)[4][SrcWords<S>::n], const uint8_t *rows, int row_bytes, const int *perm, int64_t T, int row,
                                              int count, int64_t c0, int g, int64_t cols) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        int t = row + 4 * e < count ? __ldg(perm + row + 4 * e) : -1;
        if (!DYBIT_CHECK(t < T, 0x7a)) t = -1;
        load_src8_any<S>(x[e], rows + (int64_t)max(t, 0) * row_bytes, t >= 0, c0, g, cols);
    }
}

// A warp's sums once more, infinities kept apart: taken where the first ones are not all finite.
template <GradSrc S, int MR>
__device__ __noinline__ void adapter_grad_apart(float (&out)[MR][8][4], const uint8_t *rows, int row_bytes, const int *perm, int64_t T, int wt, int mine,
                                                int ntg, int count, int64_t c0, int64_t cols, const uint4 *frag, int r0, int mtr) {
    const int lane = threadIdx.x & 31;
    float acc[MR][8][4];
#pragma unroll
    for (int m = 0; m < MR; ++m)
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[m][j][i] = 0.0f;
    for (int i = 0; i < mine; ++i) {
        const int st = wt + i * ntg;
        unsigned x[4][SrcWords<S>::n];
        load_step_any<S>(x, rows, row_bytes, perm, T, st * 16 + (lane & 3), count, c0, lane >> 2, cols);
        uint4 f[MR][3];
#pragma unroll
        for (int m = 0; m < MR; ++m)
#pragma unroll
            for (int k = 0; k < 3; ++k)
                f[m][k] = MR == 1 || r0 + m < mtr ? __ldg(frag + (st * mtr + m) * 96 + k * 32) : make_uint4(0u, 0u, 0u, 0u);
        grad_multiply<S, MR, true>(acc, x, f);
    }
#pragma unroll
    for (int m = 0; m < MR; ++m)
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) out[m][j][i] = acc[m][j][i];
}

// sum over a chunk's tokens of left[r] * src[column]: 16 * MR ranks x 64 columns per warp.  The rows of a 16-token step
// travel by cp.async through a ring of the warp's own in shared memory, several steps ahead.  Lane (g, q) reads eight
// columns of rows q, 4 + q, 8 + q, 12 + q; two rows interleave into the fragment's K pairs (for codes that is the byte
// permutation that starts their decoding).
template <GradSrc S, int MR>
__device__ __forceinline__ void adapter_grad_body(const AdapterGrad &p, const AdapterGradSide &sd, int block, const AdapterChunk &ch, int r0, float *smem) {
    constexpr int W = SrcWords<S>::n;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
    const int wc = warp % p.wc, wt = warp / p.wc, ntg = kTokWarps / p.wc;
    const int64_t c0 = ((int64_t)block * p.wc + wc) * 64;
    const int mtr = (p.R + 15) / 16, count = min(ch.rest, kChunkTokens), steps = (count + 15) / 16;
    const bool fast = sd.vec && c0 + 64 <= sd.cols;
    const int *perm = p.plan + p.perm_at + ch.start;
    const uint4 *frag = sd.frag + ((int64_t)ch.step * mtr + r0) * 96 + lane;
    float acc[MR][8][4];
#pragma unroll
    for (int m = 0; m < MR; ++m)
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[m][j][i] = 0.0f;
    using Ring = SrcRing<S>;
    constexpr int kRuns = 16 * 4 * Ring::kElem / 32;           // 16-byte runs of a step per lane
    const int row_bytes = (int)(sd.ld * Ring::kElem);
    const uint8_t *rows = static_cast<const uint8_t *>(sd.src);
    uint8_t *ring = reinterpret_cast<uint8_t *>(smem) + warp * (Ring::kStages * Ring::kStage);
    constexpr bool kFragAhead = MR <= 2;                       // (four blocks of ranks leave no registers for it)
    uint4 a[kFragAhead ? 2 : 1][MR][3];
    auto load_left = [&](int st, uint4 (&f)[MR][3]) {
#pragma unroll
        for (int m = 0; m < MR; ++m)
#pragma unroll
            for (int i = 0; i < 3; ++i)
                f[m][i] = MR == 1 || r0 + m < mtr ? __ldg(frag + (st * mtr + m) * 96 + i * 32) : make_uint4(0u, 0u, 0u, 0u);
    };
    const int mine = wt < steps && c0 < sd.cols ? (steps - wt + ntg - 1) / ntg : 0;      // this warp's steps: wt, wt + ntg, ...
    if (fast) {
        // lane l holds the token of row l % 16 of the step that is fetched next; missing rows are zero-filled
        constexpr int kRowRuns = 4 * Ring::kElem;              // 16-byte runs of a row
        const int lane_row = lane / kRowRuns;
        const uint8_t *from = rows + c0 * Ring::kElem + lane % kRowRuns * 16;
        const uint32_t into = smem_u32(ring) + lane_row * Ring::kPitch + lane % kRowRuns * 16;
        const int *look = perm + wt * 16 + (lane & 15);        // of the step whose tokens are looked up next
        int look_rows = count - wt * 16, fill_rows = 0, fill = 0;
        auto token = [&]() {
            int t = (lane & 15) < look_rows ? __ldg(look) : 0;
            if (!DYBIT_CHECK((unsigned)t < p.T, 0x7a)) t = 0;
            look += ntg * 16;
            fill_rows = look_rows;
            look_rows -= ntg * 16;
            return t;
        };
        auto fetch = [&](int tok, int present) {
            if (present >= 16) {
#pragma unroll
                for (int k = 0; k < kRuns; ++k)
                    cp_async_16_full(into + fill + k * (32 / kRowRuns) * Ring::kPitch,
                                     from + (int64_t)__shfl_sync(0xffffffffu, tok, k * (32 / kRowRuns) + lane_row) * row_bytes);
            } else if (present > 0) {
#pragma unroll
                for (int k = 0; k < kRuns; ++k)
                    cp_async_16(into + fill + k * (32 / kRowRuns) * Ring::kPitch,
                                from + (int64_t)__shfl_sync(0xffffffffu, tok, k * (32 / kRowRuns) + lane_row) * row_bytes,
                                k * (32 / kRowRuns) + lane_row < present ? 16u : 0u);
            }
            cp_async_commit();
            fill = fill == (Ring::kStages - 1) * Ring::kStage ? 0 : fill + Ring::kStage;
        };
        int tok = token(), present = fill_rows;
#pragma unroll
        for (int i = 0; i < Ring::kStages - 1; ++i) {
            const int next = token(), next_rows = fill_rows;
            fetch(tok, present);
            tok = next, present = next_rows;
        }
        int drained = 0;
        if (kFragAhead && mine > 0) load_left(wt, a[0]);
        auto step = [&](int i, uint4 (&f)[MR][3], uint4 (&ahead)[MR][3]) {
            cp_async_wait_group<Ring::kStages - 2>();
            __syncwarp();                                      // the other lanes' copies too, and nobody still reads the stage refilled below
            const int next = token(), next_rows = fill_rows;
            fetch(tok, present);
            tok = next, present = next_rows;
            if (kFragAhead) {
                if (i + 1 < mine) load_left(wt + (i + 1) * ntg, ahead);
            } else {
                load_left(wt + i * ntg, f);
            }
            const uint8_t *stage = ring + drained + q * Ring::kPitch;
            drained = drained == (Ring::kStages - 1) * Ring::kStage ? 0 : drained + Ring::kStage;
            unsigned x[4][W];
#pragma unroll
            for (int e = 0; e < 4; ++e) read_src8<S>(x[e], stage + 4 * e * Ring::kPitch, g);
            grad_multiply<S, MR, false>(acc, x, f);
        };
        for (int i = 0; i < mine; i += 2) {
            step(i, a[0], a[kFragAhead]);
            if (i + 1 < mine) step(i + 1, a[kFragAhead], a[0]);
        }
        cp_async_wait_group<0>();
    }
    if (!fast) {
        for (int i = 0; i < mine; ++i) {
            const int st = wt + i * ntg;
            unsigned x[4][W];
            load_step_any<S>(x, rows, row_bytes, perm, p.T, st * 16 + q, count, c0, g, sd.cols);
            load_left(st, a[0]);
            grad_multiply<S, MR, false>(acc, x, a[0]);
        }
    }
    if constexpr (S == GradSrc::F32 || S == GradSrc::Bf16) {   // (codes are finite and have one part)
        bool finite = true;
#pragma unroll
        for (int m = 0; m < MR; ++m)
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) finite = finite && fabsf(acc[m][j][i]) < __uint_as_float(0x7f800000u);
        if (__any_sync(0xffffffffu, !finite)) {
            float again[MR][8][4];
            adapter_grad_apart<S, MR>(again, rows, row_bytes, perm, p.T, wt, mine, ntg, count, c0, sd.cols, frag, r0, mtr);
#pragma unroll
            for (int m = 0; m < MR; ++m)
#pragma unroll
                for (int j = 0; j < 8; ++j)
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[m][j][i] = again[m][j][i];
        }
    }
    // the token groups' sums meet in shared memory, added in order
    constexpr int kWarpTile = MR * 16 * 64;
    if (ntg > 1) {
        __syncthreads();                                       // the rings make room
        if (wt > 0) {
            float *mine = smem + (size_t)((wt - 1) * p.wc + wc) * kWarpTile;
#pragma unroll
            for (int m = 0; m < MR; ++m)
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    *reinterpret_cast<float4 *>(mine + ((m * 8 + j) * 32 + lane) * 4) = make_float4(acc[m][j][0], acc[m][j][1], acc[m][j][2], acc[m][j][3]);
        }
        __syncthreads();
        if (wt > 0) return;
        for (int o = 1; o < ntg; ++o) {
            const float *other = smem + (size_t)((o - 1) * p.wc + wc) * kWarpTile;
#pragma unroll
            for (int m = 0; m < MR; ++m)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float4 f = *reinterpret_cast<const float4 *>(other + ((m * 8 + j) * 32 + lane) * 4);
                    acc[m][j][0] += f.x;
                    acc[m][j][1] += f.y;
                    acc[m][j][2] += f.z;
                    acc[m][j][3] += f.w;
                }
        }
    }
    const bool whole = ch.index == 0 && ch.rest <= kChunkTokens;
    float *out = whole ? sd.out + (int64_t)ch.adapter * p.R * sd.cols
                       : sd.partial + (int64_t)(ch.partial + ch.index) * p.R * sd.cols;
    const bool vec = sd.cols % 4 == 0 && aligned16(out);
#pragma unroll
    for (int m = 0; m < MR; ++m)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int r = (r0 + m) * 16 + g + 8 * h;
            if (r >= p.R) continue;
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int j = 0; j < 8; j += 4) {
                    const int64_t c = c0 + (S == GradSrc::F32 ? j * 8 + (2 * q + b) * 4 : (2 * q + b) * 8 + j);
                    if (c < sd.cols)
                        store4<float>(out + (int64_t)r * sd.cols, c, sd.cols, vec,
                                  make_float4(acc[m][j][2 * h + b], acc[m][j + 1][2 * h + b], acc[m][j + 2][2 * h + b], acc[m][j + 3][2 * h + b]));
                }
        }
}

// blockIdx: x = columns (side 0, then side 1), y = chunk (then adapters without tokens, whose gradients are zero),
// z = ranks beyond 16 * MR.
template <GradSrc S0, GradSrc S1, int MR>
__global__ void __launch_bounds__(kTokThreads, MR == 1 ? 2 : 1) adapter_grad_kernel(const __grid_constant__ AdapterGrad p) {
    extern __shared__ __align__(16) float smem_f[];
    pdl_enter();
    const int r0 = (int)blockIdx.z * MR;
    const bool first = (int)blockIdx.x < p.blocks0;
    const int block = (int)blockIdx.x - (first ? 0 : p.blocks0);
    if ((int)blockIdx.y >= p.chunk_slots) {
        const int a = (int)blockIdx.y - p.chunk_slots;
        const int *off = p.plan + p.offsets_at + (int64_t)a * kPlanColumns;
        if (off[kPlanColumns] != off[0]) return;
        const int64_t cols = p.side[first ? 0 : 1].cols, width = 64 * p.wc;
        float *out = p.side[first ? 0 : 1].out + (int64_t)a * p.R * cols;
        for (int64_t i = threadIdx.x; i < 16 * MR * width; i += kTokThreads) {
            const int64_t r = r0 * 16 + i / width, c = (int64_t)block * width + i % width;
            if (r < p.R && c < cols) out[r * cols + c] = 0.0f;
        }
        return;
    }
    if ((int)blockIdx.y >= p.plan[3]) return;
    const AdapterChunk ch = reinterpret_cast<const AdapterChunk *>(p.plan + p.chunks_at)[blockIdx.y];
    if (!DYBIT_CHECK((unsigned)ch.adapter < (unsigned)p.n && ch.start >= 0 && ch.rest >= 1 && (int64_t)ch.start + min(ch.rest, kChunkTokens) <= p.T &&
                         ch.step >= 0 && ch.step + (min(ch.rest, kChunkTokens) + 15) / 16 <= p.steps_cap &&
                         ((ch.index == 0 && ch.rest <= kChunkTokens) || (ch.index >= 0 && ch.partial >= 0 && ch.partial + ch.index < p.partials_cap)), 0x79))
        return;
    if (first) adapter_grad_body<S0, MR>(p, p.side[0], block, ch, r0, smem_f);
    else adapter_grad_body<S1, MR>(p, p.side[1], block, ch, r0, smem_f);
}

// Adapters that several blocks worked on: their sums, added in order.
__global__ void __launch_bounds__(256) adapter_grad_sum_kernel(const __grid_constant__ AdapterGrad p) {
    pdl_enter();
    const int a = blockIdx.y;
    const int *off = p.plan + p.offsets_at + (int64_t)a * kPlanColumns;
    const int parts = off[kPlanColumns + 4] - off[4], first = off[5];
    if (parts <= 1 || !DYBIT_CHECK(first >= 0 && first + parts <= p.partials_cap, 0x7b)) return;
    for (int s = 0; s < 2; ++s) {
        const AdapterGradSide &sd = p.side[s];
        const int64_t size = p.R * sd.cols;                    // a multiple of 8
        for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < size / 4; i += (int64_t)gridDim.x * 256) {
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
            for (int c = 0; c < parts; ++c) {
                const float4 o = __ldcg(reinterpret_cast<const float4 *>(sd.partial + (int64_t)(first + c) * size) + i);
                v.x += o.x;
                v.y += o.y;
                v.z += o.z;
                v.w += o.w;
            }
            float *dst = sd.out + a * size + 4 * i;
            if (aligned16(dst)) {
                *reinterpret_cast<float4 *>(dst) = v;
            } else {
                dst[0] = v.x;
                dst[1] = v.y;
                dst[2] = v.z;
                dst[3] = v.w;
            }
        }
    }
}

// ------------------------------------------------------------------ host side

// Lets a kernel use `bytes` of dynamic shared memory; once per kernel and device.
static dybit_status allow_smem(const void *kernel, int bytes, std::atomic<bool> *ready) {
    int dev = 0;
    DYBIT_CUDA_TRY(cudaGetDevice(&dev));
    if (dev < 0 || dev >= 64) return DYBIT_ERR_CUDA;
    if (!ready[dev].load(std::memory_order_acquire)) {
        DYBIT_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes));
        ready[dev].store(true, std::memory_order_release);
    }
    return DYBIT_OK;
}

static bool rows_vec(const void *p, int64_t ld, int elem, int bytes) { return aligned(p, bytes) && (ld * elem) % bytes == 0; }

template <typename TX, typename TW, typename TY, int RT, int MT, bool BWD, bool FAST>
static dybit_status launch_tokens_inst(AdapterTokens p, int cs, cudaStream_t s) {
    auto kern = adapter_tokens_kernel<TX, TW, TY, RT, MT, BWD, FAST>;
    constexpr int smem = TokSmem<RT, MT>::kBytes;
    static std::atomic<bool> ready[64];
    const dybit_status st = allow_smem(reinterpret_cast<const void *>(kern), smem, ready);
    if (st != DYBIT_OK) return st;
    const PlanLayout L(p.T, p.n);
    constexpr int kList = MT == 1 ? 0 : (MT == 2 ? 1 : 2);
    p.perm_at = L.perm, p.tiles_at = L.tiles[kList], p.tiles_cap = L.tiles_cap[kList], p.steps_cap = L.steps_cap;
    const int64_t blocks = L.tiles_cap[kList] * cs;
    if (blocks > 0x7fffffff) return DYBIT_ERR_UNSUPPORTED;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)blocks);
    cfg.blockDim = dim3(kTokThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)cs;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    (void)cudaLaunchKernelEx(&cfg, kern, p);
    return launch_status();
}

template <typename TX, typename TW, typename TY, int RT, int MT, bool BWD>
static dybit_status launch_tokens(const AdapterTokens &p, int cs, cudaStream_t s) {
    return p.fast ? launch_tokens_inst<TX, TW, TY, RT, MT, BWD, true>(p, cs, s) : launch_tokens_inst<TX, TW, TY, RT, MT, BWD, false>(p, cs, s);
}

template <typename TX, typename TW, typename TY, bool BWD>
static dybit_status launch_tokens_rank(const AdapterTokens &p, cudaStream_t s) {
    const PlanLayout L(p.T, p.n);
    // CTAs of a tile: enough of them to give every SM most of two, but at least four of the 64-column blocks to each
    const int64_t widest = ((p.K > p.N ? p.K : p.N) + 63) / 64;
    auto cluster = [&](int64_t tiles) {
        int cs = 1;
        while (cs < kMaxClusterCtas && cs * 4 < widest && tiles * cs * 4 < (int64_t)sm_count() * 7) cs *= 2;
        return cs;
    };
    const int c1 = cluster(L.tiles_cap[0]), c2 = cluster(L.tiles_cap[1]), c4 = cluster(L.tiles_cap[2]);
    // tiles of several 16-token slices read the factors once for all of them: taken where adapters have that many tokens
    // and the tiles still fill the device
    const bool many = p.T >= 32 * (int64_t)p.n, four = many && L.tiles_cap[2] * c4 >= sm_count(), two = many && L.tiles_cap[1] * c2 >= sm_count();
    if (p.R <= 16) return four ? launch_tokens<TX, TW, TY, 16, 4, BWD>(p, c4, s) : launch_tokens<TX, TW, TY, 16, 1, BWD>(p, c1, s);
    if (p.R <= 32) return two ? launch_tokens<TX, TW, TY, 32, 2, BWD>(p, c2, s) : launch_tokens<TX, TW, TY, 32, 1, BWD>(p, c1, s);
    if (p.R <= 64) return two ? launch_tokens<TX, TW, TY, 64, 2, BWD>(p, c2, s) : launch_tokens<TX, TW, TY, 64, 1, BWD>(p, c1, s);
    return launch_tokens<TX, TW, TY, 128, 1, BWD>(p, c1, s);
}

// Whether the gradient kernel's grid can hold the problem: chunks and adapters along y, at most blocks of 64 columns along x.
// Asked before anything is launched.
inline bool grad_grid_ok(int64_t T, int64_t K, int64_t N, int n) {
    return PlanLayout(T, n).chunks_cap + n <= 65535 && (K + 63) / 64 + (N + 63) / 64 <= 0x7fffffff;
}

constexpr int kMaxGradSmem = (kTokWarps - 1) * 4 * 16 * 64 * 4;      // four blocks of ranks, one group of columns

template <GradSrc S0, GradSrc S1, int MR>
static dybit_status launch_grad_ranks(const AdapterGrad &p, dim3 grid, int smem, cudaStream_t s) {
    static std::atomic<bool> ready[64];
    auto kern = adapter_grad_kernel<S0, S1, MR>;
    const dybit_status st = allow_smem(reinterpret_cast<const void *>(kern), kMaxGradSmem, ready);
    if (st != DYBIT_OK) return st;
    launch_k(kern, grid, dim3(kTokThreads), (size_t)smem, s, p);
    return launch_status();
}

template <GradSrc S0, GradSrc S1>
static dybit_status launch_grad(const AdapterGrad &p_in, cudaStream_t s) {
    AdapterGrad p = p_in;
    const PlanLayout L(p.T, p.n);
    p.perm_at = L.perm, p.chunks_at = L.chunks, p.offsets_at = L.offsets, p.steps_cap = L.steps_cap, p.partials_cap = L.partials_cap;
    const int mtr = (p.R + 15) / 16, mr = mtr >= 3 ? 4 : mtr, z = (mtr + mr - 1) / mr;
    // wide blocks read longer runs of a row and the left operand less often, as far as the device stays full
    const int64_t fill = (int64_t)sm_count() * 3 / 2;
    p.wc = 4;
    auto blocks = [&](int side) { return (p.side[side].cols + 64 * p.wc - 1) / (64 * p.wc); };
    while (p.wc > 1 && (blocks(0) + blocks(1)) * L.chunks_cap * z < fill) p.wc /= 2;
    p.blocks0 = (int)blocks(0);
    p.chunk_slots = (int)L.chunks_cap;
    const int64_t bx = blocks(0) + blocks(1), by = L.chunks_cap + p.n;      // (within the grid's limits: grad_grid_ok)
    constexpr int kRing = SrcRing<S1>::kBytes > SrcRing<S0>::kBytes ? SrcRing<S1>::kBytes : SrcRing<S0>::kBytes;
    const int sums = (kTokWarps - p.wc) * mr * 16 * 64 * 4, smem = sums > kRing ? sums : kRing;
    const dim3 grid((unsigned)bx, (unsigned)by, (unsigned)z);
    dybit_status st;
    if (mr == 1) st = launch_grad_ranks<S0, S1, 1>(p, grid, smem, s);
    else if (mr == 2) st = launch_grad_ranks<S0, S1, 2>(p, grid, smem, s);
    else st = launch_grad_ranks<S0, S1, 4>(p, grid, smem, s);
    if (st != DYBIT_OK || p.T <= kChunkTokens) return st;       // no adapter has several parts
    const int64_t most = p.side[0].cols > p.side[1].cols ? p.side[0].cols : p.side[1].cols;
    int64_t bs = (p.R * most / 4 + 255) / 256, cap = 8 * (int64_t)sm_count() / p.n + 1;
    if (bs > cap) bs = cap;
    launch_k(adapter_grad_sum_kernel, dim3((unsigned)bs, (unsigned)p.n), dim3(256), 0, s, p);
    return launch_status();
}

static dybit_status check_adapters(int64_t T, int64_t K, int64_t N, int R, int n, const void *A, const void *B, dybit_dtype tw,
                                   const float *alpha, const void *plan) {
    if (T < 0 || K < 1 || N < 1 || K > 0x7fffffff || N > 0x7fffffff || R < 8 || dybit_adapters_plan_bytes(T, n) == 0) return DYBIT_ERR_INVALID_ARG;
    if (R % 8 != 0 || R > DYBIT_MAX_RANK) return DYBIT_ERR_UNSUPPORTED;
    if (A == nullptr || B == nullptr || plan == nullptr) return DYBIT_ERR_INVALID_ARG;
    if (!dtype_ok(tw)) return DYBIT_ERR_INVALID_ARG;
    if (!aligned(A, 2) || !aligned(B, 2) || !aligned(plan, 16) || !aligned(alpha, 4)) return DYBIT_ERR_ALIGNMENT;
    return DYBIT_OK;
}

struct BackwardWs {
    int64_t frag_u, frag_v, partial_a, partial_b, bytes;
    BackwardWs(int64_t T, int64_t K, int64_t N, int R, int n) {
        const PlanLayout L(T, n);
        const int64_t frag = L.steps_cap * ((R + 15) / 16) * 3 * 512;
        int64_t at = 0;
        frag_u = at, at += round_up(frag, 1024);
        frag_v = at, at += round_up(frag, 1024);
        partial_a = at, at += round_up(L.partials_cap * R * K * 4, 1024);
        partial_b = at, at += round_up(L.partials_cap * R * N * 4, 1024);
        bytes = at + 1024;
    }
};

}  // namespace dybit

extern "C" {

dybit_status dybit_adapters(int64_t T, int64_t K, int64_t N, int R, const void *X, dybit_dtype tx, int64_t ldx,
                            int n_adapters, const void *A, const void *B, dybit_dtype tw, const float *alpha,
                            const void *plan, const void *base, int64_t ldbase, dybit_dtype ty, void *Y, int64_t ldy,
                            float *V, void *stream) {
    using namespace dybit;
    dybit_status st = check_adapters(T, K, N, R, n_adapters, A, B, tw, alpha, plan);
    if (st != DYBIT_OK) return st;
    if (!dtype_ok(tx) || !dtype_ok(ty) || ldx < K || ldy < N || (base != nullptr && ldbase < N)) return DYBIT_ERR_INVALID_ARG;
    if (!((tx == DYBIT_F32 && tw == DYBIT_BF16) || (tx != DYBIT_F32 && tw == tx)) || !(ty == DYBIT_F32 || ty == tx)) return DYBIT_ERR_UNSUPPORTED;
    if (T == 0) return DYBIT_OK;
    if (X == nullptr || Y == nullptr) return DYBIT_ERR_INVALID_ARG;
    const int ex = dtype_bytes(tx), ey = dtype_bytes(ty);
    if (!aligned(X, ex) || !aligned(Y, ey) || !aligned(base, ey) || !aligned(V, 16)) return DYBIT_ERR_ALIGNMENT;
    AdapterTokens p = {};
    p.x = X, p.ldx = ldx, p.w1 = A, p.w2 = B, p.alpha = alpha, p.plan = static_cast<const int *>(plan);
    p.base = base, p.ldbase = ldbase, p.y = Y, p.ldy = ldy, p.v_out = V;
    p.T = T, p.K = K, p.N = N, p.n = n_adapters, p.R = R;
    p.fast = rows_vec(X, ldx, ex, 16) && rows_vec(A, K, 2, 16) && rows_vec(B, N, 2, 8) && rows_vec(Y, ldy, ey, 4 * ey) &&
             (base == nullptr || rows_vec(base, ldbase, ey, 4 * ey));
    p.wide = N % 8 == 0 && rows_vec(Y, ldy, ey, 16) && (base == nullptr || rows_vec(base, ldbase, ey, 16));
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (tx == DYBIT_F32) return launch_tokens_rank<float, __nv_bfloat16, float, false>(p, s);
    if (tx == DYBIT_BF16)
        return ty == DYBIT_F32 ? launch_tokens_rank<__nv_bfloat16, __nv_bfloat16, float, false>(p, s)
                               : launch_tokens_rank<__nv_bfloat16, __nv_bfloat16, __nv_bfloat16, false>(p, s);
    return ty == DYBIT_F32 ? launch_tokens_rank<__half, __half, float, false>(p, s) : launch_tokens_rank<__half, __half, __half, false>(p, s);
}

size_t dybit_adapters_backward_workspace_bytes(int64_t T, int64_t K, int64_t N, int R, int n_adapters) {
    if (dybit_adapters_plan_bytes(T, n_adapters) == 0 || K < 1 || N < 1 || R < 8 || R % 8 != 0 || R > DYBIT_MAX_RANK) return 0;
    return (size_t)dybit::BackwardWs(T, K, N, R, n_adapters).bytes;
}

dybit_status dybit_adapters_backward(int64_t T, int64_t K, int64_t N, int R, const void *dY, dybit_dtype tdy, int64_t lddy,
                                     const void *codes, int64_t row_stride_bytes, dybit_fmt fmt, const float *scales,
                                     int64_t scale_stride, int n_adapters, const void *A, const void *B,
                                     dybit_dtype tw, const float *alpha, const void *plan, const float *V,
                                     const void *dXbase, int64_t lddxbase, void *dX, int64_t lddx, float *dA,
                                     float *dB, void *ws, size_t ws_bytes, void *stream) {
    using namespace dybit;
    dybit_status st = check_adapters(T, K, N, R, n_adapters, A, B, tw, alpha, plan);
    if (st != DYBIT_OK) return st;
    st = check_codes(codes, T, K, row_stride_bytes, fmt);
    if (st != DYBIT_OK) return st;
    if (!dtype_ok(tdy) || lddy < N || lddx < K || (dXbase != nullptr && lddxbase < K) || scale_stride < 0) return DYBIT_ERR_INVALID_ARG;
    if (tdy == DYBIT_F16 || tw != DYBIT_BF16) return DYBIT_ERR_UNSUPPORTED;
    if (row_stride_bytes > 0x7fffffff || lddy > 0x7fffffff / dtype_bytes(tdy) || !grad_grid_ok(T, K, N, n_adapters)) return DYBIT_ERR_UNSUPPORTED;
    if (dA == nullptr || dB == nullptr) return DYBIT_ERR_INVALID_ARG;
    if (T > 0 && (dY == nullptr || dX == nullptr || V == nullptr || scales == nullptr)) return DYBIT_ERR_INVALID_ARG;
    const int e = dtype_bytes(tdy);
    if (!aligned(dY, e) || !aligned(dX, e) || !aligned(dXbase, e) || !aligned(V, 4) || !aligned(scales, 4) || !aligned(dA, 4) ||
        !aligned(dB, 4) || !aligned(ws, 1024))
        return DYBIT_ERR_ALIGNMENT;
    const BackwardWs w(T, K, N, R, n_adapters);
    if (ws == nullptr || ws_bytes < (size_t)w.bytes) return DYBIT_ERR_WORKSPACE;
    uint8_t *base = static_cast<uint8_t *>(ws);
    cudaStream_t s = static_cast<cudaStream_t>(stream);

    AdapterTokens p = {};
    p.x = dY, p.ldx = lddy, p.w1 = B, p.w2 = A, p.alpha = alpha, p.plan = static_cast<const int *>(plan);
    p.base = dXbase, p.ldbase = lddxbase, p.y = dX, p.ldy = lddx;
    p.T = T, p.K = N, p.N = K, p.n = n_adapters, p.R = R;
    p.fast = rows_vec(dY, lddy, e, 16) && rows_vec(B, N, 2, 16) && rows_vec(A, K, 2, 8) && rows_vec(dX, lddx, e, 4 * e) &&
             (dXbase == nullptr || rows_vec(dXbase, lddxbase, e, 4 * e));
    p.wide = K % 8 == 0 && rows_vec(dX, lddx, e, 16) && (dXbase == nullptr || rows_vec(dXbase, lddxbase, e, 16));
    p.v_in = V, p.scales = scales, p.scale_stride = scale_stride;
    p.frag_u = reinterpret_cast<uint4 *>(base + w.frag_u), p.frag_v = reinterpret_cast<uint4 *>(base + w.frag_v);
    if (T > 0) {
        st = tdy == DYBIT_F32 ? launch_tokens_rank<float, __nv_bfloat16, float, true>(p, s)
                              : launch_tokens_rank<__nv_bfloat16, __nv_bfloat16, __nv_bfloat16, true>(p, s);
        if (st != DYBIT_OK) return st;
    }
    AdapterGrad gp = {};
    gp.plan = p.plan, gp.T = T, gp.n = n_adapters, gp.R = R;
    gp.side[0] = {codes, row_stride_bytes, K, p.frag_u, dA, reinterpret_cast<float *>(base + w.partial_a), 1};
    gp.side[1] = {dY, lddy, N, p.frag_v, dB, reinterpret_cast<float *>(base + w.partial_b), rows_vec(dY, lddy, e, 16) ? 1 : 0};
    if (fmt.is_signed)
        return tdy == DYBIT_F32 ? launch_grad<GradSrc::CodesSigned, GradSrc::F32>(gp, s) : launch_grad<GradSrc::CodesSigned, GradSrc::Bf16>(gp, s);
    return tdy == DYBIT_F32 ? launch_grad<GradSrc::CodesUnsigned, GradSrc::F32>(gp, s) : launch_grad<GradSrc::CodesUnsigned, GradSrc::Bf16>(gp, s);
}

}  // extern "C"
