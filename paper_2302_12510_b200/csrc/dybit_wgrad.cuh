// Weight gradient of a linear layer from the 8-bit checkpoint of its input:
//     dW[n][k] = sum_t dY[t][n] * x^[t][k],   x^[t][k] = scale_t * value(code[t][k]).
//
// A matrix product whose two operands both have the contraction (tokens) as their slow dimension.  Two steps:
//   1. wgrad_expand_kernel writes x^ as bf16 (exact: a value has at most eight significant bits and a row's scale is a
//      power of two) and, where dY is not bf16 already or its rows cannot be fetched by the TMA, dY as one to three bf16
//      terms whose sum it is.  HBM-bound, 3 bytes per code.
//   2. dybit_wgrad_kernel: tcgen05 on CTA pairs, 256 x 256 outputs per pair.  The operands are fetched as they lie, 64
//      tokens x 64 columns per TMA box, and multiplied from shared memory in the layout where rows run along the
//      contraction (MN-major descriptors), so nothing is transposed anywhere.
#pragma once

#include <string.h>

#include <algorithm>

#include "dybit_checkpoint.cuh"
#include "dybit_wait.cuh"

namespace dybit {

using namespace sm100;

// ------------------------------------------------------------------ step 1: bf16 operands

struct WgradExpand {
    const uint8_t *codes;
    int64_t stride;
    const float *scales;
    int64_t scale_stride;        // 0: the scale multiplies the sum instead
    __nv_bfloat16 *xe;           // [T][ldx]
    int64_t ldx;
    const void *dy;              // null: read by the product as it is
    int64_t lddy;
    __nv_bfloat16 *dye;          // [terms][T][ldn]
    int64_t ldn;
    int64_t T, N, K;
    int64_t x_blocks;            // blocks that expand codes; the others take dY
    int x_chunks, dy_chunks;     // of a row
};

constexpr int kExpandThreads = 256;
constexpr int kExpandUnroll = 4;

// Eight consecutive elements of dY as floats, zeros beyond N.
template <typename T>
__device__ __forceinline__ void load8f(float (&f)[8], const T *row, int64_t c, int64_t cols, bool vec) {
    constexpr int E = 16 / (int)sizeof(T);
    if (vec && c + 8 <= cols) {
#pragma unroll
        for (int i = 0; i < 8 / E; ++i) {
            const VecFloats<T> o = vec_floats<T>(__ldg(reinterpret_cast<const uint4 *>(row + c) + i));
#pragma unroll
            for (int j = 0; j < E / 4; ++j) {
                const float4 v = o.f[j];
                f[i * E + 4 * j] = v.x;
                f[i * E + 4 * j + 1] = v.y;
                f[i * E + 4 * j + 2] = v.z;
                f[i * E + 4 * j + 3] = v.w;
            }
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = c + j < cols ? to_f32(row[c + j]) : 0.0f;
    }
}

// A warp takes 1024 columns of a row, 8 per lane and round.
template <typename T, bool SIGNED, bool VEC>
__global__ void __launch_bounds__(kExpandThreads) wgrad_expand_kernel(const WgradExpand p) {
    constexpr int kTerms = sizeof(T) == 4 ? 3 : (__is_same(T, __half) ? 2 : 1);
    pdl_enter();
    const int lane = threadIdx.x & 31;
    const bool is_x = (int64_t)blockIdx.x < p.x_blocks;
    const int64_t item = ((int64_t)blockIdx.x - (is_x ? 0 : p.x_blocks)) * (kExpandThreads / 32) + (threadIdx.x >> 5);
    const int chunks = is_x ? p.x_chunks : p.dy_chunks;
    const int64_t t = item / chunks;
    if (t >= p.T) return;
    const int64_t c0 = (item - t * chunks) * (kExpandUnroll * 256) + lane * 8;
    if (is_x) {
        const uint8_t *in = p.codes + t * p.stride;
        const float scale = p.scale_stride != 0 ? __ldg(p.scales + t * p.scale_stride) : 1.0f;
        uint2 w[kExpandUnroll];
#pragma unroll
        for (int i = 0; i < kExpandUnroll; ++i)                 // rows of codes are padded to 16, rows of x^ to 8
            w[i] = c0 + i * 256 < p.K ? __ldg(reinterpret_cast<const uint2 *>(in + c0 + i * 256)) : make_uint2(0u, 0u);
#pragma unroll
        for (int i = 0; i < kExpandUnroll; ++i) {
            const int64_t c = c0 + i * 256;
            if (c >= p.K || !DYBIT_CHECK(c + 8 <= p.ldx && c + 8 <= p.stride, 0x67)) break;
            const float4 a = decode4<SIGNED>(w[i].x), b = decode4<SIGNED>(w[i].y);
            *reinterpret_cast<uint4 *>(p.xe + t * p.ldx + c) =
                make_uint4(pack_bf16(__fmul_rn(a.x, scale), __fmul_rn(a.y, scale)), pack_bf16(__fmul_rn(a.z, scale), __fmul_rn(a.w, scale)),
                           pack_bf16(__fmul_rn(b.x, scale), __fmul_rn(b.y, scale)), pack_bf16(__fmul_rn(b.z, scale), __fmul_rn(b.w, scale)));
        }
    } else {
        const T *in = static_cast<const T *>(p.dy) + t * p.lddy;
#pragma unroll
        for (int i = 0; i < kExpandUnroll; ++i) {
            const int64_t c = c0 + i * 256;
            if (c >= p.N || !DYBIT_CHECK(c + 8 <= p.ldn, 0x68)) break;
            float f[8];
            load8f<T>(f, in, c, p.N, VEC);
#pragma unroll
            for (int k = 0; k < kTerms; ++k) {
                // cut off all but eight significant bits; the last term takes what is left (an f16 has three more bits, an
                // f32 sixteen); nothing is left of an infinity
                float h[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    h[j] = k + 1 < kTerms ? __uint_as_float(__float_as_uint(f[j]) & 0xffff0000u) : f[j];
                    f[j] = fabsf(f[j]) == __uint_as_float(0x7f800000u) ? 0.0f : __fsub_rn(f[j], h[j]);
                }
                *reinterpret_cast<uint4 *>(p.dye + ((int64_t)k * p.T + t) * p.ldn + c) =
                    make_uint4(pack_bf16(h[0], h[1]), pack_bf16(h[2], h[3]), pack_bf16(h[4], h[5]), pack_bf16(h[6], h[7]));
            }
        }
    }
}

// ------------------------------------------------------------------ step 2: the product

constexpr int kWgTile = 256;                 // outputs of a CTA pair in each direction
constexpr int kWgTokens = 64;                // contraction per stage
constexpr int kWgBox = 64 * kWgTokens * 2;   // 64 columns x 64 tokens of bf16
constexpr int kWgStageBytes = 4 * kWgBox;    // per CTA: 128 columns of dY and 128 of x^
constexpr int kWgStages = 6;
constexpr int kWgStoreStage = 128 * 128;     // 128 rows x 32 fp32 columns
constexpr int kWgSmem = kWgStages * kWgStageBytes + 2 * kWgStoreStage + 512 + 1024;
constexpr int kWgThreads = 320;
// The tensor core cuts off what an addition to its fp32 accumulator cannot hold, so its error grows with the length of the
// sum (3.4e-6 of the result over 8192 tokens).  After this many stages (1024 tokens) the epilogue warps take the
// accumulator and add it to sums of their own in registers, rounded to nearest, while the next one fills
// (8192 tokens: 2.4e-7; a product in plain fp32 has 3.3e-7).
constexpr int kWgSegment = 16;

struct WgradParams {
    int N, K;                    // extent of dW
    int n_tiles, k_tiles;
    int splits;                  // the contraction is cut into this many parts
    int blocks;                  // stages of a whole contraction: terms * blocks_per_term
    int blocks_per_term;
    int split_from;              // work items from here on are halves (256 x 128) of a tile
    const float *scale;          // multiplies the sum, or null
    float *out;                  // dW, or the parts [splits][N][ld]
    int64_t ld, part;
    int tma_store;
};

// Shared-memory descriptor of an operand whose rows (128 bytes, 64 columns) run along the contraction, 128-byte
// swizzle: eight rows (1024 bytes) to the next group along the contraction, one box to the next 64 columns.
__device__ __forceinline__ uint64_t umma_desc_mnmajor(uint32_t smem_addr) {
    uint64_t d = 0;
    d |= (uint64_t)((smem_addr & 0x3ffffu) >> 4);
    d |= (uint64_t)(kWgBox >> 4) << 16;                // leading byte offset: between groups of 64 columns
    d |= (uint64_t)(1024 >> 4) << 32;                  // stride byte offset: between groups of eight contraction rows
    d |= (uint64_t)1 << 46;
    d |= (uint64_t)2 << 61;
    return d;
}

// 3-D box load whose completion is counted on the pair leader's barrier (no multicast).
__device__ __forceinline__ void tma_load_3d_pair(void *smem_dst, const CUtensorMap *map, int x, int y, int z, uint32_t bar_cluster_addr) {
    asm volatile(
        "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
        ::"r"(smem_u32(smem_dst)), "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(bar_cluster_addr)
        : "memory");
}

struct WgradItem { int n_blk, k_blk, k_off, width, split, first, last; };

__device__ __forceinline__ WgradItem wgrad_item(int item, const WgradParams &p) {
    WgradItem o;
    int tile = item, half = 0;
    o.width = kWgTile;
    if (item >= p.split_from) {
        tile = p.split_from + ((item - p.split_from) >> 1);
        half = (item - p.split_from) & 1;
        o.width = kWgTile / 2;
    }
    o.k_off = half * (kWgTile / 2);
    const int tiles = p.n_tiles * p.k_tiles;
    o.split = tile / tiles;
    tile -= o.split * tiles;
    // groups of eight tile rows sweep all tile columns, so one wave of pairs shares few operand tiles
    const int per_group = 8 * p.k_tiles, group = tile / per_group, first_n = group * 8;
    const int rows = min(8, p.n_tiles - first_n), in_group = tile - group * per_group;
    o.n_blk = first_n + in_group % rows;
    o.k_blk = in_group / rows;
    o.first = (int)((int64_t)p.blocks * o.split / p.splits);
    o.last = (int)((int64_t)p.blocks * (o.split + 1) / p.splits);
    return o;
}

__global__ void __launch_bounds__(kWgThreads, 1)
dybit_wgrad_kernel(const __grid_constant__ CUtensorMap tmap_dy, const __grid_constant__ CUtensorMap tmap_x,
                   const __grid_constant__ CUtensorMap tmap_out, const WgradParams p) {
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint8_t *out_stages = smem + kWgStages * kWgStageBytes;
    uint64_t *bars = reinterpret_cast<uint64_t *>(out_stages + 2 * kWgStoreStage);
    uint64_t *full = bars;                       // used in the leader CTA: both CTAs' loads complete on it
    uint64_t *empty = bars + kWgStages;          // one per CTA, released by the leader's commit
    uint64_t *acc_full = bars + 2 * kWgStages;   // one per CTA
    uint64_t *acc_empty = acc_full + 2;          // used in the leader CTA: the epilogue warps of both arrive
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(acc_empty + 2);
    volatile uint32_t *abort_flag = tmem_slot + 1;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_ctarank();     // 0 = leader
    const int pair = blockIdx.x >> 1, num_pairs = gridDim.x >> 1;
    const int whole = p.n_tiles * p.k_tiles * p.splits;
    const int items = whole + (whole - p.split_from);
    constexpr uint32_t kTmemCols = 2 * kWgTile;  // two accumulators

    if (threadIdx.x == 0) {
        for (int s = 0; s < kWgStages; ++s) {
            mbar_init(&full[s], 1);
            mbar_init(&empty[s], 1);
        }
        for (int a = 0; a < 2; ++a) {
            mbar_init(&acc_full[a], 1);
            mbar_init(&acc_empty[a], 16);
        }
        *abort_flag = 0;
        fence_mbar_init();
        prefetch_tensormap(&tmap_dy);
        prefetch_tensormap(&tmap_x);
        if (p.tma_store) prefetch_tensormap(&tmap_out);
    }
    if (warp == 1) {
        tmem_alloc_pair(tmem_slot, kTmemCols);
        tmem_relinquish_pair();
    }
    tc_fence_before_sync();
    __syncthreads();
    cluster_sync_all();                          // the peer's barriers exist before anything signals them
    tc_fence_after_sync();
    const uint32_t tmem_base = *tmem_slot;
    pdl_enter();

    if (warp == 0) {
        // ------------------------------------------------ TMA producer (both CTAs)
        if (lane == 0) {
            uint32_t it = 0;
            bool ok = true;
            for (int item = pair; item < items && ok; item += num_pairs) {
                const WgradItem w = wgrad_item(item, p);
                const int n0 = w.n_blk * kWgTile + (int)rank * 128;
                // (a half item still loads 128 columns of x^ per CTA; the instruction reads the first 64 of each)
                const int k0 = w.k_blk * kWgTile + w.k_off + (int)rank * (w.width / 2);
                for (int b = w.first; b < w.last; ++b, ++it) {
                    const int s = it % kWgStages, term = b / p.blocks_per_term, t0 = (b - term * p.blocks_per_term) * kWgTokens;
                    if (!wait_bounded(&empty[s], ((it / kWgStages) & 1u) ^ 1u, abort_flag, 0x61)) { ok = false; break; }
                    if (rank == 0) mbar_arrive_expect_tx(&full[s], 2u * kWgStageBytes);
                    const uint32_t bar = mapa_u32(smem_u32(&full[s]), 0u);
                    uint8_t *stage = smem + s * kWgStageBytes;
                    tma_load_3d_pair(stage, &tmap_dy, n0, t0, term, bar);
                    tma_load_3d_pair(stage + kWgBox, &tmap_dy, n0 + 64, t0, term, bar);
                    tma_load_3d_pair(stage + 2 * kWgBox, &tmap_x, k0, t0, 0, bar);
                    tma_load_3d_pair(stage + 3 * kWgBox, &tmap_x, k0 + 64, t0, 0, bar);
                }
            }
            if (!ok) {
                for (int i = 0; i < 64; ++i) __nanosleep(2000);
            }
        }
    } else if (warp == 1) {
        // ------------------------------------------------ MMA issuer (leader CTA only)
        if (lane == 0 && rank == 0) {
            constexpr uint32_t kMnMajor = (1u << 15) | (1u << 16);             // both operands
            constexpr uint32_t idesc_whole = umma_idesc(1u, 1u, 256, 256) | kMnMajor;
            constexpr uint32_t idesc_half = umma_idesc(1u, 1u, 256, 128) | kMnMajor;
            uint32_t it = 0, lt = 0;
            bool ok = true;
            for (int item = pair; item < items && ok; item += num_pairs) {
                const WgradItem w = wgrad_item(item, p);
                const uint32_t idesc = w.width == kWgTile ? idesc_whole : idesc_half;
                for (int b0 = w.first; b0 < w.last && ok; b0 += kWgSegment, ++lt) {
                    const uint32_t as = lt & 1u, aph = (lt >> 1) & 1u;
                    if (!wait_bounded(&acc_empty[as], aph ^ 1u, abort_flag, 0x62)) { ok = false; break; }
                    tc_fence_after_sync();
                    const uint32_t d = tmem_base + as * kWgTile;
                    const int b1 = min(w.last, b0 + kWgSegment);
                    for (int b = b0; b < b1; ++b, ++it) {
                        const int s = it % kWgStages;
                        if (!wait_bounded(&full[s], (it / kWgStages) & 1u, abort_flag, 0x63)) { ok = false; break; }
                        tc_fence_after_sync();
                        const uint64_t adesc = umma_desc_mnmajor(smem_u32(smem + s * kWgStageBytes));
                        const uint64_t bdesc = umma_desc_mnmajor(smem_u32(smem + s * kWgStageBytes + 2 * kWgBox));
#pragma unroll
                        for (int k = 0; k < kWgTokens / 16; ++k)               // 16 contraction rows are 2048 bytes
                            umma_pair<Kind::F16>(d, adesc + (uint64_t)(k * 128), bdesc + (uint64_t)(k * 128), idesc, (uint32_t)(b != b0 || k != 0));
                        umma_commit_pair(&empty[s], (uint16_t)3);
                    }
                    if (ok) umma_commit_pair(&acc_full[as], (uint16_t)3);
                }
            }
        }
    } else {
        // ------------------------------------------------ epilogue (both CTAs): TMEM -> registers -> shared -> TMA store
        const int q = warp & 3, row_in_tile = q * 32 + lane, group = (warp - 2) >> 2;
        const bool issuer = (threadIdx.x & 127) == 64;
        const float alpha = p.scale != nullptr ? __ldg(p.scale) : 1.0f;
        uint32_t lt = 0;
        bool ok = true;
        for (int item = pair; item < items && ok; item += num_pairs) {
            const WgradItem w = wgrad_item(item, p);
            const int row0 = w.n_blk * kWgTile + (int)rank * 128, tile_col = w.k_blk * kWgTile + w.k_off;
            float f[4][32];                                    // chunks group, group + 2, ... of 32 columns
#pragma unroll
            for (int c = 0; c < 4; ++c)
#pragma unroll
                for (int j = 0; j < 32; ++j) f[c][j] = 0.0f;
            for (int b0 = w.first; b0 < w.last; b0 += kWgSegment, ++lt) {
                const uint32_t as = lt & 1u, aph = (lt >> 1) & 1u;
                ok = named_barrier_and(1 + group, 128, wait_bounded(&acc_full[as], aph, abort_flag, 0x64));
                if (!ok) break;
                tc_fence_after_sync();
                const uint32_t taddr = tmem_base + as * kWgTile + ((uint32_t)(q * 32) << 16);
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const int cc = group + 2 * c;
                    if (cc * 32 >= w.width) continue;
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        uint32_t r[16];
                        tmem_ld_32x16(taddr + cc * 32 + h * 16, r);
                        tmem_ld_wait();
#pragma unroll
                        for (int j = 0; j < 16; ++j) f[c][h * 16 + j] = __fadd_rn(f[c][h * 16 + j], __uint_as_float(r[j]));
                    }
                }
                tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive_cluster(mapa_u32(smem_u32(&acc_empty[as]), 0u));
            }
            if (!ok) break;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const int col0 = tile_col + (group + 2 * c) * 32;
                if ((group + 2 * c) * 32 >= w.width || col0 >= p.K || row0 >= p.N) continue;
                if (p.scale != nullptr) {
#pragma unroll
                    for (int j = 0; j < 32; ++j) f[c][j] = __fmul_rn(f[c][j], alpha);
                }
                if (p.tma_store) {
                    uint8_t *stage = out_stages + group * kWgStoreStage;
                    if (issuer) bulk_wait_group_read<0>();
                    named_barrier(1 + group, 128);
                    uint8_t *srow = stage + row_in_tile * 128;
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        *reinterpret_cast<float4 *>(srow + ((j ^ (row_in_tile & 7)) << 4)) =
                            make_float4(f[c][4 * j], f[c][4 * j + 1], f[c][4 * j + 2], f[c][4 * j + 3]);
                    fence_proxy_async_smem();
                    named_barrier(1 + group, 128);
                    if (issuer) {
                        tma_store_3d(&tmap_out, stage, col0, row0, w.split);
                        bulk_commit_group();
                    }
                } else if (row0 + row_in_tile < p.N) {
                    // rows that the TMA cannot address
                    float *row = p.out + w.split * p.part + (int64_t)(row0 + row_in_tile) * p.ld;
#pragma unroll
                    for (int j = 0; j < 32; ++j)
                        if (col0 + j < p.K && DYBIT_CHECK(w.split < p.splits && col0 + j < p.ld, 0x69)) row[col0 + j] = f[c][j];
                }
            }
        }
        if (issuer) bulk_wait_group_read<0>();
    }

    tc_fence_before_sync();
    __syncthreads();
    cluster_sync_all();          // neither CTA leaves (or frees TMEM) while the other may still touch its memory
    if (warp == 1) {
        tc_fence_after_sync();
        tmem_dealloc_pair(tmem_base, kTmemCols);
    }
}

// The parts of a cut contraction, added in order.
__global__ void __launch_bounds__(256) wgrad_sum_kernel(const float *__restrict__ parts, int splits, int64_t part, int64_t ld, int64_t N,
                                                        int64_t K, float *__restrict__ dw, int64_t lddw, int vec) {
    pdl_enter();
    const int64_t cols4 = (K + 3) / 4;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < N * cols4; i += (int64_t)gridDim.x * 256) {
        const int64_t n = i / cols4, c = (i - n * cols4) * 4;
        if (!DYBIT_CHECK(c + 4 <= ld && (n + 1) * ld <= part, 0x6a)) continue;
        float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int k = 0; k < splits; ++k) {
            const float4 v = __ldcg(reinterpret_cast<const float4 *>(parts + k * part + n * ld + c));
            s.x += v.x;
            s.y += v.y;
            s.z += v.z;
            s.w += v.w;
        }
        float *dst = dw + n * lddw + c;
        if (vec && c + 4 <= K) {
            *reinterpret_cast<float4 *>(dst) = s;
        } else {
            const float e[4] = {s.x, s.y, s.z, s.w};
            for (int j = 0; j < 4; ++j)
                if (c + j < K) dst[j] = e[j];
        }
    }
}

__global__ void __launch_bounds__(256) wgrad_zero_kernel(float *__restrict__ dw, int64_t N, int64_t K, int64_t ld) {
    pdl_enter();
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < N * K; i += (int64_t)gridDim.x * 256) {
        const int64_t n = i / K;
        dw[n * ld + i - n * K] = 0.0f;
    }
}

// ------------------------------------------------------------------ host side

inline int wgrad_terms(dybit_dtype t) { return t == DYBIT_F32 ? 3 : (t == DYBIT_F16 ? 2 : 1); }

struct WgradPlan {
    int terms, n_tiles, k_tiles, splits;
    int64_t blocks, blocks_per_term, ldx, ldn, ldp;
    int64_t xe, dye, parts, bytes;
    WgradPlan(int64_t T, int64_t N, int64_t K, dybit_dtype t) {
        terms = wgrad_terms(t);
        n_tiles = (int)((N + kWgTile - 1) / kWgTile);
        k_tiles = (int)((K + kWgTile - 1) / kWgTile);
        blocks_per_term = (T + kWgTokens - 1) / kWgTokens;
        blocks = blocks_per_term * terms;
        // a product of few tiles is cut along the contraction until the pairs of SMs have work, with at least eight stages
        // to each part.  The pairs are counted as the B200 has them, not asked of the device: the workspace's size depends on
        // the parts, and is the same wherever it is asked for.  Fewer resident pairs work the same parts off in more rounds.
        const int64_t tiles = (int64_t)n_tiles * k_tiles, pairs = 74;
        splits = 1;
        while (tiles * splits * 2 <= pairs && blocks / (splits * 2) >= 8 && splits < 16) splits *= 2;
        ldx = round_up(K, 8);
        ldn = round_up(N, 8);
        ldp = round_up(K, 4);
        int64_t at = 0;
        xe = at, at += round_up(T * ldx * 2, 1024);
        dye = at, at += round_up(terms * T * ldn * 2, 1024);
        parts = at, at += splits > 1 ? round_up(splits * N * ldp * 4, 1024) : 0;
        bytes = at + 1024;
    }
};

// bf16 tensor [depth][rows][cols] whose boxes are 64 columns x 64 rows, 128-byte swizzle.
static bool make_wgrad_map(CUtensorMap *map, const void *base, int64_t cols, int64_t rows, int64_t ld, int64_t depth) {
    EncodeTiledFn fn = encode_tiled_fn();
    if (fn == nullptr) return false;
    cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)depth};
    cuuint64_t strides[2] = {(cuuint64_t)ld * 2, (cuuint64_t)(rows * ld) * 2};
    cuuint32_t box[3] = {64, (cuuint32_t)kWgTokens, 1}, estr[3] = {1, 1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void *>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// fp32 output [depth][N][ld], boxes of 32 columns x 128 rows.
static bool make_wgrad_out_map(CUtensorMap *map, float *out, int64_t N, int64_t K, int64_t ld, int64_t depth) {
    EncodeTiledFn fn = encode_tiled_fn();
    if (fn == nullptr || !aligned(out, 16) || ld % 4 != 0) return false;
    cuuint64_t dims[3] = {(cuuint64_t)K, (cuuint64_t)N, (cuuint64_t)depth};
    cuuint64_t strides[2] = {(cuuint64_t)ld * 4, (cuuint64_t)(N * ld) * 4};
    cuuint32_t box[3] = {32, 128, 1}, estr[3] = {1, 1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 3, out, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

struct ExpandLauncher {
    const WgradExpand &p;
    int64_t blocks;
    cudaStream_t s;
    template <typename T, bool SIGNED, bool VEC> dybit_status operator()() const {
        launch_k(wgrad_expand_kernel<T, SIGNED, VEC>, dim3((unsigned)blocks), dim3(kExpandThreads), 0, s, p);
        return launch_status();
    }
};

static dybit_status launch_wgrad_product(const CUtensorMap &tdy, const CUtensorMap &tx, const CUtensorMap &tout, WgradParams p, cudaStream_t s) {
    static std::atomic<int> max_pairs[64];
    int dev = 0;
    DYBIT_CUDA_TRY(cudaGetDevice(&dev));
    if (dev < 0 || dev >= 64) return DYBIT_ERR_CUDA;
    cudaLaunchConfig_t cfg = {};
    cfg.blockDim = dim3(kWgThreads);
    cfg.dynamicSmemBytes = kWgSmem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 2;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    if (max_pairs[dev].load(std::memory_order_acquire) == 0) {
        DYBIT_CUDA_TRY(cudaFuncSetAttribute(dybit_wgrad_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kWgSmem));
        cfg.gridDim = dim3((unsigned)sm_count() / 2 * 2);
        cfg.numAttrs = 1;                        // the occupancy query wants the cluster shape only
        int n = 0;
        DYBIT_CUDA_TRY(cudaOccupancyMaxActiveClusters(&n, dybit_wgrad_kernel, &cfg));
        if (n < 1) return DYBIT_ERR_UNSUPPORTED;
        max_pairs[dev].store(n, std::memory_order_release);
    }
    const int tiles = p.n_tiles * p.k_tiles * p.splits, resident = max_pairs[dev];
    const int pairs = tiles < resident ? tiles : resident;
    // a last wave that fills at most half of the pairs is worked on as halves
    const int rest = tiles % pairs;
    p.split_from = (rest > 0 && 2 * rest <= pairs) ? tiles - rest : tiles;
    cfg.gridDim = dim3((unsigned)(2 * pairs));
    cfg.numAttrs = 2;
    (void)cudaLaunchKernelEx(&cfg, dybit_wgrad_kernel, tdy, tx, tout, p);
    return launch_status();
}

}  // namespace dybit

extern "C" {

size_t dybit_checkpoint_wgrad_workspace_bytes(int64_t T, int64_t N, int64_t K, dybit_dtype tdy) {
    using namespace dybit;
    if (T < 0 || N < 1 || K < 1 || T > 0x1fffffff || N > 0x1fffffff || K > 0x1fffffff || !dtype_ok(tdy)) return 0;
    return (size_t)WgradPlan(T, N, K, tdy).bytes;
}

dybit_status dybit_checkpoint_wgrad(int64_t T, int64_t N, int64_t K, const void *dY, dybit_dtype tdy, int64_t lddy,
                                    const void *codes, int64_t row_stride_bytes, dybit_fmt fmt, const float *scales,
                                    int64_t scale_stride, float *dW, int64_t lddw, void *ws, size_t ws_bytes,
                                    void *stream) {
    using namespace dybit;
    dybit_status st = check_codes(codes, T, K, row_stride_bytes, fmt);
    if (st != DYBIT_OK) return st;
    const size_t need = dybit_checkpoint_wgrad_workspace_bytes(T, N, K, tdy);
    if (need == 0 || lddy < N || lddw < K || scale_stride < 0 || dW == nullptr) return DYBIT_ERR_INVALID_ARG;
    if (T > 0 && (dY == nullptr || scales == nullptr)) return DYBIT_ERR_INVALID_ARG;
    if (!aligned(dY, dtype_bytes(tdy)) || !aligned(scales, 4) || !aligned(dW, 4) || !aligned(ws, 1024)) return DYBIT_ERR_ALIGNMENT;
    if (ws == nullptr || ws_bytes < need) return DYBIT_ERR_WORKSPACE;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (T == 0) {
        const int64_t blocks = std::min<int64_t>((N * K + 255) / 256, 4 * (int64_t)sm_count());
        launch_k(wgrad_zero_kernel, dim3((unsigned)blocks), dim3(256), 0, s, dW, N, K, lddw);
        return launch_status();
    }
    const WgradPlan w(T, N, K, tdy);
    if ((int64_t)w.n_tiles * w.k_tiles * w.splits > 0x3fffffff || w.blocks > 0x3fffffff) return DYBIT_ERR_UNSUPPORTED;
    uint8_t *base = static_cast<uint8_t *>(ws);
    const bool direct = tdy == DYBIT_BF16 && rows_vec16(dY, lddy, 2);          // the TMA fetches dY itself
    WgradExpand e = {};
    e.codes = static_cast<const uint8_t *>(codes), e.stride = row_stride_bytes, e.scales = scales, e.scale_stride = scale_stride;
    e.xe = reinterpret_cast<__nv_bfloat16 *>(base + w.xe), e.ldx = w.ldx;
    e.dy = direct ? nullptr : dY, e.lddy = lddy, e.dye = reinterpret_cast<__nv_bfloat16 *>(base + w.dye), e.ldn = w.ldn;
    e.T = T, e.N = N, e.K = K;
    constexpr int kCols = kExpandUnroll * 256, kRows = kExpandThreads / 32;
    e.x_chunks = (int)((K + kCols - 1) / kCols), e.dy_chunks = (int)((N + kCols - 1) / kCols);
    e.x_blocks = (T * e.x_chunks + kRows - 1) / kRows;
    const int64_t blocks = e.x_blocks + (direct ? 0 : (T * e.dy_chunks + kRows - 1) / kRows);
    if (blocks > kMaxGridX) return DYBIT_ERR_UNSUPPORTED;

    CUtensorMap tdy_map, tx_map, tout_map;
    memset(&tout_map, 0, sizeof(tout_map));
    const bool maps = make_wgrad_map(&tdy_map, direct ? dY : e.dye, N, T, direct ? lddy : w.ldn, w.terms) &&
                      make_wgrad_map(&tx_map, e.xe, K, T, w.ldx, 1);
    if (!maps) return DYBIT_ERR_CUDA;
    WgradParams p = {};
    p.N = (int)N, p.K = (int)K, p.n_tiles = w.n_tiles, p.k_tiles = w.k_tiles, p.splits = w.splits;
    p.blocks = (int)w.blocks, p.blocks_per_term = (int)w.blocks_per_term;
    p.scale = scale_stride == 0 ? scales : nullptr;
    p.out = w.splits > 1 ? reinterpret_cast<float *>(base + w.parts) : dW;
    p.ld = w.splits > 1 ? w.ldp : lddw;
    p.part = N * p.ld;
    p.tma_store = make_wgrad_out_map(&tout_map, p.out, N, K, p.ld, w.splits) ? 1 : 0;

    st = with_elem(tdy, fmt.is_signed != 0, rows_vec16(dY, lddy, dtype_bytes(tdy)), ExpandLauncher{e, blocks, s});
    if (st != DYBIT_OK) return st;
    st = launch_wgrad_product(tdy_map, tx_map, tout_map, p, s);
    if (st != DYBIT_OK || w.splits == 1) return st;
    const int64_t sum_blocks = std::min<int64_t>((N * ((K + 3) / 4) + 255) / 256, 8 * (int64_t)sm_count());
    launch_k(wgrad_sum_kernel, dim3((unsigned)sum_blocks), dim3(256), 0, s, (const float *)p.out, w.splits, p.part, p.ld, N, K, dW, lddw,
             (aligned(dW, 16) && lddw % 4 == 0) ? 1 : 0);
    return launch_status();
}

}  // extern "C"
