// Attention over the 8-bit cache for tiles of 256 query rows: both products on the tensor cores (tcgen05).
//
// A block of the tile takes its keys 128 at a time.  Roles, a warp each or several:
//   decode    codes -> f16 or bf16 keys and f16 values in shared memory, in the operands' swizzled layouts (nothing but
//             codes crosses the memory system, and the 256 rows share what is decoded); four warps for keys, four for values
//   issue     S_t = Q_t K^T into TMEM and O_t += P_t V with P_t read from TMEM, for the two halves t of the rows in turn
//   softmax   four warps to a half, a thread to a row: S_t -> P_t in place (f16), the running maximum and sum, and now and then a
//             factor on O_t
// While one half's scores are on their way through the softmax the tensor core works for the other half.  Per 128 keys
// and SM the products take 2048 clocks of the tensor core, the exponentials 2048 of the special-function units, decoding
// and softmax together about 1800 issue slots of each scheduler, and the operands about 2048 clocks of shared memory.
#pragma once

#include "dybit_cache_attention.cuh"

namespace dybit {

constexpr int kLgKeys = 128;                 // keys of a block
constexpr int kLgWarps = 17, kLgThreads = 32 * kLgWarps;     // 2 x 4 softmax, 4 + 4 decode, 1 issue
constexpr int kLgStages = 2;

template <int DP> __host__ __device__ constexpr int large_panel_bytes() { return 128 * 128; }       // 128 rows of 64 16-bit elements
template <int DP> __host__ __device__ constexpr int large_tile_bytes() { return (DP / 64) * 128 * 128; }
template <int DP> __host__ __device__ constexpr int large_smem_bytes() { return (2 + 2 * kLgStages) * large_tile_bytes<DP>() + 1024; }

// Operand whose rows (128 bytes, 64 columns) run along the contraction: groups of eight rows 1024 bytes apart, the next 64 columns a
// panel further on.
__device__ __forceinline__ uint64_t large_desc_values(uint32_t smem_addr) {
    uint64_t d = 0;
    d |= (uint64_t)((smem_addr & 0x3ffffu) >> 4);
    d |= (uint64_t)((128 * 128) >> 4) << 16;
    d |= (uint64_t)(1024 >> 4) << 32;
    d |= (uint64_t)1 << 46;
    d |= (uint64_t)2 << 61;
    return d;
}

// D (128 x N, TMEM) += A (128 x 16 f16, TMEM, two elements to a column) * B
__device__ __forceinline__ void umma_ts_f16(uint32_t tmem_d, uint32_t tmem_a, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\n"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}\n" ::"r"(tmem_d),
        "r"(tmem_a), "l"(bdesc), "r"(idesc), "r"(accumulate)
        : "memory");
}

__device__ __forceinline__ void tmem_st_32x16(uint32_t taddr, const uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};" ::"r"(r[0]),
        "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]),
        "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(taddr)
        : "memory");
}
__device__ __forceinline__ void tmem_st_32x8(uint32_t taddr, const uint32_t (&r)[8]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%8], {%0, %1, %2, %3, %4, %5, %6, %7};" ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]),
                 "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(taddr)
                 : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Two fp32 operations to an instruction.
__device__ __forceinline__ uint64_t pack_f32x2(float a, float b) {
    uint64_t v;
    asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(a), "f"(b));
    return v;
}
__device__ __forceinline__ float2 unpack_f32x2(uint64_t v) {
    float2 f;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(f.x), "=f"(f.y) : "l"(v));
    return f;
}
__device__ __forceinline__ uint64_t fma_f32x2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ uint64_t add_f32x2(uint64_t a, uint64_t b) {
    uint64_t d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}

// What the decoding warps need to know of their tile.
struct LargeDecode {
    const int *table;
    int len, head, first, last;
    volatile uint32_t *abort_flag;
};

// Page of the 16 keys from `key` on, or -1.
__device__ __forceinline__ int large_page(const CacheAttn &p, const int *table, int len, int key) {
    const int pg = key < len ? __ldg(table + (key >> p.page_shift)) : -1;
    return (unsigned)pg < (uint64_t)p.pages ? pg : -1;
}

// Four warps turn the codes of a block's keys (or values) into 16-bit numbers of type T in the operand's layout, a unit
// of 16 codes to a thread and pass.  The codes of the next half block are on their way while one is decoded.
template <typename T, int DP, bool VALUES>
__device__ __forceinline__ void large_decode(const CacheAttn &p, const LargeDecode &t, const uint8_t *__restrict__ codes, uint8_t *tiles, uint64_t *full,
                                             uint64_t *empty) {
    constexpr int UNITS = DP / 16, ROWS = 128 / UNITS, PASSES = kLgKeys / ROWS, HALF = PASSES / 2, PANEL = large_panel_bytes<DP>();
    const int lane = threadIdx.x & 31, i = threadIdx.x & 127, u = i % UNITS, row0 = i / UNITS;
    const bool in_dim = u * 16 < p.dim;
    const int page_mask = (1 << p.page_shift) - 1;
    const int64_t page_bytes = (int64_t)p.heads * p.dim << p.page_shift;
    const uint8_t *base = codes + ((int64_t)t.head * p.dim << p.page_shift) + u * 16;
    auto load = [&](int key, int pg) {
        uint4 v = make_uint4(0u, 0u, 0u, 0u);
        if (pg >= 0 && in_dim) v = __ldg(reinterpret_cast<const uint4 *>(base + pg * page_bytes + (key & page_mask) * p.dim));
        return v;
    };
    auto page_at = [&](int b) { return b < t.last ? large_page(p, t.table, t.len, b * kLgKeys + 16 * (lane & 7)) : -1; };
    // values whose scale is 0 are zeros whatever their codes
    auto held = [&](int pg) { return !VALUES || (pg >= 0 && __ldg(p.v_scales + (int64_t)pg * p.heads + t.head) > 0.0f); };
    // lane k < 8 has the page of 16 keys k of a block
    int page_now = page_at(t.first), page_next = page_at(t.first + 1);
    bool held_now = held(page_now);
    uint4 c[HALF];
#pragma unroll
    for (int s = 0; s < HALF; ++s) {
        const int key = row0 + s * ROWS;
        c[s] = load(key, __shfl_sync(0xffffffffu, page_now, key >> 4));
    }
    // threads of the second panel store their second half first: eight lanes then fill eight different 16-byte columns
    const bool swap = DP == 128 && (u & 4) != 0;
    const int chunk = 2 * (u & 3) + (swap ? 1 : 0);
    uint8_t *const dst0 = tiles + (u >> 2) * PANEL + row0 * 128;
    for (int b = t.first, n = 0; b < t.last; ++b, ++n) {
        const int stage = n % kLgStages;
        const int page_after = page_at(b + 2);
        const bool held_next = held(page_next);
        if (!__all_sync(0xffffffffu, wait_bounded(&empty[stage], ((n / kLgStages) & 1u) ^ 1u, t.abort_flag, 0x82))) break;
        const uint32_t holds = __ballot_sync(0xffffffffu, held_now);
#pragma unroll 1
        for (int h = 0; h < 2; ++h) {
            uint8_t *dst = dst0 + stage * large_tile_bytes<DP>() + h * (HALF * ROWS * 128);
            const int ahead = h == 0 ? page_now : page_next;
#pragma unroll
            for (int s = 0; s < HALF; ++s) {
                const int key = row0 + (h * HALF + s) * ROWS, next = row0 + ((h ^ 1) * HALF + s) * ROWS;
                uint4 w = c[s];
                if (VALUES && !((holds >> (key >> 4)) & 1u)) w = make_uint4(0u, 0u, 0u, 0u);
                c[s] = load(next, __shfl_sync(0xffffffffu, ahead, next >> 4));
                const unsigned a0 = swap ? w.z : w.x, a1 = swap ? w.w : w.y, a2 = swap ? w.x : w.z, a3 = swap ? w.y : w.w;
                auto pair = [&](unsigned x, int sel) { return decode_pair<T>(__byte_perm(x, 0u, sel)); };
                const uint4 lo = make_uint4(pair(a0, 0x1100), pair(a0, 0x3322), pair(a1, 0x1100), pair(a1, 0x3322));
                const uint4 hi = make_uint4(pair(a2, 0x1100), pair(a2, 0x3322), pair(a3, 0x1100), pair(a3, 0x3322));
                uint8_t *row = dst + s * (ROWS * 128);
                *reinterpret_cast<uint4 *>(row + ((chunk ^ (key & 7)) << 4)) = lo;
                *reinterpret_cast<uint4 *>(row + (((chunk ^ 1) ^ (key & 7)) << 4)) = hi;
            }
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(&full[stage]);
        page_now = page_next, page_next = page_after, held_now = held_next;
    }
}

// The largest of a row's 128 scores (TMEM address ts), times 16 keys' factor plus their exponent.
template <bool EDGE>
__device__ __forceinline__ float large_row_max(uint32_t ts, const float4 *blk, int lo, int hi) {
    float top = -INFINITY;
#pragma unroll 2
    for (int c = 0; c < 8; ++c) {
        uint32_t v[16];
        tmem_ld_32x16(ts + c * 16, v);
        const float4 f = blk[c];
        tmem_ld_wait();
        if (EDGE) {
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                const float x = __fmaf_rn(__uint_as_float(v[j]), f.x, f.y);
                top = c * 16 + j >= lo && c * 16 + j < hi ? fmaxf(top, x) : top;
            }
        } else {                                           // the factor is not negative: the largest product has the largest x
            float a = __uint_as_float(v[0]);
#pragma unroll
            for (int j = 1; j < 15; j += 2) a = fmaxf(fmaxf(a, __uint_as_float(v[j])), __uint_as_float(v[j + 1]));
            a = fmaxf(a, __uint_as_float(v[15]));
            top = fmaxf(top, __fmaf_rn(a, f.x, f.y));
        }
    }
    return top;
}

// The row's probabilities at maximum um, written over its scores; returns l with their sum.
template <bool EDGE>
__device__ __forceinline__ float large_row_exp(uint32_t ts, const float4 *blk, int lo, int hi, float um, float l) {
#pragma unroll 2
    for (int c = 0; c < 8; ++c) {
        uint32_t v[16], pr[8];
        tmem_ld_32x16(ts + c * 16, v);
        const float4 f = blk[c];
        const float shift = f.y - um;
        const uint64_t cc = pack_f32x2(f.x, f.x), ss = pack_f32x2(shift, shift);
        uint64_t sum = 0;
        tmem_ld_wait();
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            float2 x = unpack_f32x2(fma_f32x2(pack_f32x2(__uint_as_float(v[2 * j]), __uint_as_float(v[2 * j + 1])), cc, ss));
            if (EDGE) {
                if (c * 16 + 2 * j < lo || c * 16 + 2 * j >= hi) x.x = -INFINITY;
                if (c * 16 + 2 * j + 1 < lo || c * 16 + 2 * j + 1 >= hi) x.y = -INFINITY;
            }
            x.x = ex2(x.x), x.y = ex2(x.y);
            sum = j == 0 ? pack_f32x2(x.x, x.y) : add_f32x2(sum, pack_f32x2(x.x, x.y));
            pr[j] = pack_f16(x.x, x.y);
        }
        const float2 s = unpack_f32x2(sum);
        l = __fmaf_rn(s.x + s.y, f.z, l);
        tmem_st_32x8(ts + c * 8, pr);
    }
    return l;
}

// A tile's own blocks: those between the first and the last key that a row of its half sees, within the part's range.
struct LargeHalf { int first, last; };

template <typename T, int DP>
__global__ void __launch_bounds__(kLgThreads, 1)
cache_large_kernel(const uint8_t *__restrict__ k_codes, const uint8_t *__restrict__ v_codes, const CacheAttn p) {
    constexpr int KS = DP / 16, PANEL = large_panel_bytes<DP>(), TILE = large_tile_bytes<DP>();
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint8_t *s_q = smem, *s_k = smem + 2 * TILE, *s_v = s_k + kLgStages * TILE;
    __shared__ uint64_t k_full[kLgStages], k_empty[kLgStages], v_full[kLgStages], v_empty[kLgStages], s_full[2], p_full[2], o_full[2];
    __shared__ uint32_t s_tmem, s_abort;
    __shared__ float4 s_info[8][2][8];                     // softmax warp, parity, 16 keys: {x's factor, values' exponent, 2^-exponent, -}

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int item = (int)(blockIdx.x / (unsigned)p.heads), head = (int)(blockIdx.x - (unsigned)item * (unsigned)p.heads);
    if (threadIdx.x == 0) {
        for (int s = 0; s < kLgStages; ++s) {
            mbar_init(&k_full[s], 4);
            mbar_init(&k_empty[s], 1);
            mbar_init(&v_full[s], 4);
            mbar_init(&v_empty[s], 1);
        }
        for (int t = 0; t < 2; ++t) {
            mbar_init(&s_full[t], 1);
            mbar_init(&p_full[t], 4);
            mbar_init(&o_full[t], 1);
        }
        s_abort = 0;
        fence_mbar_init();
    }
    if (warp == 16) {
        tmem_alloc(&s_tmem, 512);
        tmem_relinquish();
    }
    pdl_enter();
    const bool there = item < p.plan[2];
    CacheTile tile = {};
    if (there) tile = p.tiles[item];
    const int r0 = tile.tile * kLargeRows, rows = there ? min(kLargeRows, tile.n * p.group - r0) : 0;
    const KeyRange range = there ? tile_keys(p, tile, r0, kLargeRows, kLgKeys) : KeyRange{0, 0};
    auto half_of = [&](int t) {
        LargeHalf h = {0, 0};
        if (128 * t >= rows) return h;
        const RowKeys a = row_keys(p, tile, r0 + 128 * t), z = row_keys(p, tile, r0 + min(rows, 128 * t + 128) - 1);
        if (z.hi <= a.lo) return h;
        h.first = max(range.first, a.lo & ~(kLgKeys - 1)) / kLgKeys;
        h.last = max(h.first, min(range.last, (z.hi + kLgKeys - 1) & ~(kLgKeys - 1)) / kLgKeys);
        return h;
    };
    const LargeHalf half0 = half_of(0), half1 = half_of(1);
    const int b_first = half0.first == half0.last ? half1.first : half1.first == half1.last ? half0.first : min(half0.first, half1.first);
    const int b_last = half0.first == half0.last ? half1.last : half1.first == half1.last ? half0.last : max(half0.last, half1.last);
    const int *table = p.table + tile.seq * p.table_stride;
    auto page_at = [&](int key) { return large_page(p, table, tile.len, key); };

    if (warp < 8 && there) {
        // a thread loads its row of queries
        const int r = warp * 32 + lane, row = r & 127;
        const int token = (r0 + r) / p.group, h = head * p.group + (r0 + r - token * p.group);
        const T *q = r < rows ? static_cast<const T *>(p.q) + (tile.row + token) * p.q_token + h * p.q_head : nullptr;
        uint8_t *dst = s_q + (r >> 7) * TILE + row * 128;
#pragma unroll
        for (int c = 0; c < DP / 8; ++c) {
            uint4 v = make_uint4(0u, 0u, 0u, 0u);
            if (q != nullptr && c * 8 < p.dim) {
                if (p.q_vec16) {
                    v = __ldg(reinterpret_cast<const uint4 *>(q) + c);
                } else {
                    T e[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) e[i] = q[c * 8 + i];
                    memcpy(&v, e, 16);
                }
            }
            *reinterpret_cast<uint4 *>(dst + (c >> 3) * PANEL + (((c & 7) ^ (row & 7)) << 4)) = v;
        }
        fence_proxy_async_smem();
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = s_tmem;
    // columns: scores of the halves (their first 64 become the probabilities), then the outputs
    const uint32_t t_o = tmem + 256;

    if (warp >= 8 && warp < 16) {
        // ------------------------------------------------ decode: warps 8 .. 11 keys, 12 .. 15 values
        const LargeDecode d = {table, tile.len, head, b_first, b_last, &s_abort};
        if (warp < 12) large_decode<T, DP, false>(p, d, k_codes, s_k, k_full, k_empty);
        else large_decode<__half, DP, true>(p, d, v_codes, s_v, v_full, v_empty);
    } else if (warp == 16) {
        // ------------------------------------------------ issue
        if (lane == 0 && b_first < b_last) {
            constexpr uint32_t ab = __is_same(T, __half) ? 0u : 1u;
            constexpr uint32_t idesc_s = umma_idesc(1u, ab, 128, kLgKeys), idesc_o = umma_idesc(1u, 0u, 128, DP) | (1u << 16);
            uint32_t phase_p[2] = {0, 0};
            bool ok = true;
            auto active = [&](int t, int b) { return t == 0 ? b >= half0.first && b < half0.last : b >= half1.first && b < half1.last; };
            auto scores = [&](int t, int b) {
                const uint32_t qa = smem_u32(s_q + t * TILE), ka = smem_u32(s_k + ((b - b_first) % kLgStages) * TILE);
#pragma unroll
                for (int k = 0; k < KS; ++k) {
                    const uint32_t off = (uint32_t)((k >> 2) * PANEL + (k & 3) * 32);
                    umma<Kind::F16>(tmem + t * 128, umma_desc_kmajor<128>(qa + off), umma_desc_kmajor<128>(ka + off), idesc_s, (uint32_t)(k != 0));
                }
                umma_commit(&s_full[t]);
            };
            auto outputs = [&](int t, int b, bool first) {
                const uint64_t vd = large_desc_values(smem_u32(s_v + ((b - b_first) % kLgStages) * TILE));
#pragma unroll
                for (int k = 0; k < kLgKeys / 16; ++k)     // 16 keys are 2048 bytes of values and 8 columns of probabilities
                    umma_ts_f16(t_o + t * 128, tmem + t * 128 + k * 8, vd + (uint64_t)(k * 128), idesc_o, (uint32_t)(!first || k != 0));
            };
            ok = wait_bounded(&k_full[0], 0, &s_abort, 0x83);
            if (ok) {
                tc_fence_after_sync();
                for (int t = 0; t < 2; ++t)
                    if (active(t, b_first)) scores(t, b_first);
                umma_commit(&k_empty[0]);
            }
            for (int b = b_first; b < b_last && ok; ++b) {
                const int n = b - b_first, stage = n % kLgStages, next = (n + 1) % kLgStages;
                ok = wait_bounded(&v_full[stage], (n / kLgStages) & 1u, &s_abort, 0x84);
                bool fetched = false;
                for (int t = 0; t < 2 && ok; ++t) {
                    if (active(t, b)) {
                        ok = wait_bounded(&p_full[t], phase_p[t], &s_abort, 0x85);
                        if (!ok) break;
                        phase_p[t] ^= 1u;
                        tc_fence_after_sync();
                        outputs(t, b, b == (t == 0 ? half0.first : half1.first));
                        if (!active(t, b + 1)) umma_commit(&o_full[t]);
                    }
                    if (b + 1 < b_last && active(t, b + 1)) {
                        if (!fetched) {
                            ok = wait_bounded(&k_full[next], ((n + 1) / kLgStages) & 1u, &s_abort, 0x86);
                            if (!ok) break;
                            tc_fence_after_sync();
                            fetched = true;
                        }
                        scores(t, b + 1);
                    }
                }
                if (ok && b + 1 < b_last && !fetched) ok = wait_bounded(&k_full[next], ((n + 1) / kLgStages) & 1u, &s_abort, 0x86);
                if (!ok) break;
                umma_commit(&v_empty[stage]);
                if (b + 1 < b_last) umma_commit(&k_empty[next]);
            }
            if (!ok) {                                     // products in flight end before their memory is given up
                for (int i = 0; i < 64; ++i) __nanosleep(2000);
            }
        }
    } else if (warp < 8 && there) {
        // ------------------------------------------------ softmax
        const int t = warp >> 2, r = warp * 32 + lane, w4 = warp & 3;
        const LargeHalf half = t == 0 ? half0 : half1;
        const uint32_t ts = tmem + t * 128 + ((uint32_t)(w4 * 32) << 16), to = t_o + t * 128 + ((uint32_t)(w4 * 32) << 16);
        const RowKeys keys = row_keys(p, tile, r0 + r);
        const int w_first = min(rows - 1, 32 * warp), w_last = min(rows - 1, 32 * warp + 31);
        const int all_lo = rows > 0 ? row_keys(p, tile, r0 + w_last).lo : 0, all_hi = rows > 0 ? row_keys(p, tile, r0 + w_first).hi : 0;
        float m = -INFINITY, l = 0.0f, e0 = 0.0f;
        {
            const int pg = range.last > range.first ? page_at(range.first) : -1;
            const float s = pg >= 0 ? __ldg(p.v_scales + (int64_t)pg * p.heads + head) : 0.0f;
            e0 = s > 0.0f ? (float)((int)((__float_as_uint(s) >> 23) & 255u) - 127) : 0.0f;
        }
        // what 16 keys' scores are scaled by: lane k < 8 fetches it for 16 keys k, a block ahead
        auto info_of = [&](int pg) {
            float4 f = make_float4(0.0f, -INFINITY, 0.0f, 0.0f);      // not there: seen by no row
            if (pg >= 0) {
                const int64_t at = (int64_t)pg * p.heads + head;
                const float ks = __ldg(p.k_scales + at), vs = __ldg(p.v_scales + at);
                f.x = ks * p.scale_log2;
                f.y = vs > 0.0f ? (float)((int)((__float_as_uint(vs) >> 23) & 255u) - 127) - e0 : 0.0f;
                f.z = __uint_as_float((unsigned)(127 - max(-126, min(126, (int)f.y))) << 23);
            }
            return f;
        };
        auto page_of = [&](int b) { return b < half.last ? page_at(b * kLgKeys + 16 * (lane & 7)) : -1; };
        float4 info = make_float4(0.f, 0.f, 0.f, 0.f);
        int page_next = -1;
        if (half.first < half.last) {
            info = info_of(page_of(half.first));
            page_next = page_of(half.first + 1);
        }
        bool ok = true;
        for (int b = half.first, n = 0; b < half.last; ++b, ++n) {
            float4 *blk = s_info[warp][n & 1];
            if (lane < 8) blk[lane] = info;
            __syncwarp();
            if (b + 1 < half.last) {
                info = info_of(page_next);
                page_next = page_of(b + 2);
            }
            ok = __all_sync(0xffffffffu, wait_bounded(&s_full[t], n & 1u, &s_abort, 0x87));
            if (!ok) break;
            tc_fence_after_sync();
            const int key0 = b * kLgKeys;
            const bool edge = key0 < all_lo || key0 + kLgKeys > all_hi;
            const float top = edge ? large_row_max<true>(ts, blk, keys.lo - key0, keys.hi - key0) : large_row_max<false>(ts, blk, 0, 0);
            if (__any_sync(0xffffffffu, top > m + kRaise)) {
                const float raised = fmaxf(m, top), f = m == raised ? 1.0f : ex2(m - raised);
                m = raised;
                l *= f;
                if (n > 0) {                               // the products up to the last block have ended: s_full comes behind them
#pragma unroll 1
                    for (int c = 0; c < DP / 16; ++c) {
                        uint32_t v[16];
                        tmem_ld_32x16(to + c * 16, v);
                        tmem_ld_wait();
#pragma unroll
                        for (int j = 0; j < 16; ++j) v[j] = __float_as_uint(__uint_as_float(v[j]) * f);
                        tmem_st_32x16(to + c * 16, v);
                    }
                }
            }
            const float um = m == -INFINITY ? 0.0f : m;
            l = edge ? large_row_exp<true>(ts, blk, keys.lo - key0, keys.hi - key0, um, l) : large_row_exp<false>(ts, blk, 0, 0, um, l);
            tmem_st_wait();
            tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) mbar_arrive(&p_full[t]);
        }
        if (half.first < half.last && ok) {
            ok = __all_sync(0xffffffffu, wait_bounded(&o_full[t], 0, &s_abort, 0x88));
            tc_fence_after_sync();
        }
        const bool any = half.first < half.last && ok;
        if (128 * t + 32 * w4 < rows) {                    // whole warps
            const int64_t at = ((int64_t)tile.slot * p.heads + head) * kLargeRows + r;
#pragma unroll 1
            for (int c = 0; c < DP / 16; ++c) {
                uint32_t v[16];
                if (any) {
                    tmem_ld_32x16(to + c * 16, v);
                    tmem_ld_wait();
                } else {
#pragma unroll
                    for (int j = 0; j < 16; ++j) v[j] = 0u;
                }
                if (r >= rows || c * 16 >= p.dim) continue;
#pragma unroll
                for (int j = 0; j < 16; j += 4) {
                    const float4 s = make_float4(__uint_as_float(v[j]), __uint_as_float(v[j + 1]), __uint_as_float(v[j + 2]), __uint_as_float(v[j + 3]));
                    const int d = c * 16 + j;
                    if (tile.splits > 1) *reinterpret_cast<float4 *>(p.part_y + at * p.dim + d) = s;
                    else store_attention_row<T>(p, tile, head, r0 + r, d, s, l, m, e0);
                }
            }
            if (tile.splits > 1 && r < rows) p.part_ml[at] = make_float4(m + e0, l, e0, 0.0f);
        }
    }

    tc_fence_before_sync();
    __syncthreads();
    if (warp == 16) {
        tc_fence_after_sync();
        tmem_dealloc(tmem, 512);
    }
}

}  // namespace dybit
