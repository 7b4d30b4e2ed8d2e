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

// The blocks of 128 keys of a half of a tile's rows: those between the first and the last key that one of its rows sees, within the
// part's.
struct LargeHalf { int first, last; };

// A part of a tile as all roles of a block see it.
struct LargePart {
    CachePart part;
    int r0, rows, first, last;   // rows of the tile; blocks of both halves
    KeyRange range;
    LargeHalf half[2];
    const int *table;
};

__device__ __forceinline__ bool large_next(const CacheAttn &p, CacheStart &at, const CacheStart &end, int n_tiles, LargePart &w) {
    if (!cache_next(p, blockIdx.x, at, end, n_tiles, w.part)) return false;
    const CacheTile &t = w.part.tile;
    w.r0 = t.tile * kLargeRows;
    w.rows = min(kLargeRows, t.n * p.group - w.r0);
    w.range = part_keys(p, w.part, w.r0, kLargeRows, kLgKeys);
    w.table = p.table + t.seq * p.table_stride;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        LargeHalf b = {0, 0};
        if (128 * h < w.rows) {
            const RowKeys a = row_keys(p, t, w.r0 + 128 * h), z = row_keys(p, t, w.r0 + min(w.rows, 128 * h + 128) - 1);
            if (z.hi > a.lo) {
                b.first = max(w.range.first, a.lo & ~(kLgKeys - 1)) / kLgKeys;
                b.last = max(b.first, min(w.range.last, (z.hi + kLgKeys - 1) & ~(kLgKeys - 1)) / kLgKeys);
            }
        }
        w.half[h] = b;
    }
    const bool none0 = w.half[0].first == w.half[0].last, none1 = w.half[1].first == w.half[1].last;
    w.first = none0 ? w.half[1].first : none1 ? w.half[0].first : min(w.half[0].first, w.half[1].first);
    w.last = none0 ? w.half[1].last : none1 ? w.half[0].last : max(w.half[0].last, w.half[1].last);
    if (none0 && none1) w.last = w.first;
    return true;
}

// Page of the 16 keys from `key` on, or -1.
__device__ __forceinline__ int large_page(const CacheAttn &p, const int *table, int len, int key) {
    const int pg = key < len ? __ldg(table + (key >> p.page_shift)) : -1;
    return (unsigned)pg < (uint64_t)p.pages ? pg : -1;
}

// Four warps turn the codes of a block's keys (or values) into 16-bit numbers of type T in the operand's layout, a unit
// of 16 codes to a thread and pass.  The codes of the next half block are on their way while one is decoded.
template <typename T, int DP, bool VALUES>
__device__ __forceinline__ bool large_decode(const CacheAttn &p, const LargePart &t, const uint8_t *__restrict__ codes, uint8_t *tiles, uint64_t *full,
                                             uint64_t *empty, volatile uint32_t *abort_flag, uint32_t &n) {
    constexpr int UNITS = DP / 16, ROWS = 128 / UNITS, PASSES = kLgKeys / ROWS, HALF = PASSES / 2, PANEL = large_panel_bytes<DP>();
    const int lane = threadIdx.x & 31, i = threadIdx.x & 127, u = i % UNITS, row0 = i / UNITS;
    const bool in_dim = u * 16 < p.dim;
    const int page_mask = (1 << p.page_shift) - 1;
    const int64_t page_bytes = (int64_t)p.heads * p.dim << p.page_shift;
    const int head = t.part.head;
    const uint8_t *base = codes + ((int64_t)head * p.dim << p.page_shift) + u * 16;
    auto load = [&](int key, int pg) {
        uint4 v = make_uint4(0u, 0u, 0u, 0u);
        if (pg >= 0 && in_dim) v = __ldg(reinterpret_cast<const uint4 *>(base + pg * page_bytes + (key & page_mask) * p.dim));
        return v;
    };
    auto page_at = [&](int b) { return b < t.last ? large_page(p, t.table, t.part.tile.len, b * kLgKeys + 16 * (lane & 7)) : -1; };
    // values whose scale is 0 are zeros whatever their codes
    auto held = [&](int pg) { return !VALUES || (pg >= 0 && __ldg(p.v_scales + (int64_t)pg * p.heads + head) > 0.0f); };
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
    const unsigned minus = p.minus_one;
    uint8_t *const dst0 = tiles + (u >> 2) * PANEL + row0 * 128;
    for (int b = t.first; b < t.last; ++b, ++n) {
        const uint32_t stage = n % kLgStages;
        const int page_after = page_at(b + 2);
        const bool held_next = held(page_next);
        if (!__all_sync(0xffffffffu, wait_bounded(&empty[stage], ((n / kLgStages) & 1u) ^ 1u, abort_flag, 0x82))) return false;
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
                uint4 lo, hi;
                decode_word<T>(a0, minus, lo.x, lo.y);
                decode_word<T>(a1, minus, lo.z, lo.w);
                decode_word<T>(a2, minus, hi.x, hi.y);
                decode_word<T>(a3, minus, hi.z, hi.w);
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
    return true;
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

template <typename T, int DP>
__global__ void __launch_bounds__(kLgThreads, 1)
cache_large_kernel(const uint8_t *__restrict__ k_codes, const uint8_t *__restrict__ v_codes, const CacheAttn p) {
    constexpr int KS = DP / 16, PANEL = large_panel_bytes<DP>(), TILE = large_tile_bytes<DP>();
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint8_t *s_q = smem, *s_k = smem + 2 * TILE, *s_v = s_k + kLgStages * TILE;
    __shared__ uint64_t k_full[kLgStages], k_empty[kLgStages], v_full[kLgStages], v_empty[kLgStages], q_full[2], s_full[2], p_full[2], o_full[2];
    __shared__ uint32_t s_tmem, s_abort;
    __shared__ float4 s_info[8][2][8];                     // softmax warp, parity, 16 keys: {x's factor, values' exponent, 2^-exponent, -}

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int s = 0; s < kLgStages; ++s) {
            mbar_init(&k_full[s], 4);
            mbar_init(&k_empty[s], 1);
            mbar_init(&v_full[s], 4);
            mbar_init(&v_empty[s], 1);
        }
        for (int t = 0; t < 2; ++t) {
            mbar_init(&q_full[t], 4);
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
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    pdl_enter();
    const int n_tiles = __ldg(p.n_tiles), n_blocks = __ldg(p.n_blocks);
    CacheStart at = p.starts[blockIdx.x], end = at;
    if ((int)blockIdx.x < n_blocks) end = p.starts[blockIdx.x + 1];
    const uint32_t tmem = s_tmem;
    // columns: scores of the halves (their first 64 become the probabilities), then the outputs
    const uint32_t t_o = tmem + 256;
    LargePart w;

    if ((int)blockIdx.x >= n_blocks) {
        // nothing to do
    } else if (warp >= 8 && warp < 16) {
        // ------------------------------------------------ decode: warps 8 .. 11 keys, 12 .. 15 values
        uint32_t n = 0;
        if (warp < 12) {
            while (large_next(p, at, end, n_tiles, w) && large_decode<T, DP, false>(p, w, k_codes, s_k, k_full, k_empty, &s_abort, n)) {}
        } else {
            while (large_next(p, at, end, n_tiles, w) && large_decode<__half, DP, true>(p, w, v_codes, s_v, v_full, v_empty, &s_abort, n)) {}
        }
    } else if (warp == 16) {
        // ------------------------------------------------ issue
        if (lane == 0) {
            constexpr uint32_t ab = __is_same(T, __half) ? 0u : 1u;
            constexpr uint32_t idesc_s = umma_idesc(1u, ab, 128, kLgKeys), idesc_o = umma_idesc(1u, 0u, 128, DP) | (1u << 16);
            uint32_t phase_p[2] = {0, 0}, phase_q[2] = {0, 0}, n = 0;      // n: blocks so far
            bool ok = true;
            auto scores = [&](int t, uint32_t stage) {
                const uint32_t qa = smem_u32(s_q + t * TILE), ka = smem_u32(s_k + stage * TILE);
#pragma unroll
                for (int k = 0; k < KS; ++k) {
                    const uint32_t off = (uint32_t)((k >> 2) * PANEL + (k & 3) * 32);
                    umma<Kind::F16>(tmem + t * 128, umma_desc_kmajor<128>(qa + off), umma_desc_kmajor<128>(ka + off), idesc_s, (uint32_t)(k != 0));
                }
                umma_commit(&s_full[t]);
            };
            auto outputs = [&](int t, uint32_t stage, bool first) {
                const uint64_t vd = large_desc_values(smem_u32(s_v + stage * TILE));
#pragma unroll
                for (int k = 0; k < kLgKeys / 16; ++k)     // 16 keys are 2048 bytes of values and 8 columns of probabilities
                    umma_ts_f16(t_o + t * 128, tmem + t * 128 + k * 8, vd + (uint64_t)(k * 128), idesc_o, (uint32_t)(!first || k != 0));
            };
            while (ok && large_next(p, at, end, n_tiles, w)) {
                auto active = [&](int t, int b) { return b >= w.half[t].first && b < w.half[t].last; };
                if (w.first == w.last) continue;
                // a half's queries are there, and the part before has taken what lies in its columns
#pragma unroll
                for (int t = 0; t < 2; ++t)
                    if (ok && w.half[t].first < w.half[t].last) {
                        ok = wait_bounded(&q_full[t], phase_q[t], &s_abort, 0x89);
                        phase_q[t] ^= 1u;
                    }
                if (ok) ok = wait_bounded(&k_full[n % kLgStages], (n / kLgStages) & 1u, &s_abort, 0x83);
                if (!ok) break;
                tc_fence_after_sync();
#pragma unroll
                for (int t = 0; t < 2; ++t)
                    if (active(t, w.first)) scores(t, n % kLgStages);
                umma_commit(&k_empty[n % kLgStages]);
                for (int b = w.first; b < w.last; ++b, ++n) {
                    const uint32_t stage = n % kLgStages, next = (n + 1) % kLgStages;
                    ok = wait_bounded(&v_full[stage], (n / kLgStages) & 1u, &s_abort, 0x84);
                    bool fetched = false;
#pragma unroll
                    for (int t = 0; t < 2; ++t) {
                        if (ok && active(t, b)) {
                            ok = wait_bounded(&p_full[t], phase_p[t], &s_abort, 0x85);
                            phase_p[t] ^= 1u;
                            tc_fence_after_sync();
                            if (ok) {
                                outputs(t, stage, b == w.half[t].first);
                                if (!active(t, b + 1)) umma_commit(&o_full[t]);
                            }
                        }
                        if (ok && b + 1 < w.last && active(t, b + 1)) {
                            if (!fetched) {
                                ok = wait_bounded(&k_full[next], ((n + 1) / kLgStages) & 1u, &s_abort, 0x86);
                                tc_fence_after_sync();
                                fetched = true;
                            }
                            if (ok) scores(t, next);
                        }
                    }
                    if (ok && b + 1 < w.last && !fetched) ok = wait_bounded(&k_full[next], ((n + 1) / kLgStages) & 1u, &s_abort, 0x86);
                    if (!ok) break;
                    umma_commit(&v_empty[stage]);
                    if (b + 1 < w.last) umma_commit(&k_empty[next]);
                }
            }
            if (!ok) {                                     // products in flight end before their memory is given up
                for (int i = 0; i < 64; ++i) __nanosleep(2000);
            }
        }
    } else if (warp < 8) {
        // ------------------------------------------------ softmax
        const int t = warp >> 2, r = warp * 32 + lane, w4 = warp & 3, row = r & 127;
        const uint32_t ts = tmem + t * 128 + ((uint32_t)(w4 * 32) << 16), to = t_o + t * 128 + ((uint32_t)(w4 * 32) << 16);
        uint32_t n = 0, parts = 0;                         // blocks of this half so far, parts in which it had some
        bool ok = true;
        while (ok && large_next(p, at, end, n_tiles, w)) {
            const CacheTile &tile = w.part.tile;
            const LargeHalf half = t == 0 ? w.half[0] : w.half[1];
            const int head = w.part.head, rows = w.rows;
            const bool any = half.first < half.last;
            if (any) {
                // a thread loads its row of queries
                const int token = (w.r0 + r) / p.group, h = head * p.group + (w.r0 + r - token * p.group);
                const T *q = r < rows ? static_cast<const T *>(p.q) + (tile.row + token) * p.q_token + h * p.q_head : nullptr;
                uint8_t *dst = s_q + t * TILE + row * 128;
#pragma unroll 8
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
                    // keys lie in the order that their codes are decoded in: of every four elements 0, 2, 1, 3
                    v = make_uint4(__byte_perm(v.x, v.y, 0x5410), __byte_perm(v.x, v.y, 0x7632), __byte_perm(v.z, v.w, 0x5410), __byte_perm(v.z, v.w, 0x7632));
                    *reinterpret_cast<uint4 *>(dst + (c >> 3) * PANEL + (((c & 7) ^ (row & 7)) << 4)) = v;
                }
                fence_proxy_async_smem();
                tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(&q_full[t]);
            }
            const RowKeys keys = row_keys(p, tile, w.r0 + r);
            // keys between these two are seen by every row of the warp that is there
            const int all_lo = row_keys(p, tile, w.r0 + min(rows - 1, 32 * warp + 31)).lo, all_hi = row_keys(p, tile, w.r0 + min(rows - 1, 32 * warp)).hi;
            float m = -INFINITY, l = 0.0f, e0 = 0.0f;
            auto page_of = [&](int b) { return b < half.last ? large_page(p, w.table, tile.len, b * kLgKeys + 16 * (lane & 7)) : -1; };
            // what 16 keys' scores are scaled by: lane k < 8 fetches it for 16 keys k, a block ahead
            auto info_of = [&](int pg) {
                float4 f = make_float4(0.0f, -INFINITY, 0.0f, 0.0f);      // not there: seen by no row
                if (pg >= 0) {
                    const int64_t i = (int64_t)pg * p.heads + head;
                    const float ks = __ldg(p.k_scales + i), vs = __ldg(p.v_scales + i);
                    f.x = ks * p.scale_log2;
                    f.y = vs > 0.0f ? (float)((int)((__float_as_uint(vs) >> 23) & 255u) - 127) - e0 : 0.0f;
                    f.z = __uint_as_float((unsigned)(127 - max(-126, min(126, (int)f.y))) << 23);
                }
                return f;
            };
            float4 info = make_float4(0.f, 0.f, 0.f, 0.f);
            int page_next = -1;
            if (any) {
                const int pg = page_of(half.first);
                page_next = page_of(half.first + 1);
                // exponent of the first keys' value scale
                const float s = pg >= 0 ? __ldg(p.v_scales + (int64_t)pg * p.heads + head) : 0.0f;
                e0 = __shfl_sync(0xffffffffu, s > 0.0f ? (float)((int)((__float_as_uint(s) >> 23) & 255u) - 127) : 0.0f, 0);
                info = info_of(pg);
            }
            for (int b = half.first; b < half.last; ++b, ++n) {
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
                    if (b > half.first) {                  // the products up to the last block have ended: s_full comes behind them
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
            if (any && ok) {
                ok = __all_sync(0xffffffffu, wait_bounded(&o_full[t], parts & 1u, &s_abort, 0x88));
                tc_fence_after_sync();
                ++parts;
            }
            if (ok && 32 * warp < rows) {                  // whole warps
                const int64_t to_row = (int64_t)w.part.slot * kLargeRows + r;
                const int token = (w.r0 + r) / p.group, h = head * p.group + (w.r0 + r - token * p.group);
                T *y = static_cast<T *>(p.y) + (tile.row + token) * p.y_token + h * p.y_head;
                // a row that sees no key: zeros (and minus infinity)
                const float inv = l == 0.0f ? 0.0f : __fdiv_rn(1.0f, l), up = __uint_as_float((unsigned)((int)e0 + 127) << 23);
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
                    float f[16];                           // (columns lie as the values were decoded)
#pragma unroll
                    for (int j = 0; j < 16; ++j) f[j] = __uint_as_float(v[(j & ~3) | ((j & 1) << 1) | ((j >> 1) & 1)]);
                    if (r < rows && c * 16 < p.dim && DYBIT_CHECK(token < tile.n, 0x87)) {
                        if (w.part.slot >= 0) {
#pragma unroll
                            for (int j = 0; j < 16; j += 4)
                                *reinterpret_cast<float4 *>(p.part_y + to_row * p.dim + c * 16 + j) = make_float4(f[j], f[j + 1], f[j + 2], f[j + 3]);
                        } else {
                            uint32_t u[8];
#pragma unroll
                            for (int j = 0; j < 8; ++j) u[j] = pack2<T>(f[2 * j] * inv * up, f[2 * j + 1] * inv * up);
                            if (p.y_vec16) {
                                *reinterpret_cast<uint4 *>(y + c * 16) = make_uint4(u[0], u[1], u[2], u[3]);
                                *reinterpret_cast<uint4 *>(y + c * 16 + 8) = make_uint4(u[4], u[5], u[6], u[7]);
                            } else {
                                T e[16];
                                memcpy(e, u, 32);
#pragma unroll
                                for (int j = 0; j < 16; ++j) y[c * 16 + j] = e[j];
                            }
                        }
                    }
                    __syncwarp();
                }
                if (r < rows) {
                    if (w.part.slot >= 0) p.part_ml[to_row] = make_float4(m + e0, l, e0, 0.0f);
                    else if (p.lse != nullptr) p.lse[(int64_t)(tile.row + token) * (p.heads * p.group) + h] = l == 0.0f ? -INFINITY : (m + __log2f(l)) * kLn2;
                }
                tc_fence_before_sync();
            }
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
