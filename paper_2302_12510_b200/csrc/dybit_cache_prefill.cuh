// Attention over the 8-bit cache for tiles of 256 query rows: both products on the tensor cores (tcgen05).
//
// A block takes a tile's keys 64 at a time.  Roles, a warp each or several:
//   decode    codes -> f16 or bf16 keys and f16 values in shared memory, in the operands' swizzled layouts (nothing but
//             codes crosses the memory system, and the 256 rows share what is decoded); four warps for keys, four for values
//   issue     a warp to each half t of the rows: S_t = Q_t K^T into TMEM and O_t += P_t V with P_t read from TMEM
//   softmax   four warps to a half, a thread to a row: S_t -> P_t in place (f16), the running maximum and sum, and now and then a
//             factor on O_t
// Scores have two buffers for each half and run two blocks ahead, so that the softmax warps find the next block's ready.
// Per 128 keys and SM the products take 2048 clocks of the tensor core, the exponentials 2048 of the special-function units,
// decoding and softmax together about 1800 issue slots of each scheduler, and the operands about 2300 clocks of shared memory; it
// takes about 5900, and no one of these bounds it.  A prompt of 2048 tokens behind 2048, 188 us: 174 without the exponentials, 178
// without the maxima, 184 without decoding; blocks of 128 keys with one buffer of scores 198.  What remains is the way of a block of
// scores through the two softmax warps of a scheduler, and some 12,000 clocks where a part of a tile begins and ends.
#pragma once

#include "dybit_cache_attention.cuh"
#include "dybit_cache_turns.cuh"

namespace dybit {

constexpr int kLgKeys = 64;                  // keys of a block
constexpr int kLgThreads = 576;              // warps: 2 x 4 softmax, 4 + 4 decode, 2 issue
constexpr int kLgStages = 4;

constexpr int kLgQPanel = 128 * 128, kLgPanel = kLgKeys * 128;       // bytes of 64 head elements of a half's queries, of a block's keys or values
template <int DP> __host__ __device__ constexpr int large_smem_bytes() { return (DP / 64) * (2 * kLgQPanel + 2 * kLgStages * kLgPanel) + 1024; }

// Descriptor of an operand whose rows (128 bytes, 64 columns) run along the contraction: groups of eight rows 1024 bytes apart, the
// next 64 columns a panel further on.
__device__ __forceinline__ uint32_t large_values_lo(uint32_t smem_addr) { return ((smem_addr & 0x3ffffu) >> 4) | ((uint32_t)(kLgPanel >> 4) << 16); }
__host__ __device__ constexpr uint32_t large_values_hi() { return (uint32_t)(1024 >> 4) | (1u << 14) | (2u << 29); }

// What an issuing warp asks of the tensor core: all lanes take part, one of them issues.  (A warp that stays together keeps addresses
// and descriptors in uniform registers, where the instructions want them.)
//   D (128 x N, TMEM) (+)= A (128 x 16, shared memory) * B
__device__ __forceinline__ void umma_ss_elect(uint32_t tmem_d, uint32_t a_lo, uint32_t b_lo, uint32_t desc_hi, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n.reg .pred p, q;\n.reg .b64 da, db;\nelect.sync _|q, 0xffffffff;\nsetp.ne.b32 p, %5, 0;\nmov.b64 da, {%1, %3};\nmov.b64 db, {%2, %3};\n"
        "@q tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %4, p;\n}\n" ::"r"(tmem_d),
        "r"(a_lo), "r"(b_lo), "r"(desc_hi), "r"(idesc), "r"(accumulate)
        : "memory");
}
//   D (128 x N, TMEM) (+)= A (128 x 16 f16, TMEM, two elements to a column) * B
__device__ __forceinline__ void umma_ts_elect(uint32_t tmem_d, uint32_t tmem_a, uint32_t b_lo, uint32_t b_hi, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n.reg .pred p, q;\n.reg .b64 db;\nelect.sync _|q, 0xffffffff;\nsetp.ne.b32 p, %5, 0;\nmov.b64 db, {%2, %3};\n"
        "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %4, p;\n}\n" ::"r"(tmem_d),
        "r"(tmem_a), "r"(b_lo), "r"(b_hi), "r"(idesc), "r"(accumulate)
        : "memory");
}
// Arrives on the barrier once every product that the warp has asked for is done (the same lane is elected every time).
__device__ __forceinline__ void umma_commit_elect(uint32_t bar_addr) {
    asm volatile(
        "{\n.reg .pred q;\nelect.sync _|q, 0xffffffff;\n@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n}\n" ::"r"(bar_addr)
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
// The wait for a load whose registers are used behind it only.
__device__ __forceinline__ void tmem_ld_wait_for(uint32_t (&r)[32]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]),
                   "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]),
                   "+r"(r[16]), "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]), "+r"(r[23]),
                   "+r"(r[24]), "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]), "+r"(r[30]), "+r"(r[31])
                 :
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

// The blocks of keys of a half of a tile's rows: those between the first and the last key that one of its rows sees, within the
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

__device__ __forceinline__ bool large_next(const CacheAttn &p, CachePlace &at, const CachePlace &end, int n_tiles, LargePart &w) {
    w.part.tile = p.tiles[at.tile];
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

// Waits for block n's phase of a pair of barriers.
__device__ __forceinline__ bool wait_turn(uint64_t (&bars)[2], uint32_t n, volatile uint32_t *abort_flag, unsigned site) {
    const Turn w = turn_of(n);
    return wait_bounded(&bars[w.bar], w.parity, abort_flag, site);
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
    constexpr int UNITS = DP / 16, ROWS = 128 / UNITS, PASSES = kLgKeys / ROWS, HALF = PASSES / 2, TILE = (DP / 64) * kLgPanel;
    const int lane = threadIdx.x & 31, i = threadIdx.x & 127, u = i % UNITS, row0 = i / UNITS;
    const bool in_dim = u * 16 < p.dim;
    const int page_mask = (1 << p.page_shift) - 1;
    const int64_t page_bytes = (int64_t)p.heads * p.dim << p.page_shift;
    const int head = t.part.head;
    const uint8_t *base = codes + ((int64_t)head * p.dim << p.page_shift) + u * 16;
    auto load = [&](int key, int pg) {                     // key: its number in the sequence
        uint4 v = make_uint4(0u, 0u, 0u, 0u);
        if (pg >= 0 && in_dim) v = __ldg(reinterpret_cast<const uint4 *>(base + pg * page_bytes + (key & page_mask) * p.dim));
        return v;
    };
    auto page_at = [&](int b) { return b < t.last ? large_page(p, t.table, t.part.tile.len, b * kLgKeys + 16 * (lane & 3)) : -1; };
    // values whose scale is 0 are zeros whatever their codes
    auto held = [&](int pg) { return !VALUES || (pg >= 0 && __ldg(p.v_scales + (int64_t)pg * p.heads + head) > 0.0f); };
    // lane k < 4 has the page of 16 keys k of a block
    int page_now = page_at(t.first), page_next = page_at(t.first + 1);
    bool held_now = held(page_now);
    uint4 c[HALF];
#pragma unroll
    for (int s = 0; s < HALF; ++s) {
        const int key = row0 + s * ROWS;
        c[s] = load(t.first * kLgKeys + key, __shfl_sync(0xffffffffu, page_now, key >> 4));
    }
    // threads of the second panel store their second half first: eight lanes then fill eight different 16-byte columns
    const bool swap = DP == 128 && (u & 4) != 0;
    const int chunk = 2 * (u & 3) + (swap ? 1 : 0);
    uint8_t *const dst0 = tiles + (u >> 2) * kLgPanel + row0 * 128;
    for (int b = t.first; b < t.last; ++b, ++n) {
        const uint32_t stage = n % kLgStages;
        const int page_after = page_at(b + 2);
        const bool held_next = held(page_next);
        if (!__all_sync(0xffffffffu, wait_bounded(&empty[stage], ((n / kLgStages) & 1u) ^ 1u, abort_flag, 0x82))) return false;
        const uint32_t holds = __ballot_sync(0xffffffffu, held_now);
#pragma unroll 1
        for (int h = 0; h < 2; ++h) {
            uint8_t *dst = dst0 + stage * TILE + h * (HALF * ROWS * 128);
            const int ahead = h == 0 ? page_now : page_next;
#pragma unroll
            for (int s = 0; s < HALF; ++s) {
                const int key = row0 + (h * HALF + s) * ROWS, next = row0 + ((h ^ 1) * HALF + s) * ROWS;
                uint4 w = c[s];
                if (VALUES && !((holds >> (key >> 4)) & 1u)) w = make_uint4(0u, 0u, 0u, 0u);
                c[s] = load((b + h) * kLgKeys + next, __shfl_sync(0xffffffffu, ahead, next >> 4));
                const unsigned a0 = swap ? w.z : w.x, a1 = swap ? w.w : w.y, a2 = swap ? w.x : w.z, a3 = swap ? w.y : w.w;
                uint4 lo, hi;
                decode_word<T>(a0, lo.x, lo.y);
                decode_word<T>(a1, lo.z, lo.w);
                decode_word<T>(a2, hi.x, hi.y);
                decode_word<T>(a3, hi.z, hi.w);
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

// The largest of a row's scores (TMEM address ts), times 16 keys' factor plus their exponent.  The loops of all roles are kept
// short: written out they no longer fit the instruction caches together, and a block of keys took twice the time.
template <bool EDGE>
__device__ __forceinline__ float large_row_max(uint32_t ts, const float4 *blk, int lo, int hi) {
    float top = -INFINITY;
#pragma unroll 1
    for (int c = 0; c < kLgKeys / 32; ++c) {
        uint32_t v[32];
        tmem_ld_32x32(ts + c * 32, v);
        tmem_ld_wait_for(v);
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            const float4 f = blk[2 * c + g];
            if (EDGE) {
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    const float y = __fmaf_rn(__uint_as_float(v[g * 16 + j]), f.x, f.y);
                    const int key = c * 32 + g * 16 + j;
                    top = key >= lo && key < hi ? fmaxf(top, y) : top;
                }
            } else {                                       // the factor is not negative: the largest product has the largest score
                float a = __uint_as_float(v[g * 16]);
#pragma unroll
                for (int j = 1; j < 15; j += 2) a = fmaxf(fmaxf(a, __uint_as_float(v[g * 16 + j])), __uint_as_float(v[g * 16 + j + 1]));
                a = fmaxf(a, __uint_as_float(v[g * 16 + 15]));
                top = fmaxf(top, __fmaf_rn(a, f.x, f.y));
            }
        }
    }
    return top;
}

// The row's probabilities at maximum um, written over its scores; returns l with their sum.
template <bool EDGE>
__device__ __forceinline__ float large_row_exp(uint32_t ts, const float4 *blk, int lo, int hi, float um, float l) {
#pragma unroll 1
    for (int c = 0; c < kLgKeys / 32; ++c) {
        uint32_t v[32], pr[16];
        tmem_ld_32x32(ts + c * 32, v);
        tmem_ld_wait_for(v);
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            const float4 f = blk[2 * c + g];
            const float shift = f.y - um;
            const uint64_t cc = pack_f32x2(f.x, f.x), ss = pack_f32x2(shift, shift);
            uint64_t sum = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                float2 s = unpack_f32x2(fma_f32x2(pack_f32x2(__uint_as_float(v[g * 16 + 2 * j]), __uint_as_float(v[g * 16 + 2 * j + 1])), cc, ss));
                if (EDGE) {
                    const int key = c * 32 + g * 16 + 2 * j;
                    if (key < lo || key >= hi) s.x = -INFINITY;
                    if (key + 1 < lo || key + 1 >= hi) s.y = -INFINITY;
                }
                s.x = ex2(s.x), s.y = ex2(s.y);
                sum = j == 0 ? pack_f32x2(s.x, s.y) : add_f32x2(sum, pack_f32x2(s.x, s.y));
                pr[g * 8 + j] = pack_f16(s.x, s.y);
            }
            const float2 s = unpack_f32x2(sum);
            l = __fmaf_rn(s.x + s.y, f.z, l);
        }
        tmem_st_32x16(ts + c * 16, pr);                    // (columns whose scores have been read)
    }
    return l;
}

template <typename T, int DP>
__global__ void __launch_bounds__(kLgThreads, 1)
cache_large_kernel(const uint8_t *__restrict__ k_codes, const uint8_t *__restrict__ v_codes, const CacheAttn p) {
    constexpr int KS = DP / 16, QTILE = (DP / 64) * kLgQPanel, TILE = (DP / 64) * kLgPanel;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint8_t *s_q = smem, *s_k = smem + 2 * QTILE, *s_v = s_k + kLgStages * TILE;
    // s_full, p_full, o_done: a half's scores, probabilities and products with values, its blocks in turn
    __shared__ uint64_t k_full[kLgStages], k_empty[kLgStages], v_full[kLgStages], v_empty[kLgStages], q_full[2], s_full[2][2], p_full[2][2], o_done[2][2];
    __shared__ uint32_t s_tmem, s_abort;
    __shared__ float4 s_info[8][2][kLgKeys / 16];          // softmax warp, parity, 16 keys: {x's factor, values' exponent, 2^-exponent, -}

    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int s = 0; s < kLgStages; ++s) {
            mbar_init(&k_full[s], 4);
            mbar_init(&k_empty[s], 2);
            mbar_init(&v_full[s], 4);
            mbar_init(&v_empty[s], 2);
        }
        for (int t = 0; t < 2; ++t) {
            mbar_init(&q_full[t], 4);
            for (int j = 0; j < 2; ++j) {
                mbar_init(&o_done[t][j], 1);
                mbar_init(&s_full[t][j], 1);
                mbar_init(&p_full[t][j], 4);
            }
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
    const int n_tiles = __ldg(p.counts), n_blocks = __ldg(p.counts + 1);
    CachePlace at = {0, 0, 0}, end = {0, 0, 0};
    if ((int)blockIdx.x < n_blocks) at = cache_place(p.starts[blockIdx.x]), end = cache_place(p.starts[blockIdx.x + 1]);
    const uint32_t tmem = s_tmem;
    // columns: two buffers of 64 scores for each half (32 of which become the probabilities), then the outputs
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
    } else if (warp >= 16) {
        // ------------------------------------------------ issue: warp 16 + t for half t
        constexpr uint32_t ab = __is_same(T, __half) ? 0u : 1u;
        constexpr uint32_t idesc_s = umma_idesc(1u, ab, 128, kLgKeys), idesc_o = umma_idesc(1u, 0u, 128, DP) | (1u << 16);
        const int t = warp - 16;
        const uint32_t d_s = tmem + t * 128, d_o = t_o + t * 128, q_lo = umma_desc_lo(smem_u32(s_q + t * QTILE));
        const uint32_t k_lo = umma_desc_lo(smem_u32(s_k)), v_lo = large_values_lo(smem_u32(s_v));
        uint32_t done = 0, asked = 0, parts = 0, n = 0;    // blocks so far: of the half (outputs, scores), its parts, blocks of both halves
        bool ok = true;
        auto uniform = [](int v) { return __shfl_sync(0xffffffffu, v, 0); };
        while (ok && large_next(p, at, end, n_tiles, w)) {
            const int first = uniform(w.first), last = uniform(w.last), h_first = uniform(t == 0 ? w.half[0].first : w.half[1].first),
                      h_last = uniform(t == 0 ? w.half[0].last : w.half[1].last);
            // the half's queries are there, and the part before has taken what lies in its columns
            if (h_first < h_last) ok = __all_sync(0xffffffffu, wait_bounded(&q_full[t], parts++ & 1u, &s_abort, 0x89));
            // scores run two blocks ahead of the outputs
#pragma unroll 1
            for (int b = first - 2; ok && b < last; ++b) {
                if (b >= first) {
                    const uint32_t stage = n % kLgStages;
                    // (a half that does not see the block lets go of it in its turn all the same, once it has been there)
                    ok = __all_sync(0xffffffffu, wait_bounded(&v_full[stage], (n / kLgStages) & 1u, &s_abort, 0x84));
                    if (ok && b >= h_first && b < h_last) {
                        ok = __all_sync(0xffffffffu, wait_turn(p_full[t], done, &s_abort, 0x85));
                        if (!ok) break;
                        tc_fence_after_sync();
                        const uint32_t a = d_s + (done & 1u) * 64, v = v_lo + stage * (TILE >> 4);
#pragma unroll
                        for (int k = 0; k < kLgKeys / 16; ++k)         // 16 keys are 2048 bytes of values and 8 columns of probabilities
                            umma_ts_elect(d_o, a + k * 8, v + k * 128, large_values_hi(), idesc_o, (uint32_t)(b != h_first || k != 0));
                        umma_commit_elect(smem_u32(&o_done[t][turn_of(done).bar]));
                        ++done;
                    }
                    if (!ok) break;
                    umma_commit_elect(smem_u32(&v_empty[stage]));
                    ++n;
                }
                if (b + 2 < last) {
                    const uint32_t i = n + (b < first ? b + 2 - first : 1), stage = i % kLgStages;       // (n counts block b already)
                    ok = __all_sync(0xffffffffu, wait_bounded(&k_full[stage], (i / kLgStages) & 1u, &s_abort, 0x86));
                    if (!ok) break;
                    if (b + 2 >= h_first && b + 2 < h_last) {
                        tc_fence_after_sync();
                        const uint32_t d = d_s + (asked & 1u) * 64, kd = k_lo + stage * (TILE >> 4);
#pragma unroll
                        for (int k = 0; k < KS; ++k)
                            umma_ss_elect(d, q_lo + (((k >> 2) * kLgQPanel + (k & 3) * 32) >> 4), kd + (((k >> 2) * kLgPanel + (k & 3) * 32) >> 4), umma_desc_hi<128>(),
                                          idesc_s, (uint32_t)(k != 0));
                        umma_commit_elect(smem_u32(&s_full[t][turn_of(asked).bar]));
                        ++asked;
                    }
                    umma_commit_elect(smem_u32(&k_empty[stage]));
                }
            }
        }
        if (!ok) {                                         // products in flight end before their memory is given up
            for (int i = 0; i < 64; ++i) __nanosleep(2000);
        }
    } else {
        // ------------------------------------------------ softmax
        const int t = warp >> 2, r = warp * 32 + lane, w4 = warp & 3, row0 = 32 * w4;
        const uint32_t t_s = tmem + t * 128 + ((uint32_t)(w4 * 32) << 16), to = t_o + t * 128 + ((uint32_t)(w4 * 32) << 16);
        uint32_t n = 0;                                    // blocks of this half so far
        bool ok = true;
        while (ok && large_next(p, at, end, n_tiles, w)) {
            const CacheTile &tile = w.part.tile;
            const LargeHalf half = t == 0 ? w.half[0] : w.half[1];
            const int head = w.part.head, rows = w.rows;
            const bool any = half.first < half.last;
            const int token = (w.r0 + r) / p.group, h = head * p.group + (w.r0 + r - token * p.group);
            if (any) {
                // the warp's rows of queries, 16 bytes to a lane; keys lie in the order that their codes are decoded in: of every four
                // elements 0, 2, 1, 3
                constexpr int CH = DP / 8, PER = 32 / CH;  // chunks of a row, rows at a time
                const int c = lane % CH;
                uint8_t *const dst = s_q + t * QTILE + (c >> 3) * kLgQPanel;
                auto chunk = [&](int i) { return dst + (row0 + i) * 128 + (((c & 7) ^ ((row0 + i) & 7)) << 4); };
                const int qr = w.r0 + 32 * warp + lane / CH;
                int qt = qr / p.group, qh = qr - qt * p.group;
#pragma unroll 1
                for (int i = lane / CH; i < 32; i += PER) {
                    const T *q = static_cast<const T *>(p.q) + (tile.row + qt) * p.q_token + (head * p.group + qh) * p.q_head + c * 8;
                    for (qh += PER; qh >= p.group; qh -= p.group) ++qt;
                    if (32 * warp + i >= rows || c * 8 >= p.dim) {
                        *reinterpret_cast<uint4 *>(chunk(i)) = make_uint4(0u, 0u, 0u, 0u);
                    } else if (p.q_vec16) {
                        cp_async_16_full(smem_u32(chunk(i)), q);
                    } else {
                        T *e = reinterpret_cast<T *>(chunk(i));
#pragma unroll 1
                        for (int j = 0; j < 8; ++j) e[j] = q[j];
                    }
                }
                cp_async_commit();
                cp_async_wait_group<0>();
#pragma unroll 2
                for (int i = lane / CH; i < 32; i += PER) {
                    uint4 *at_c = reinterpret_cast<uint4 *>(chunk(i));
                    uint4 v = *at_c;
                    v.x = nan_for_infinity<T>(v.x), v.y = nan_for_infinity<T>(v.y), v.z = nan_for_infinity<T>(v.z), v.w = nan_for_infinity<T>(v.w);
                    *at_c = make_uint4(__byte_perm(v.x, v.y, 0x5410), __byte_perm(v.x, v.y, 0x7632), __byte_perm(v.z, v.w, 0x5410), __byte_perm(v.z, v.w, 0x7632));
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
            auto page_of = [&](int b) { return b < half.last ? large_page(p, w.table, tile.len, b * kLgKeys + 16 * (lane & 3)) : -1; };
            // what 16 keys' scores are scaled by: lane k < 4 fetches it for 16 keys k, a block ahead
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
                // exponent of a value scale that a row sees: of the first block's 16 keys those with the first key that all rows of the warp
                // see, or else the last
                const float s = pg >= 0 ? __ldg(p.v_scales + (int64_t)pg * p.heads + head) : 0.0f;
                const int seen = min(max(0, all_lo - half.first * kLgKeys) / 16, kLgKeys / 16 - 1);
                e0 = __shfl_sync(0xffffffffu, s > 0.0f ? (float)((int)((__float_as_uint(s) >> 23) & 255u) - 127) : 0.0f, seen);
                info = info_of(pg);
            }
            for (int b = half.first; b < half.last; ++b, ++n) {
                float4 *blk = s_info[warp][n & 1];
                if (lane < kLgKeys / 16) blk[lane] = info;
                __syncwarp();
                if (b + 1 < half.last) {
                    info = info_of(page_next);
                    page_next = page_of(b + 2);
                }
                ok = __all_sync(0xffffffffu, wait_turn(s_full[t], n, &s_abort, 0x87));
                if (!ok) break;
                tc_fence_after_sync();
                const int key0 = b * kLgKeys;
                const uint32_t ts = t_s + (n & 1u) * 64;
                const bool edge = key0 < all_lo || key0 + kLgKeys > all_hi;
                const float top = edge ? large_row_max<true>(ts, blk, keys.lo - key0, keys.hi - key0) : large_row_max<false>(ts, blk, 0, 0);
                if (__any_sync(0xffffffffu, top > m + kRaise)) {
                    const float raised = fmaxf(m, top), f = m == raised ? 1.0f : ex2(m - raised);
                    m = raised;
                    l *= f;
                    if (b > half.first) {                  // once the products up to the last block have ended
                        ok = __all_sync(0xffffffffu, wait_turn(o_done[t], n - 1u, &s_abort, 0x88));
                        if (!ok) break;
                        tc_fence_after_sync();
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
                if (lane == 0) mbar_arrive(&p_full[t][turn_of(n).bar]);
            }
            if (any && ok) {
                // (products end in the order that they are asked for: the last block's is the end of all)
                ok = __all_sync(0xffffffffu, wait_turn(o_done[t], n - 1u, &s_abort, 0x88));
                tc_fence_after_sync();
            }
            if (ok && 32 * warp < rows) {                  // whole warps
                const int64_t to_row = (int64_t)w.part.slot * kLargeRows + r;
                T *y = static_cast<T *>(p.y) + (tile.row + token) * p.y_token + h * p.y_head;
                [[maybe_unused]] auto in_range = [&](int d) {
                    return token < tile.n && tile.row >= 0 && tile.row + token < p.tokens && d <= p.dim && w.part.slot < 2 * kLargeBlocks && r < kLargeRows;
                };
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
                    if (r < rows && c * 16 < p.dim && DYBIT_CHECK(in_range(c * 16 + 16), 0x87)) {
                        if (w.part.slot >= 0) {
#pragma unroll
                            for (int j = 0; j < 16; j += 4)
                                *reinterpret_cast<float4 *>(p.part_y + large_part_at(to_row, c * 16 + j, p.dim)) = make_float4(f[j], f[j + 1], f[j + 2], f[j + 3]);
                        } else {
                            uint32_t u[8];
#pragma unroll
                            for (int j = 0; j < 8; ++j) u[j] = pack2<T>(f[2 * j] * inv * up, f[2 * j + 1] * inv * up);
                            if (p.y_vec16) {
                                *reinterpret_cast<uint4 *>(y + c * 16) = make_uint4(u[0], u[1], u[2], u[3]);
                                *reinterpret_cast<uint4 *>(y + c * 16 + 8) = make_uint4(u[4], u[5], u[6], u[7]);
                            } else {
#pragma unroll
                                for (int j = 0; j < 16; ++j) y[c * 16 + j] = from_f32<T>(f[j] * inv * up);
                            }
                        }
                    }
                    __syncwarp();
                }
                if (r < rows && DYBIT_CHECK(in_range(0), 0x8e)) {
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
