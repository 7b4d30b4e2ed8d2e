// Activation checkpoints: 8-bit codes with one power-of-two scale per row, written and read back.  Both kernels are
// bound by HBM: save reads the activation once and keeps the row in registers between its maximum and its codes, load
// reads one byte per element.
#pragma once

#include "dybit_code8.cuh"

namespace dybit {

constexpr int kCkptThreads = 256;
constexpr int kCkptPerThread = 32;           // elements of a row that a thread keeps in registers

// scale 2^(ceil(log2 amax) - top) and its inverse from the bits of the largest finite |x|.
__device__ __forceinline__ void pow2_scale(unsigned amax_bits, int top, float *scale, float *inv) {
    int e = amax_bits == 0u ? 0 : (int)((amax_bits + 0x7fffffu) >> 23) - 127 - top;
    e = max(-126, min(126, e));
    *scale = __uint_as_float((unsigned)(e + 127) << 23);
    *inv = __uint_as_float((unsigned)(127 - e) << 23);
}

// A 16-byte vector of a row at column `col` as raw words; columns from `cols` on read as zeros.
template <typename T, bool VEC>
__device__ __forceinline__ uint4 load_row_vec(const T *__restrict__ row, int64_t col, int64_t cols) {
    constexpr int E = 16 / (int)sizeof(T);
    uint4 v = make_uint4(0u, 0u, 0u, 0u);
    if (VEC && col + E <= cols) {
        v = __ldg(reinterpret_cast<const uint4 *>(row + col));
    } else if (col < cols) {
        T e[E];
#pragma unroll
        for (int i = 0; i < E; ++i) e[i] = col + i < cols ? row[col + i] : from_f32<T>(0.0f);
        v = *reinterpret_cast<const uint4 *>(e);
    }
    return v;
}

template <typename T> struct VecFloats { float4 f[sizeof(T) == 4 ? 1 : 2]; };
template <typename T>
__device__ __forceinline__ VecFloats<T> vec_floats(const uint4 &v) {
    VecFloats<T> o;
    if constexpr (sizeof(T) == 4) {
        o.f[0] = make_float4(__uint_as_float(v.x), __uint_as_float(v.y), __uint_as_float(v.z), __uint_as_float(v.w));
    } else {
        const float2 a = unpack2<T>(v.x), b = unpack2<T>(v.y), c = unpack2<T>(v.z), d = unpack2<T>(v.w);
        o.f[0] = make_float4(a.x, a.y, b.x, b.y);
        o.f[1] = make_float4(c.x, c.y, d.x, d.y);
    }
    return o;
}

// Largest bit pattern of |x| over vectors: patterns order like the numbers, with infinities and then NaN on top.  16-bit
// elements are compared two at a time.
template <typename T>
__device__ __forceinline__ unsigned vec_absmax(const uint4 &v, unsigned best) {
    if constexpr (sizeof(T) == 4) {
        return max(max(max(best, v.x & 0x7fffffffu), v.y & 0x7fffffffu), max(v.z & 0x7fffffffu, v.w & 0x7fffffffu));
    } else {
        best = __vmaxu2(__vmaxu2(best, v.x & 0x7fff7fffu), v.y & 0x7fff7fffu);
        return __vmaxu2(__vmaxu2(best, v.z & 0x7fff7fffu), v.w & 0x7fff7fffu);
    }
}
// The pattern as that of an fp32 number (NaN stays NaN, infinity infinity).
template <typename T>
__device__ __forceinline__ unsigned absmax_as_f32(unsigned best) {
    if constexpr (sizeof(T) == 4) return best;
    const unsigned top = max(best & 0xffffu, best >> 16);
    if constexpr (__is_same(T, __half)) return __float_as_uint(__half2float(__ushort_as_half((unsigned short)top)));
    return top << 16;
}
template <typename T>
__device__ __forceinline__ float vec_absmax_finite(const uint4 &v, float best) {
    const VecFloats<T> o = vec_floats<T>(v);
#pragma unroll
    for (int i = 0; i < (sizeof(T) == 4 ? 1 : 2); ++i)
        best = fmaxf(best, __uint_as_float(max(max(finite_abs_bits(o.f[i].x), finite_abs_bits(o.f[i].y)),
                                               max(finite_abs_bits(o.f[i].z), finite_abs_bits(o.f[i].w)))));
    return best;
}

// Codes of a vector, stored at column `col` (row strides are multiples of 16, so the store is aligned and in the row).
// LIMIT: for rows with infinities or NaN.
template <typename T, bool SIGNED, bool LIMIT>
__device__ __forceinline__ void store_vec_codes(const uint4 &v, float inv, uint8_t *dst) {
    const VecFloats<T> o = vec_floats<T>(v);
    if constexpr (!LIMIT && __is_same(T, __nv_bfloat16)) {
        *reinterpret_cast<uint2 *>(dst) = encode8_bf16<SIGNED>(v, (__float_as_uint(inv) >> 16) * 0x00010001u);
    } else if constexpr (sizeof(T) == 4) {
        *reinterpret_cast<unsigned *>(dst) = encode4_8<SIGNED, LIMIT>(o.f[0], inv);
    } else {
        *reinterpret_cast<uint2 *>(dst) = make_uint2(encode4_8<SIGNED, LIMIT>(o.f[0], inv), encode4_8<SIGNED, LIMIT>(o.f[1], inv));
    }
}

struct CkptSave {
    const void *x;
    int64_t rows, cols, ld;
    uint8_t *codes;
    int64_t stride;              // bytes of a row of codes
    int64_t width;               // columns written: cols and the code 0 behind them
    float *scales;
    int top;
};

// W warps per row (8 / W rows per block).  Rows of up to 1024 * W columns stay in registers; longer ones (W = 8) are
// read twice, the second time from the caches.
template <typename T, bool SIGNED, bool VEC, int W, bool LONG>
__global__ void __launch_bounds__(kCkptThreads) checkpoint_save_kernel(const CkptSave p) {
    constexpr int E = 16 / (int)sizeof(T), NV = kCkptPerThread / E, TPR = W * 32;
    __shared__ unsigned s_best[8];
    pdl_enter();
    const int sub = threadIdx.x / TPR, t = threadIdx.x % TPR;
    const int64_t row = (int64_t)blockIdx.x * (8 / W) + sub;
    if (W < 8 && row >= p.rows) return;                    // whole warps; with W > 1 the row's warps meet in a named barrier
    const T *x = static_cast<const T *>(p.x) + row * p.ld;
    uint4 v[NV];
    unsigned best = 0u;
    if constexpr (!LONG) {
#pragma unroll
        for (int i = 0; i < NV; ++i) v[i] = load_row_vec<T, VEC>(x, (int64_t)(i * TPR + t) * E, p.cols);
#pragma unroll
        for (int i = 0; i < NV; ++i) best = vec_absmax<T>(v[i], best);
    } else {
        for (int64_t c = (int64_t)t * E; c < p.cols; c += TPR * E) best = vec_absmax<T>(load_row_vec<T, VEC>(x, c, p.cols), best);
    }
    best = absmax_as_f32<T>(best);
    // maximum of the row; a row with infinities or NaN takes the maximum of its finite elements instead
    auto row_max = [&](unsigned b) {
        b = __reduce_max_sync(0xffffffffu, b);
        if constexpr (W > 1) {
            if ((threadIdx.x & 31) == 0) s_best[threadIdx.x >> 5] = b;
            asm volatile("bar.sync %0, %1;" ::"r"(1 + sub), "n"(TPR) : "memory");
#pragma unroll
            for (int w = 0; w < W; ++w) b = max(b, s_best[sub * W + w]);
        }
        return b;
    };
    best = row_max(best);
    const bool special = best >= 0x7f800000u;
    if (special) {
        float finite = 0.0f;
        if constexpr (!LONG) {
#pragma unroll
            for (int i = 0; i < NV; ++i) finite = vec_absmax_finite<T>(v[i], finite);
        } else {
            for (int64_t c = (int64_t)t * E; c < p.cols; c += TPR * E)
                finite = vec_absmax_finite<T>(load_row_vec<T, VEC>(x, c, p.cols), finite);
        }
        if constexpr (W > 1) asm volatile("bar.sync %0, %1;" ::"r"(1 + sub), "n"(TPR) : "memory");   // s_best is free again
        best = row_max(__float_as_uint(finite));
    }
    float scale, inv;
    pow2_scale(best, p.top, &scale, &inv);
    if (t == 0 && DYBIT_CHECK(row < p.rows, 0x60)) p.scales[row] = scale;
    uint8_t *out = p.codes + row * p.stride;
    if constexpr (!LONG) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int64_t c = (int64_t)(i * TPR + t) * E;
            if (c < p.width && DYBIT_CHECK(row < p.rows && c + E <= p.stride, 0x65)) {
                if (special) store_vec_codes<T, SIGNED, true>(v[i], inv, out + c);
                else store_vec_codes<T, SIGNED, false>(v[i], inv, out + c);
            }
        }
    } else {
        for (int64_t c = (int64_t)t * E; c < p.width; c += TPR * E)
            if (DYBIT_CHECK(row < p.rows && c + E <= p.stride, 0x65))
                store_vec_codes<T, SIGNED, true>(load_row_vec<T, VEC>(x, c, p.cols), inv, out + c);
    }
}

struct CkptLoad {
    const uint8_t *codes;
    int64_t stride;
    const float *scales;
    int64_t scale_stride;
    int64_t rows, cols, ld;
    void *y;
    int64_t chunks;              // of a row: 4 vectors per lane of a warp
};

// One warp per chunk of a row: four 16-byte output vectors per lane, their codes loaded first.
template <typename T, bool SIGNED, bool VEC>
__global__ void __launch_bounds__(kCkptThreads) checkpoint_load_kernel(const CkptLoad p) {
    constexpr int E = 16 / (int)sizeof(T), NV = 4;
    pdl_enter();
    const int lane = threadIdx.x & 31;
    const int64_t item = (int64_t)blockIdx.x * (kCkptThreads / 32) + (threadIdx.x >> 5);
    const int64_t row = item / p.chunks, chunk = item - row * p.chunks;
    if (row >= p.rows) return;
    const uint8_t *in = p.codes + row * p.stride;
    T *out = static_cast<T *>(p.y) + row * p.ld;
    const float scale = __ldg(p.scales + row * p.scale_stride);
    const int64_t c0 = chunk * (NV * 32 * E) + lane * E;
    if constexpr (!VEC) {
        // rows of y that start anywhere: neighbouring lanes take neighbouring elements, so their stores fill whole sectors
        const int64_t first = chunk * (NV * 32 * E) + lane;
        unsigned code[NV * E];
#pragma unroll
        for (int i = 0; i < NV * E; ++i) code[i] = first + i * 32 < p.cols ? __ldg(in + first + i * 32) : 0u;
#pragma unroll
        for (int i = 0; i < NV * E; ++i)
            if (first + i * 32 < p.cols)
                out[first + i * 32] = from_f32<T>(__fmul_rn(__uint_as_float(decode2<SIGNED>(code[i] * 0x0101u) << 16), scale));
        return;
    }
    uint2 w[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int64_t c = c0 + i * (32 * E);
        w[i] = make_uint2(0u, 0u);
        if (c < p.cols && DYBIT_CHECK(c + E <= p.stride, 0x66)) {      // rows of codes are padded to 16: the whole vector is there
            if constexpr (E == 4) w[i].x = __ldg(reinterpret_cast<const unsigned *>(in + c));
            else w[i] = __ldg(reinterpret_cast<const uint2 *>(in + c));
        }
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int64_t c = c0 + i * (32 * E);
        if (c >= p.cols) continue;
        float f[E];
#pragma unroll
        for (int j = 0; j < E / 4; ++j) {
            const float4 d = decode4<SIGNED>(j == 0 ? w[i].x : w[i].y);
            f[4 * j] = __fmul_rn(d.x, scale);
            f[4 * j + 1] = __fmul_rn(d.y, scale);
            f[4 * j + 2] = __fmul_rn(d.z, scale);
            f[4 * j + 3] = __fmul_rn(d.w, scale);
        }
        if (VEC && c + E <= p.cols) {
            uint4 o;
            if constexpr (E == 4) {
                o = make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
            } else {
                o = make_uint4(pack2<T>(f[0], f[1]), pack2<T>(f[2], f[3]), pack2<T>(f[4], f[5]), pack2<T>(f[6], f[7]));
            }
            *reinterpret_cast<uint4 *>(out + c) = o;
        } else {
#pragma unroll
            for (int j = 0; j < E; ++j)
                if (c + j < p.cols) out[c + j] = from_f32<T>(f[j]);
        }
    }
}

// ------------------------------------------------------------------ host side

inline bool fmt8_ok(dybit_fmt f, dybit_status *st) {
    if (!fmt_ok(f)) {
        *st = DYBIT_ERR_INVALID_ARG;
        return false;
    }
    if (f.bits != 8) {
        *st = DYBIT_ERR_UNSUPPORTED;
        return false;
    }
    return true;
}

constexpr int64_t kMaxGridX = 2147483647;

// Arguments that describe a matrix of 8-bit codes.
static dybit_status check_codes(const void *codes, int64_t rows, int64_t cols, int64_t stride, dybit_fmt fmt) {
    dybit_status st;
    if (!fmt8_ok(fmt, &st)) return st;
    if (rows < 0 || cols < 0 || stride < cols) return DYBIT_ERR_INVALID_ARG;
    if (rows > 0 && cols > 0 && codes == nullptr) return DYBIT_ERR_INVALID_ARG;
    if (stride % 16 != 0 || !aligned(codes, 16)) return DYBIT_ERR_ALIGNMENT;
    return DYBIT_OK;
}

// A matrix of real numbers whose rows can be moved in 16-byte vectors.
static bool rows_vec16(const void *p, int64_t ld, int elem) { return aligned(p, 16) && (ld * elem) % 16 == 0; }

template <typename T, bool SIGNED, bool VEC>
static dybit_status launch_checkpoint_save(const CkptSave &p, cudaStream_t s) {
    auto go = [&](auto kernel, int rows_per_block) {
        const int64_t blocks = (p.rows + rows_per_block - 1) / rows_per_block;
        if (blocks > kMaxGridX) return DYBIT_ERR_UNSUPPORTED;
        launch_k(kernel, dim3((unsigned)blocks), dim3(kCkptThreads), 0, s, p);
        return launch_status();
    };
    if (p.width <= 1024) return go(checkpoint_save_kernel<T, SIGNED, VEC, 1, false>, 8);
    if (p.width <= 2048) return go(checkpoint_save_kernel<T, SIGNED, VEC, 2, false>, 4);
    if (p.width <= 4096) return go(checkpoint_save_kernel<T, SIGNED, VEC, 4, false>, 2);
    if (p.width <= 8192) return go(checkpoint_save_kernel<T, SIGNED, VEC, 8, false>, 1);
    return go(checkpoint_save_kernel<T, SIGNED, VEC, 8, true>, 1);
}

template <typename T, bool SIGNED, bool VEC>
static dybit_status launch_checkpoint_load(CkptLoad p, cudaStream_t s) {
    constexpr int kChunk = 4 * 32 * (16 / (int)sizeof(T));
    p.chunks = (p.cols + kChunk - 1) / kChunk;
    const int64_t blocks = (p.rows * p.chunks + kCkptThreads / 32 - 1) / (kCkptThreads / 32);
    if (blocks > kMaxGridX) return DYBIT_ERR_UNSUPPORTED;
    launch_k(checkpoint_load_kernel<T, SIGNED, VEC>, dim3((unsigned)blocks), dim3(kCkptThreads), 0, s, p);
    return launch_status();
}

// Calls f<T, SIGNED, VEC>() for run-time values of the three.
template <typename F>
static dybit_status with_elem(dybit_dtype t, bool is_signed, bool vec, F &&f) {
    auto sv = [&](auto elem) {
        using T = decltype(elem);
        if (is_signed) return vec ? f.template operator()<T, true, true>() : f.template operator()<T, true, false>();
        return vec ? f.template operator()<T, false, true>() : f.template operator()<T, false, false>();
    };
    switch (t) {
        case DYBIT_F32: return sv(float());
        case DYBIT_BF16: return sv(__nv_bfloat16());
        default: return sv(__half());
    }
}

struct SaveLauncher {
    const CkptSave &p;
    cudaStream_t s;
    template <typename T, bool SIGNED, bool VEC> dybit_status operator()() const { return launch_checkpoint_save<T, SIGNED, VEC>(p, s); }
};
struct LoadLauncher {
    const CkptLoad &p;
    cudaStream_t s;
    template <typename T, bool SIGNED, bool VEC> dybit_status operator()() const { return launch_checkpoint_load<T, SIGNED, VEC>(p, s); }
};

}  // namespace dybit

extern "C" {

dybit_status dybit_checkpoint_save(const void *x, dybit_dtype tx, int64_t rows, int64_t cols, int64_t ld, dybit_fmt fmt,
                                   int top, void *codes, int64_t row_stride_bytes, float *scales, void *stream) {
    using namespace dybit;
    dybit_status st = check_codes(codes, rows, cols, row_stride_bytes, fmt);
    if (st != DYBIT_OK) return st;
    if (!dtype_ok(tx) || ld < cols || top < 0 || top >= mag_bits(fmt)) return DYBIT_ERR_INVALID_ARG;
    if (rows == 0) return DYBIT_OK;
    if (scales == nullptr || (cols > 0 && x == nullptr)) return DYBIT_ERR_INVALID_ARG;
    if (!aligned(x, dtype_bytes(tx)) || !aligned(scales, 4)) return DYBIT_ERR_ALIGNMENT;
    const int64_t padded = round_up(cols, 128);
    CkptSave p = {x, rows, cols, ld, static_cast<uint8_t *>(codes), row_stride_bytes, padded < row_stride_bytes ? padded : row_stride_bytes,
                  scales, top};
    return with_elem(tx, fmt.is_signed != 0, rows_vec16(x, ld, dtype_bytes(tx)), SaveLauncher{p, static_cast<cudaStream_t>(stream)});
}

dybit_status dybit_checkpoint_load(const void *codes, int64_t row_stride_bytes, const float *scales, int64_t scale_stride,
                                   int64_t rows, int64_t cols, dybit_fmt fmt, void *y, dybit_dtype ty, int64_t ld,
                                   void *stream) {
    using namespace dybit;
    dybit_status st = check_codes(codes, rows, cols, row_stride_bytes, fmt);
    if (st != DYBIT_OK) return st;
    if (!dtype_ok(ty) || ld < cols || scale_stride < 0) return DYBIT_ERR_INVALID_ARG;
    if (rows == 0 || cols == 0) return DYBIT_OK;
    if (scales == nullptr || y == nullptr) return DYBIT_ERR_INVALID_ARG;
    if (!aligned(y, dtype_bytes(ty)) || !aligned(scales, 4)) return DYBIT_ERR_ALIGNMENT;
    CkptLoad p = {static_cast<const uint8_t *>(codes), row_stride_bytes, scales, scale_stride, rows, cols, ld, y, 0};
    return with_elem(ty, fmt.is_signed != 0, rows_vec16(y, ld, dtype_bytes(ty)), LoadLauncher{p, static_cast<cudaStream_t>(stream)});
}

}  // extern "C"
