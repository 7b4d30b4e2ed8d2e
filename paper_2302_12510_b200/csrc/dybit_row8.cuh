// Rows of real numbers on their way to 8-bit codes: 16-byte vectors of them, their largest magnitude, the power-of-two
// scale that follows from it, and their codes.  What the checkpoints and the key-value cache share.
#pragma once

#include "dybit_code8.cuh"

namespace dybit {

constexpr int64_t kMaxGridX = 2147483647;
constexpr int kCkptThreads = 256;

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

}  // namespace dybit
