// 8-bit codes in registers: arithmetic encoder and decoder without tables, and the element types of the fine-tuning
// operators.
//
// With m magnitude bits (7 signed, 8 unsigned) the value of a magnitude code c >= 2^(m-1), which has i >= 1 leading
// ones, depends only on the distance to the top of the code axis: with 2^m - c = 2^p * (1 + y), 0 <= y < 1,
//     value(c) = 2^(m-2-p) * (2 - y).
// As floating-point bit patterns the two sides add up to a constant, since a pattern is linear in the fraction and the
// exponent alike:  bits(value) + bits(2^m - c) = (m + 253) << 23.  Decoding and encoding are one integer subtraction
// each.  Below 2^(m-1) the value is c / 2^(m-1).
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "dybit_encode.cuh"

namespace dybit {

constexpr __host__ __device__ int mag_bits8(bool is_signed) { return is_signed ? 7 : 8; }

// ---- element types

template <dybit_dtype T> struct Elem;
template <> struct Elem<DYBIT_F32> { using type = float; };
template <> struct Elem<DYBIT_BF16> { using type = __nv_bfloat16; };
template <> struct Elem<DYBIT_F16> { using type = __half; };

inline bool dtype_ok(dybit_dtype t) { return t == DYBIT_F32 || t == DYBIT_BF16 || t == DYBIT_F16; }
inline int dtype_bytes(dybit_dtype t) { return t == DYBIT_F32 ? 4 : 2; }

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }
template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }

__device__ __forceinline__ unsigned pack_bf16(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const unsigned *>(&v);
}
__device__ __forceinline__ unsigned pack_f16(float lo, float hi) {
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const unsigned *>(&v);
}
template <typename T> __device__ __forceinline__ unsigned pack2(float lo, float hi);
template <> __device__ __forceinline__ unsigned pack2<__nv_bfloat16>(float lo, float hi) { return pack_bf16(lo, hi); }
template <> __device__ __forceinline__ unsigned pack2<__half>(float lo, float hi) { return pack_f16(lo, hi); }

// The two 16-bit elements of a word as floats.
template <typename T> __device__ __forceinline__ float2 unpack2(unsigned w);
template <> __device__ __forceinline__ float2 unpack2<__nv_bfloat16>(unsigned w) {
    return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}
template <> __device__ __forceinline__ float2 unpack2<__half>(unsigned w) {
    return __half22float2(*reinterpret_cast<const __half2 *>(&w));
}

// ---- decode

__device__ __forceinline__ __nv_bfloat162 as_bf162(unsigned w) { return *reinterpret_cast<const __nv_bfloat162 *>(&w); }
__device__ __forceinline__ unsigned as_u32(__nv_bfloat162 v) { return *reinterpret_cast<const unsigned *>(&v); }

// Two codes -> their values as a pair of bf16, exact.  w holds the first code in bytes 0 and 1, the second in bytes 2 and
// 3 (unsigned: bytes 1 and 3 are not looked at).  6 instructions a pair.
template <bool SIGNED>
__device__ __forceinline__ unsigned decode2(unsigned w) {
    // 0x4300 | c is the bf16 number 128 + c for c < 128 (seven fraction bits, ulp 1)
    const __nv_bfloat162 h = as_bf162((w & 0x007f007fu) | 0x43004300u);
    const __nv_bfloat162 minus1 = as_bf162(0xbf80bf80u), c256 = as_bf162(0x43804380u), inv128 = as_bf162(0x3c003c00u);
    const unsigned g = as_u32(__hfma2(h, minus1, c256));              // 2^7 - c (signed), 2^8 - c (unsigned, top bit set)
    if constexpr (SIGNED) {
        // all codes on the curve first; below 64 it lies (64 - c) / 128 above the line c / 64
        const __nv_bfloat162 curve = as_bf162(0x82008200u - g);       // (7 + 253) << 7 in both halves, no borrow between them
        const __nv_bfloat162 above = __hfma2_relu(h, as_bf162(0xbc00bc00u), as_bf162(0x3fc03fc0u));   // max(0, 1.5 - h/128)
        return as_u32(__hsub2(curve, above)) | (w & 0x80008000u);
    } else {
        const unsigned curve = 0x82808280u - g;                       // (8 + 253) << 7
        const unsigned line = as_u32(__hfma2(h, inv128, minus1));     // c / 128 for codes without the top bit
        unsigned top;                                                 // halves of ones where bit 7 of the code is set
        asm("prmt.b32 %0, %1, 0, 0xaa88;" : "=r"(top) : "r"(w));
        return (curve & top) | (line & ~top);
    }
}

// Four codes of a word as floats.
template <bool SIGNED>
__device__ __forceinline__ float4 decode4(unsigned codes) {
    const unsigned a = decode2<SIGNED>(__byte_perm(codes, 0u, 0x1100)), b = decode2<SIGNED>(__byte_perm(codes, 0u, 0x3322));
    return make_float4(__uint_as_float(a << 16), __uint_as_float(a & 0xffff0000u), __uint_as_float(b << 16),
                       __uint_as_float(b & 0xffff0000u));
}

// ---- encode

// Magnitude code of a * inv (a = |x| signed, x unsigned): nearest value, ties to the even code.  The line below 1 and
// the curve above it are rounded on the code axis by adding 1.5 * 2^23 (the low bits are then the rounded integer, ties
// to even) and joined by an addition: the clamped line ends at 2^(m-1), where the curve starts.  NaN and negative
// numbers give 0.  LIMIT: the product may exceed the top value 2^(m-1) (an infinity); without it the caller
// knows that it does not.
template <bool SIGNED, bool LIMIT>
__device__ __forceinline__ unsigned magnitude_code8(float a, float inv) {
    constexpr int M = mag_bits8(SIGNED);
    constexpr float kMagic = 12582912.0f;
    const float line = __fmaf_rn(__saturatef(__fmul_rn(a, inv)), (float)(1 << (M - 1)), kMagic);
    float t = fmaxf(__fmul_rn(a, inv), 1.0f);
    if constexpr (LIMIT) t = fminf(t, (float)(1 << (M - 1)));
    const float dist = __fadd_rn(__uint_as_float(((unsigned)(M + 253) << 23) - __float_as_uint(t)), kMagic);   // 2^m - c
    return __float_as_uint(line) - __float_as_uint(dist) + (1u << (M - 1));
}

// Four elements -> four codes, one per byte.
template <bool SIGNED, bool LIMIT>
__device__ __forceinline__ unsigned encode4_8(const float4 v, const float inv) {
    unsigned m0, m1, m2, m3;
    if constexpr (SIGNED) {
        m0 = magnitude_code8<true, LIMIT>(fabsf(v.x), inv);
        m1 = magnitude_code8<true, LIMIT>(fabsf(v.y), inv);
        m2 = magnitude_code8<true, LIMIT>(fabsf(v.z), inv);
        m3 = magnitude_code8<true, LIMIT>(fabsf(v.w), inv);
    } else {
        m0 = magnitude_code8<false, LIMIT>(v.x, inv);
        m1 = magnitude_code8<false, LIMIT>(v.y, inv);
        m2 = magnitude_code8<false, LIMIT>(v.z, inv);
        m3 = magnitude_code8<false, LIMIT>(v.w, inv);
    }
    const unsigned mags = __byte_perm(__byte_perm(m0, m1, 0x0040), __byte_perm(m2, m3, 0x0040), 0x5410);
    if constexpr (!SIGNED) return mags;
    const unsigned tops = __byte_perm(__byte_perm(__float_as_uint(v.x), __float_as_uint(v.y), 0x0073),
                                      __byte_perm(__float_as_uint(v.z), __float_as_uint(v.w), 0x0073), 0x5410);
    // the sign goes in where the magnitude code is not zero (codes are < 128: adding 127 carries into bit 7)
    return mags | (tops & (mags + 0x7f7f7f7fu) & 0x80808080u);
}

// Eight bf16 elements (raw) -> eight codes, two elements to an instruction.  A bf16 number has as many significant bits
// as the code axis asks for, so x * 2^k, the distance to the top of the axis and both roundings fit bf16: numbers of
// 128 .. 256 have steps of 1 there, and 128 + n ends in n.  For rows without NaN and infinities.
template <bool SIGNED>
__device__ __forceinline__ uint2 encode8_bf16(const uint4 &v, unsigned inv2) {
    constexpr int M = mag_bits8(SIGNED);
    constexpr unsigned kTop = ((unsigned)(M + 253) << 7) * 0x00010001u;
    const __nv_bfloat162 one = as_bf162(0x3f803f80u), c128 = as_bf162(0x43004300u);
    const __nv_bfloat162 slope = as_bf162(SIGNED ? 0x42804280u : 0x43004300u);             // 2^(M-1)
    unsigned c[4];
    const unsigned x[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        __nv_bfloat162 t = __hmul2(as_bf162(SIGNED ? x[i] & 0x7fff7fffu : x[i]), as_bf162(inv2));
        if constexpr (!SIGNED) t = __hmax2(t, as_bf162(0u));
        const unsigned line = as_u32(__hfma2(__hmin2(t, one), slope, c128));
        const unsigned dist = as_u32(__hadd2(as_bf162(kTop - as_u32(__hmax2(t, one))), c128));
        c[i] = line + (1u << (M - 1)) * 0x00010001u - dist;    // each half is the code: no borrow
    }
    uint2 o = make_uint2(__byte_perm(c[0], c[1], 0x6420), __byte_perm(c[2], c[3], 0x6420));
    if constexpr (SIGNED) {
        o.x |= __byte_perm(x[0], x[1], 0x7531) & (o.x + 0x7f7f7f7fu) & 0x80808080u;
        o.y |= __byte_perm(x[2], x[3], 0x7531) & (o.y + 0x7f7f7f7fu) & 0x80808080u;
    }
    return o;
}

}  // namespace dybit
