// The 4-bit format of weights and cached rows.
//
// A row of n values is cut into groups.  A group keeps two bfloat16 numbers, scale and origin; its level q = 0..15 stands for
//   round( origin + scale * (16 + q) ),   rounded once, to the handle's type (bfloat16 or float32).
// Levels count from 16 because 16..31 are the bfloat16 numbers 0x4180 | q << 3: a level becomes a number by one shift and
// one and-or, two levels at a time, and one packed multiply-add makes it the value.  (Levels from 0 took a
// subtraction more; the origin is then farther from the values, by 16 scales, and rounding it to 8 bits moves all levels of a group
// together by 1/16 of a level at most where the group spans zero.)
// Eight consecutive values share a 32-bit word: value 2i at bits 4i, value 2i + 1 at bits 16 + 4i, so that the pairs that come
// out of a word are neighbours.
#pragma once

#include "common.cuh"

namespace ctcsd {

constexpr int kQ4Group = 32;                   // values of a cached row that share a scale

#ifdef __CUDACC__

// The eight levels of a word as four pairs of bfloat16 numbers 16..31: pair i = values 2i, 2i + 1.
__device__ __forceinline__ void q4_pairs(uint32_t w, uint32_t (&c)[4]) {
    c[0] = ((w << 3) & 0x00780078u) | 0x41804180u;
    c[1] = ((w >> 1) & 0x00780078u) | 0x41804180u;
    c[2] = ((w >> 5) & 0x00780078u) | 0x41804180u;
    c[3] = ((w >> 9) & 0x00780078u) | 0x41804180u;
}
__device__ __forceinline__ uint32_t q4_fma2(uint32_t a, uint32_t b, uint32_t c) {
    uint32_t d;
    asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
    return d;
}
// Scale and origin of a group, as they are stored (scale in the low half), each in both halves of a word.
__device__ __forceinline__ uint32_t q4_scale2(uint32_t so) { return __byte_perm(so, so, 0x1010); }
__device__ __forceinline__ uint32_t q4_origin2(uint32_t so) { return __byte_perm(so, so, 0x3232); }

// The values of a word in bfloat16, four pairs.
__device__ __forceinline__ uint4 q4_values_bf16(uint32_t w, uint32_t so) {
    uint32_t c[4];
    q4_pairs(w, c);
    const uint32_t s = q4_scale2(so), o = q4_origin2(so);
    return make_uint4(q4_fma2(c[0], s, o), q4_fma2(c[1], s, o), q4_fma2(c[2], s, o), q4_fma2(c[3], s, o));
}
// Value i (0..7) of a word in float32.
__device__ __forceinline__ float q4_value_f32(uint32_t w, int i, float scale, float origin) {
    const uint32_t q = (w >> (4 * (i >> 1) + 16 * (i & 1))) & 15u;
    return __fmaf_rn(__uint_as_float(0x41800000u | (q << 19)), scale, origin);
}

// Minimum and maximum that let a NaN through.
__device__ __forceinline__ float min_nan(float a, float b) {
    float r;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

// Scale and origin of a group with the limits lo, hi (float32 steps, each rounded to nearest).  A group that holds a NaN or an
// infinity, or whose range leaves the type: scale 0, origin NaN.
__device__ __forceinline__ uint32_t q4_scale_origin(float lo, float hi) {
    const float s = __bfloat162float(__float2bfloat16_rn(__fdiv_rn(__fsub_rn(hi, lo), 15.f)));
    const float o = __bfloat162float(__float2bfloat16_rn(__fsub_rn(lo, __fmul_rn(16.f, s))));
    if (!(fabsf(s) < INFINITY) || !(fabsf(o) < INFINITY)) return 0x7fc00000u;
    return (__float_as_uint(s) >> 16) | (__float_as_uint(o) & 0xffff0000u);
}
// Level of v in a group, rounded half to even.
__device__ __forceinline__ uint32_t q4_level(float v, float scale, float origin) {
    if (!(scale > 0.f)) return 0u;
    const float q = rintf(__fsub_rn(__fdiv_rn(__fsub_rn(v, origin), scale), 16.f));
    return (uint32_t)fminf(fmaxf(q, 0.f), 15.f);
}
// The word of eight values.
__device__ __forceinline__ uint32_t q4_word(const float (&v)[8], uint32_t so) {
    const float s = bf16lo(so), o = bf16hi(so);
    uint32_t w = 0u;
#pragma unroll
    for (int i = 0; i < 8; ++i) w |= q4_level(v[i], s, o) << (4 * (i >> 1) + 16 * (i & 1));
    return w;
}

// Eight neighbouring values of an activation-type array (16- or 32-byte aligned), widened.
template <typename T> __device__ __forceinline__ void load8(const T* p, float (&v)[8]);
template <> __device__ __forceinline__ void load8<__nv_bfloat16>(const __nv_bfloat16* p, float (&v)[8]) {
    const uint4 w = *reinterpret_cast<const uint4*>(p);
    v[0] = bf16lo(w.x); v[1] = bf16hi(w.x); v[2] = bf16lo(w.y); v[3] = bf16hi(w.y);
    v[4] = bf16lo(w.z); v[5] = bf16hi(w.z); v[6] = bf16lo(w.w); v[7] = bf16hi(w.w);
}
template <> __device__ __forceinline__ void load8<float>(const float* p, float (&v)[8]) {
    const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}

#endif  // __CUDACC__

}  // namespace ctcsd
