// The 4-bit format of weights and cached rows.
//
// A row of n values is cut into groups.  A group keeps two bfloat16 numbers, scale and origin; its level q = 0..15 stands for
//   round( origin + scale * (16 + q) ),   rounded once, to the handle's type (bfloat16 or float32).
// Levels count from 16 because 16..31 are the bfloat16 numbers 0x4180 | q << 3: a level becomes a number by one shift and
// one and-or, two levels at a time, and one packed multiply-add makes it the value.  (Levels from 0 took a
// subtraction more; the origin is then farther from the values, by 16 scales, and rounding it to 8 bits moves all levels of a group
// together: by 1/16 of a level at most where the group spans zero, by n/17 of one behind an offset of n times the group's range.  bfloat16
// values there lie 2n/17 levels apart themselves; float32 values behind an offset of 1000 times their range all end on one level.)
// Eight consecutive values share a 32-bit word, at the nibbles that begin at bits 3, 19, 7, 23, 11, 27, 31 (and 0..2), 15: a pair's two
// lie 16 bits apart and three shifts bring all pairs to bits 3..6 and 19..22, where a bfloat16 number takes them.
#pragma once

#include "common.cuh"

namespace ctcsd {

constexpr int kQ4Group = 32;                   // values of a cached row that share a scale

#ifdef __CUDACC__

// (a & mask) | base as one instruction: an instruction takes one constant of its own, so both are kept in registers (as
// constants the two steps stay apart, and an earlier draft head took 113 us in place of 102 for a row of the 7B shape).
__device__ __forceinline__ uint32_t q4_level_bits(uint32_t a) {
    uint32_t mask, base, r;
    asm("mov.b32 %0, 0x00780078;" : "=r"(mask));
    asm("mov.b32 %0, 0x41804180;" : "=r"(base));
    asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(r) : "r"(a), "r"(mask), "r"(base));
    return r;
}
// The eight levels of a word as four pairs of bfloat16 numbers 16..31: pair i = values 2i, 2i + 1.
__device__ __forceinline__ void q4_pairs(uint32_t w, uint32_t (&c)[4]) {
    c[0] = q4_level_bits(w);
    c[1] = q4_level_bits(w >> 4);
    c[2] = q4_level_bits(w >> 8);
    c[3] = q4_level_bits(__funnelshift_l(w, w, 4));
}
// The same for two words of two rows at once: pair i of `even` / `odd` = values 2i / 2i + 1 of the rows a and b.
__device__ __forceinline__ void q4_pairs2(uint32_t a, uint32_t b, uint32_t (&even)[4], uint32_t (&odd)[4]) {
    // (turned so that nibbles do not cross the halves: the low one holds values 0, 2, 4, 7, the high one 1, 3, 5, 6)
    const uint32_t ra = __funnelshift_r(a, a, 3), rb = __funnelshift_r(b, b, 3);
    const uint32_t lo = __byte_perm(ra, rb, 0x5410), hi = __byte_perm(ra, rb, 0x7632);
    even[0] = q4_level_bits(lo << 3);
    even[1] = q4_level_bits(lo >> 1);
    even[2] = q4_level_bits(lo >> 5);
    odd[3] = q4_level_bits(lo >> 9);
    odd[0] = q4_level_bits(hi << 3);
    odd[1] = q4_level_bits(hi >> 1);
    odd[2] = q4_level_bits(hi >> 5);
    even[3] = q4_level_bits(hi >> 9);
}
// First bit of value i (0..7) of a word.
__host__ __device__ constexpr int q4_bit(int i) { return (i < 6 ? 3 + 4 * (i >> 1) + 16 * (i & 1) : (i == 6 ? 31 : 15)); }
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
    const uint32_t q = __funnelshift_r(w, w, q4_bit(i)) & 15u;
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
    const float s = __bfloat162float(__float2bfloat16_rn(__fmul_rn(__fsub_rn(hi, lo), 1.f / 15.f)));
    const float o = __bfloat162float(__float2bfloat16_rn(__fsub_rn(lo, __fmul_rn(16.f, s))));
    if (!(fabsf(s) < INFINITY) || !(fabsf(o) < INFINITY)) return 0x7fc00000u;
    return (__float_as_uint(s) >> 16) | (__float_as_uint(o) & 0xffff0000u);
}
// Level of v in a group, rounded half to even.  (Rarely called: see q4_word.)
static __device__ __noinline__ uint32_t q4_level(float v, float scale, float origin) {
    if (!(scale > 0.f)) return 0u;
    const float q = rintf(__fsub_rn(__fdiv_rn(__fsub_rn(v, origin), scale), 16.f));
    return (uint32_t)fminf(fmaxf(q, 0.f), 15.f);
}
// The word of eight values.  A level is a division, which took most of the time of storing rows; so it is found by the group's reciprocal (off by
// less than 31 * 2^-22 from the division's result), and only where that lies within 2^-15 of a tie by the division itself.
// (32 prompts of 1024-4096 rows of 8 heads, stored and read back: 340 us with divisions, 262 us so.)
__device__ __forceinline__ uint32_t q4_word(const float (&v)[8], uint32_t so) {
    const float s = bf16lo(so), o = bf16hi(so);
    if (!(s > 0.f)) return 0u;
    const float r = __frcp_rn(s), magic = 12582912.f;                        // 1.5 * 2^23: adding it rounds to a whole number
    float q[8];
    if (fabsf(o) <= 100.f * s && s >= 1.17549435e-38f) {
        // no limits needed: the scale's rounding (2^-8 of 15 levels) and the origin's (2^-8 of 100 at most) move a level by 0.45 at most.
        // (a subnormal scale has fewer than 8 bits: there it can be 0.9, and a level 16)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float d = __fsub_rn(v[i], o), x = __fmaf_rn(d, r, -16.f);
            q[i] = __fsub_rn(__fadd_rn(x, magic), magic);
            if (fabsf(__fsub_rn(x, q[i])) > 0.5f - 3.0517578125e-5f) {
                // (14 bits hold scale times tie, so the difference is exact; the quotient of a d that is farther than 2^-20 from it is not the tie)
                const float tie = __fadd_rn(floorf(x), 0.5f), diff = __fsub_rn(d, __fmul_rn(__fadd_rn(tie, 16.f), s));
                if (diff == 0.f) q[i] = rintf(tie);
                else if (fabsf(diff) > fabsf(d) * 9.5367431640625e-7f) q[i] = diff > 0.f ? tie + 0.5f : tie - 0.5f;
                else q[i] = (float)q4_level(v[i], s, o);
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) q[i] = (float)q4_level(v[i], s, o);
    }
    // the word turned back by 3: nibbles of values 0, 2, 4, 7 in the low half, 1, 3, 5, 6 in the high one
    const float lo = fmaf(q[7], 4096.f, fmaf(q[4], 256.f, fmaf(q[2], 16.f, q[0])));
    const float hi = fmaf(q[6], 4096.f, fmaf(q[5], 256.f, fmaf(q[3], 16.f, q[1])));
    const uint32_t w = __byte_perm(__float_as_uint(__fadd_rn(lo, 8388608.f)), __float_as_uint(__fadd_rn(hi, 8388608.f)), 0x5410);
    return __funnelshift_l(w, w, 3);
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
