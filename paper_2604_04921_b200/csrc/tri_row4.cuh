// Rows of 128 components in 4 bits: TRI_ROW4_BYTES bytes, as the header describes them at tri_append.
//
// Why this layout.  Word g of the 16-byte unit t holds components 8 t .. 8 t + 7 of group g, so that a lane of attention that
// loads one unit has 8 components of each group, what a matrix instruction per group needs (see tri_attend4.cuh), and that 32 g +
// 8 t .. + 7, one word, is a run of 16 bytes of a bf16 row.  In a word, nibbles i and i + 4 are neighbours 2 i, 2 i + 1: masked with
// 0x000f000f << 4 i they are a pair of 16-bit values in order.  80 bytes is an odd number of 16-byte units: eight rows side by side
// in shared memory are read without bank conflicts.
#pragma once
#include "tri_score_tma.cuh"

namespace tri {

constexpr int kRow4Bytes = TRI_ROW4_BYTES, kRow4Scales = 64, kRow4Centres = 72;

__device__ __forceinline__ float min_nan(float a, float b)
{
    float r;
    asm("min.NaN.f32 %0, %1, %2;\n" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float min_nan(float a, float b, float c)
{
    float r;
    asm("min.NaN.f32 %0, %1, %2, %3;\n" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
__device__ __forceinline__ float max_nan(float a, float b, float c)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2, %3;\n" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
__device__ __forceinline__ float max_nan(float a, float b)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;\n" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

// Scale and centre of a group from its smallest and largest value.  (8 hi + 7 lo) / 15 as (hi / 2 + 7 lo / 16) / (15 / 16), which
// cannot overflow; with bf16 inputs every step up to the division is exact or rounded once, so that c is the correctly rounded
// one.  s is exact for that c: the differences are rounded upwards (7 s or 8 s for the s sought is an fp32 number, which they do
// not pass; to nearest, c - lo becomes c for a tiny lo < 0, and s ends a step below), the quotient by 7 is taken with a factor
// below 1 / 7, which leaves s right or a step below, and 7 s, exact, is compared with the difference.  (Divisions rounded upwards cost
// 7 % of a whole prompt's append.)  With a NaN or an infinity among the values, or a range that fp32 does not hold, c - lo is not
// finite.  Returns whether c or s lies so near the border of two bf16 numbers that lo and hi, if they are off by a few steps of fp32,
// may have put it on the wrong side.
__device__ __forceinline__ bool row4_group(float lo, float hi, float &s, float &c)
{
    const float c32 = __fdiv_rn(fmaf(hi, 0.5f, lo * 0.4375f), 0.9375f);
    c = bf16_lo(cvt_bf16x2(0.f, c32));
    const float over = __fsub_ru(hi, c), below = __fsub_ru(c, lo), need = fmaxf(over * 0x1.249248p-3f, below * 0.125f);
    // rounded up to bf16; the smallest normal number, where that is more
    uint32_t up = max((__float_as_uint(need) + 0xffffu) & 0xffff0000u, 0x00800000u);
    if (__uint_as_float(up) * 7.f < over) up += 0x10000u;
    s = need > 0.f ? __uint_as_float(up) : 0.f;
    if (!(fabsf(below) < INFINITY)) { c = __uint_as_float(0x7fc00000u); s = 0.f; }
    return ((__float_as_uint(c32) + 0x8010u) & 0xffffu) <= 0x20u || (need > 0.f && ((__float_as_uint(need) + 0x10u) & 0xffffu) <= 0x20u);
}

// Pairs of fp32 values in one register pair: sm_100a adds and multiplies both in one instruction.
typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 pair_of(float a, float b)
{
    f32x2 r;
    asm("mov.b64 %0, {%1, %2};\n" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void parts_of(f32x2 x, float &a, float &b) { asm("mov.b64 {%0, %1}, %2;\n" : "=f"(a), "=f"(b) : "l"(x)); }
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b)
{
    f32x2 r;
    asm("add.rn.f32x2 %0, %1, %2;\n" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b)
{
    f32x2 r;
    asm("mul.rn.f32x2 %0, %1, %2;\n" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c)
{
    f32x2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;\n" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}

// Codes of pairs of components, inv = 1 / s.  Adding 1.5 * 2^23 + 8 rounds a quotient to the nearest integer (ties to even) and leaves
// the code in the low bits of the sum.  TIES: the quotient is an approximate one, corrected by its exact remainder (Markstein's
// division): where (x - c) / s lies halfway between two codes, which is common with bf16 values, it is exact.  Otherwise it may be
// off by 2^-20, and `off` receives the largest distance of a quotient from its code.
template <bool TIES>
__device__ __forceinline__ void row4_codes(f32x2 x, float s, float inv, float c, float &off, uint32_t &a, uint32_t &b)
{
    constexpr float kMagic = 12582912.f + 8.f;
    const f32x2 magic = pair_of(kMagic, kMagic), inv2 = pair_of(inv, inv), v = add2(x, pair_of(-c, -c));
    f32x2 t;
    if (TIES) {
        const f32x2 q = mul2(v, inv2);
        t = add2(fma2(fma2(q, pair_of(-s, -s), v), inv2, q), magic);
    } else {
        t = fma2(v, inv2, magic);
        float e0, e1;
        parts_of(fma2(v, inv2, fma2(t, pair_of(-1.f, -1.f), magic)), e0, e1);
        off = fmaxf(off, fmaxf(fabsf(e0), fabsf(e1)));
    }
    float t0, t1;
    parts_of(t, t0, t1);
    a = __float_as_uint(t0); b = __float_as_uint(t1);
}
constexpr uint32_t kRow4Bias = 0x4b400000u * 0x11111111u;    // what the bits of 1.5 * 2^23 add to a word of eight shifted codes

// The 8 components a word stands for in bf16, rounded once: a nibble or-ed under 0x4300 is the bf16 value 128 + code, which less 136
// is exact, and the multiply-add rounds (code - 8) s + c.  s and c are pairs of the same value.
__device__ __forceinline__ uint4 row4_bf16(uint32_t w, uint32_t s, uint32_t c)
{
    uint32_t r[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t n = ((w >> 4 * i) & 0x000f000fu) | 0x43004300u;
        asm("sub.rn.bf16x2 %0, %0, %1;\n" : "+r"(n) : "r"(0x43084308u));
        asm("fma.rn.bf16x2 %0, %1, %2, %3;\n" : "=r"(r[i]) : "r"(n), "r"(s), "r"(c));
    }
    return make_uint4(r[0], r[1], r[2], r[3]);
}

// The 8 components a word stands for.
__device__ __forceinline__ void row4_values(uint32_t w, float s, float c, float *x)
{
#pragma unroll
    for (int d = 0; d < 8; ++d) {
        const uint32_t n = (w >> 4 * ((d >> 1) + 4 * (d & 1))) & 15u;
        x[d] = fmaf(__uint_as_float(0x4b000000u | n) - 8388616.f, s, c);       // 2^23 + code, less 2^23 + 8
    }
}

}  // namespace tri
