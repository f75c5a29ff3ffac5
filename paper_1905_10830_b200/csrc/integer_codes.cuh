// Codes of 8-bit integers with one scale a row: scale = fl(max|x| / 127), code = the integer nearest to x / scale (the quotient of
// the real numbers), ties to even.
#pragma once

#include "block_codes.cuh"

namespace rowcodes {

using namespace blk;

// Scale of a row from the bits of its largest magnitude; NaN where the row holds an infinity or a NaN.
__device__ __forceinline__ float row_scale(uint32_t amax_bits)
{
    if (amax_bits >= 0x7f800000u) return __int_as_float(0x7fffffff);
    // fl(a / 127): the product with fl(1 / 127), corrected by its residual (Markstein's step for quotients); equal to the quotient for all of fp32's significands
    const float a = fmaxf(__uint_as_float(amax_bits), kSmallest), q = a * (1.0f / 127.0f);
    return fmaf(fmaf(-127.0f, q, a), 1.0f / 127.0f, q);
}

// A row's scale and what its codes are computed with.
struct Coder {
    float scale, inv;
    uint32_t mask;
    __device__ __forceinline__ explicit Coder(float s)
    {
        scale = s;
        asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(s));                       // (one step off at most)
        mask = s == s ? 0xffffffffu : 0u;
    }
};
constexpr float kInteger = 12582912.0f;                       // 1.5 x 2^23: added to a value of up to 2^22 it leaves the nearest integer in the low bits
constexpr float kNearBorder = 0.5f - 1.0f / 16384.0f;

// The code next to `near_code` where x / scale comes close to the border between two.
__device__ __noinline__ static int code_at_border(float x, float scale, int near_code, float rest)
{
    const int other = near_code + (rest > 0.f ? 1 : -1);
    const float border = 0.5f * (float)(near_code + other);
    const float past = fmaf(-border, scale, x) * (rest > 0.f ? 1.f : -1.f);         // the sign is exact
    if (past != 0.f) return past > 0.f ? other : near_code;
    return near_code & 1 ? other : near_code;
}
// The largest magnitude of three values.
__device__ __forceinline__ float most_of(float a, float b, float c)
{
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(fabsf(a)), "f"(fabsf(b)), "f"(fabsf(c)));
    return d;
}
// Codes of eight values in pairs, packed.  With a NaN for its scale a row's codes are zeros.  Found with 1 / scale in fp32, whose product with x is off by
// less than 127 x 2^-22; those that come near a border between two codes are looked at again with the border's exact difference.
// (Quotients of bf16 values by a bf16 maximum lie next to borders far more often than chance has it.  8192 x 4096 normal ones by rows and columns, three tensors in turn: 59 us, 51 without the test, fp32 70 and 70; every value's
// remainder by fma instead would cost as much.)
__device__ __forceinline__ uint2 codes_of_pairs(const uint64_t (&v)[4], const Coder &c)
{
    const uint64_t inv = pair_of(c.inv, c.inv), integer = pair_of(kInteger, kInteger), minus = pair_of(-1.0f, -1.0f);
    float t[8], d[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint64_t near_code = fma2(v[i], inv, integer);
        halves(near_code, t[2 * i], t[2 * i + 1]);
        halves(fma2(v[i], inv, fma2(near_code, minus, integer)), d[2 * i], d[2 * i + 1]);
    }
    if (most_of(most_of(most_of(d[0], d[1], d[2]), d[3], d[4]), most_of(d[5], d[6], d[7]), 0.f) > kNearBorder)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float x, y;
            halves(v[i / 2], x, y);
            if (fabsf(d[i]) > kNearBorder) t[i] = kInteger + (float)code_at_border(i & 1 ? y : x, c.scale, (int)(t[i] - kInteger), d[i]);
        }
    uint32_t w[2];
#pragma unroll
    for (int h = 0; h < 2; ++h)
        w[h] = __byte_perm(__byte_perm(__float_as_uint(t[4 * h]), __float_as_uint(t[4 * h + 1]), 0x0040),
                           __byte_perm(__float_as_uint(t[4 * h + 2]), __float_as_uint(t[4 * h + 3]), 0x0040), 0x5410);
    return make_uint2(w[0] & c.mask, w[1] & c.mask);
}
__device__ __forceinline__ uint2 codes_of8(const float (&v)[8], const Coder &c)
{
    const uint64_t p[4] = {pair_of(v[0], v[1]), pair_of(v[2], v[3]), pair_of(v[4], v[5]), pair_of(v[6], v[7])};
    return codes_of_pairs(p, c);
}
// The same of four values.
__device__ __forceinline__ uint32_t codes_of4(const float *v, const Coder &c)
{
    float t[4], d[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        t[i] = fmaf(v[i], c.inv, kInteger);
        d[i] = fmaf(v[i], c.inv, -(t[i] - kInteger));
    }
    if (fmaxf(fmaxf(fabsf(d[0]), fabsf(d[1])), fmaxf(fabsf(d[2]), fabsf(d[3]))) > kNearBorder)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (fabsf(d[i]) > kNearBorder) t[i] = kInteger + (float)code_at_border(v[i], c.scale, (int)(t[i] - kInteger), d[i]);
    const uint32_t lo = __byte_perm(__float_as_uint(t[0]), __float_as_uint(t[1]), 0x0040), hi = __byte_perm(__float_as_uint(t[2]), __float_as_uint(t[3]), 0x0040);
    const uint32_t w = __byte_perm(lo, hi, 0x5410);
    return w & c.mask;
}
// One code (of the low byte).
__device__ __forceinline__ uint8_t code_of(float x, const Coder &c)
{
    const float v[4] = {x, 0.f, 0.f, 0.f};
    return (uint8_t)codes_of4(v, c);
}

}  // namespace rowcodes
