// What the kernels of block-scaled 8-bit matrices share: the scale and the codes of a block, and loads and stores
// of eight consecutive values of an fp32 or bf16 tensor.
#pragma once

#include <cuda_bf16.h>
#include <stdint.h>

#include "device_utils.cuh"

namespace blk {

constexpr int kBlock = 128;                                   // values that share a scale
constexpr float kSmallest = 7.888609052210118e-31f;           // 2^-100: scales of smaller blocks stay normal numbers, and so do their reciprocals
constexpr float kPerMax = 1.0f / 448.0f;                      // 448 is the largest e4m3 value

__device__ __forceinline__ uint32_t abs_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// Scale of a block from the bits of its largest magnitude (compared as integers, in which infinities and NaN are the
// largest: they reach the scale, which is NaN then, and with it everything that is computed from the block).
__device__ __forceinline__ float scale_of(uint32_t amax_bits)
{
    if (amax_bits >= 0x7f800000u) return __int_as_float(0x7fffffff);
    return __fmul_rn(fmaxf(__uint_as_float(amax_bits), kSmallest), kPerMax);
}

// Codes of four values: rounded to the nearest e4m3 value, ties to even, beyond the range the largest.
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d, float inv)
{
    uint32_t codes;
    asm("{\n\t.reg .b64 p, q, s;\n\t.reg .f32 x, y, z, w;\n\t.reg .b16 lo, hi;\n\t"
        "mov.b64 p, {%1, %2};\n\tmov.b64 q, {%3, %4};\n\tmov.b64 s, {%5, %5};\n\t"
        "mul.rn.f32x2 p, p, s;\n\tmul.rn.f32x2 q, q, s;\n\t"
        "mov.b64 {x, y}, p;\n\tmov.b64 {z, w}, q;\n\t"
        "cvt.rn.satfinite.e4m3x2.f32 lo, y, x;\n\tcvt.rn.satfinite.e4m3x2.f32 hi, w, z;\n\t"
        "mov.b32 %0, {lo, hi};\n\t}"
        : "=r"(codes) : "f"(a), "f"(b), "f"(c), "f"(d), "f"(inv));
    return codes;
}
__device__ __forceinline__ uint2 codes8(const float (&v)[8], float inv)
{
    return make_uint2(codes4(v[0], v[1], v[2], v[3], inv), codes4(v[4], v[5], v[6], v[7], inv));
}
// Largest of a value over kLanes neighbouring lanes.
template <int kLanes>
__device__ __forceinline__ uint32_t max_over(uint32_t v)
{
#pragma unroll
    for (int d = kLanes / 2; d; d >>= 1) v = max(v, __shfl_xor_sync(0xffffffffu, v, d));
    return v;
}

// Two fp32 values in a register pair, on which one instruction works.
__device__ __forceinline__ uint64_t pair_of(float a, float b)
{
    uint64_t v;
    asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(a), "f"(b));
    return v;
}
__device__ __forceinline__ uint64_t pair_of(uint32_t a, uint32_t b)
{
    uint64_t v;
    asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "r"(a), "r"(b));
    return v;
}
__device__ __forceinline__ void halves(uint64_t v, float &a, float &b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c)
{
    uint64_t d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b)
{
    uint64_t d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}

// Eight consecutive values as they lie in memory.
template <typename T> struct Raw8;
template <> struct Raw8<__nv_bfloat16> { uint4 v; };
template <> struct Raw8<float> { uint4 v, w; };

// Bits of the largest magnitude of two bf16 values with those of two others, as fp32's.
__device__ __forceinline__ uint32_t max_pairs(uint32_t m, uint32_t w) { return __vmaxu2(m, w & 0x7fff7fffu); }
__device__ __forceinline__ uint32_t max_of_pair(uint32_t m) { return max(m << 16, m & 0xffff0000u); }
// Bits of the largest magnitude of eight values.
__device__ __forceinline__ uint32_t max8(const Raw8<__nv_bfloat16> &r)
{
    return max_of_pair(max_pairs(max_pairs(max_pairs(r.v.x & 0x7fff7fffu, r.v.y), r.v.z), r.v.w));
}
__device__ __forceinline__ uint32_t max8(const Raw8<float> &r)
{
    const uint32_t k = 0x7fffffffu;
    return max(max(max(r.v.x & k, r.v.y & k), max(r.v.z & k, r.v.w & k)), max(max(r.w.x & k, r.w.y & k), max(r.w.z & k, r.w.w & k)));
}
__device__ __forceinline__ void zero8(Raw8<__nv_bfloat16> &r) { r.v = make_uint4(0, 0, 0, 0); }
__device__ __forceinline__ void zero8(Raw8<float> &r) { r.v = r.w = make_uint4(0, 0, 0, 0); }
__device__ __forceinline__ void load8(Raw8<__nv_bfloat16> &r, const __nv_bfloat16 *p) { r.v = *reinterpret_cast<const uint4 *>(p); }
__device__ __forceinline__ void load8(Raw8<float> &r, const float *p)
{
    r.v = reinterpret_cast<const uint4 *>(p)[0];
    r.w = reinterpret_cast<const uint4 *>(p)[1];
}
// The first `count` (fewer than eight, or all at an address that is not aligned), zeros after them.
__device__ __forceinline__ void load8(Raw8<__nv_bfloat16> &r, const __nv_bfloat16 *p, int count)
{
    const unsigned short *q = reinterpret_cast<const unsigned short *>(p);
    uint32_t h[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) h[i] = i < count ? q[i] : 0u;
    r.v = make_uint4(h[0] | h[1] << 16, h[2] | h[3] << 16, h[4] | h[5] << 16, h[6] | h[7] << 16);
}
__device__ __forceinline__ void load8(Raw8<float> &r, const float *p, int count)
{
    uint32_t h[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) h[i] = i < count ? __float_as_uint(p[i]) : 0u;
    r.v = make_uint4(h[0], h[1], h[2], h[3]);
    r.w = make_uint4(h[4], h[5], h[6], h[7]);
}
__device__ __forceinline__ void values8(const Raw8<__nv_bfloat16> &r, float (&f)[8])
{
    const uint32_t w[4] = {r.v.x, r.v.y, r.v.z, r.v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { f[2 * i] = __uint_as_float(w[i] << 16); f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
}
__device__ __forceinline__ void values8(const Raw8<float> &r, float (&f)[8])
{
    const uint32_t w[8] = {r.v.x, r.v.y, r.v.z, r.v.w, r.w.x, r.w.y, r.w.z, r.w.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = __uint_as_float(w[i]);
}
__device__ __forceinline__ uint32_t pack_bf16(float a, float b)
{
    const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&v);
}
__device__ __forceinline__ void store8(__nv_bfloat16 *p, const float (&f)[8])
{
    *reinterpret_cast<uint4 *>(p) = make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
}
__device__ __forceinline__ void store8(float *p, const float (&f)[8])
{
    reinterpret_cast<float4 *>(p)[0] = make_float4(f[0], f[1], f[2], f[3]);
    reinterpret_cast<float4 *>(p)[1] = make_float4(f[4], f[5], f[6], f[7]);
}
__device__ __forceinline__ void store1(__nv_bfloat16 *p, float f) { *p = __float2bfloat16_rn(f); }
__device__ __forceinline__ void store1(float *p, float f) { *p = f; }
__device__ __forceinline__ float load1(const __nv_bfloat16 *p) { return __uint_as_float((uint32_t) * reinterpret_cast<const unsigned short *>(p) << 16); }
__device__ __forceinline__ float load1(const float *p) { return *p; }

}  // namespace blk
