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
    uint16_t lo, hi;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(__fmul_rn(b, inv)), "f"(__fmul_rn(a, inv)));
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(__fmul_rn(d, inv)), "f"(__fmul_rn(c, inv)));
    return (uint32_t)lo | (uint32_t)hi << 16;
}
__device__ __forceinline__ uint2 codes8(const float (&v)[8], float inv)
{
    return make_uint2(codes4(v[0], v[1], v[2], v[3], inv), codes4(v[4], v[5], v[6], v[7], inv));
}
// Largest of a value over the 16 lanes of a half warp.
__device__ __forceinline__ uint32_t max16(uint32_t v)
{
#pragma unroll
    for (int d = 8; d; d >>= 1) v = max(v, __shfl_xor_sync(0xffffffffu, v, d));
    return v;
}

// Eight consecutive values as they lie in memory.
template <typename T> struct Raw8;
template <> struct Raw8<__nv_bfloat16> { uint4 v; };
template <> struct Raw8<float> { uint4 v, w; };

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
template <typename T>
__device__ __forceinline__ void store8(T *p, const float (&f)[8], int count)
{
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < count) store1(p + i, f[i]);
}

}  // namespace blk
