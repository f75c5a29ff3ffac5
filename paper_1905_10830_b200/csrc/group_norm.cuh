// What the kernels of the group norm and of its gradient share: values as pairs of fp32, the way threads are laid over pixels and channels,
// sums over a group's channels and a block's pixels.
//
// Maps have their channels as neighbours in memory.  A block works on a run of a map's pixels with all their channels, contiguous in memory.
// Its threads are laid as `rows` x `lanes`: a lane holds V neighbouring channels (16 bytes, or a single value where rows do not begin
// at 16 bytes), a row every rows-th pixel, so that a thread's weights stay in registers.  More channels than threads are worked through in
// column blocks.
#pragma once

#include "block_codes.cuh"
#include "tc_internal.h"

namespace groups {

using namespace tcdev;
using namespace blk;

enum { kNoAct = 0, kRelu = 1, kSilu = 2 };

struct GroupArgs {
    const void *x, *dy;
    const float *weight, *bias;       // null: 1 and 0
    void *out;                        // y, or dx
    RowMatrix codes;                  // forward: codes by pixels, or none
    float2 *stats;                    // [n][groups] mean, 1 / deviation; forward: written, may be null
    float eps;
    long long n;
    int c, hw, groups;
    int share, shares;                // pixels of a block, blocks of a map
    float2 *part, *runs;              // what blocks leave for the next kernel
    float2 *sums;                     // [n][groups], by that kernel
    float *dweight, *dbias;
    unsigned int *status;
};

// V values as pairs (one value: a pair with a zero).
template <int V> constexpr int kPairs = (V + 1) / 2;
template <int V> using Pairs = uint64_t[kPairs<V>];

template <int V>
__device__ __forceinline__ void load_pairs(const __nv_bfloat16 *p, Pairs<V> &v)
{
    if constexpr (V == 8) {
        const uint4 r = *reinterpret_cast<const uint4 *>(p);
        const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = pair_of(w[i] << 16, w[i] & 0xffff0000u);
    } else
        v[0] = pair_of(load1(p), 0.f);
}
template <int V>
__device__ __forceinline__ void load_pairs(const float *p, Pairs<V> &v)
{
    if constexpr (V == 4) {
        const uint4 r = *reinterpret_cast<const uint4 *>(p);
        v[0] = pair_of(r.x, r.y);
        v[1] = pair_of(r.z, r.w);
    } else
        v[0] = pair_of(*p, 0.f);
}
template <int V, typename T>
__device__ __forceinline__ void store_pairs(T *p, const Pairs<V> &v)
{
    float f[2 * kPairs<V>];
#pragma unroll
    for (int i = 0; i < kPairs<V>; ++i) halves(v[i], f[2 * i], f[2 * i + 1]);
    if constexpr (V == 8) *reinterpret_cast<uint4 *>(p) = make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
    else if constexpr (V == 4) *reinterpret_cast<float4 *>(p) = make_float4(f[0], f[1], f[2], f[3]);
    else store1(p, f[0]);
}
// A vector's values from channel c on, `other` without the vector.
template <int V>
__device__ __forceinline__ void vector_pairs(const float *p, int c, float other, Pairs<V> &v)
{
    float f[2 * kPairs<V>] = {};
#pragma unroll
    for (int i = 0; i < V; ++i) f[i] = p ? p[c + i] : other;
#pragma unroll
    for (int i = 0; i < kPairs<V>; ++i) v[i] = pair_of(f[2 * i], f[2 * i + 1]);
}
// Means (negated) and 1 / deviations of V channels' groups.
template <int V>
__device__ __forceinline__ void stats_pairs(const float2 *stats, int c, int per_group, Pairs<V> &minus_mean, Pairs<V> &rstd)
{
    float m[2 * kPairs<V>] = {}, r[2 * kPairs<V>] = {};
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const float2 s = stats[(c + i) / per_group];
        m[i] = -s.x;
        r[i] = s.y;
    }
#pragma unroll
    for (int i = 0; i < kPairs<V>; ++i) {
        minus_mean[i] = pair_of(m[2 * i], m[2 * i + 1]);
        rstd[i] = pair_of(r[2 * i], r[2 * i + 1]);
    }
}
__device__ __forceinline__ uint64_t both(float v) { return pair_of(v, v); }

// 1 / (1 + e^-z): an fp32 exponential and quotient of a few roundings each; 0 where e^-z is beyond fp32.
__device__ __forceinline__ float sigmoid(float z) { return __fdividef(1.0f, 1.0f + __expf(-z)); }
template <int kAct>
__device__ __forceinline__ float activate(float z)
{
    return kAct == kRelu ? (z < 0.f ? 0.f : z) : kAct == kSilu ? z * sigmoid(z) : z;
}
template <int kAct>
__device__ __forceinline__ uint64_t activate2(uint64_t z)
{
    if constexpr (kAct == kNoAct) return z;
    float a, b;
    halves(z, a, b);
    return pair_of(activate<kAct>(a), activate<kAct>(b));
}
// The activation's derivative at z, times d.
template <int kAct>
__device__ __forceinline__ uint64_t slope2(uint64_t z, uint64_t d)
{
    if constexpr (kAct == kNoAct) return d;
    float a, b;
    halves(z, a, b);
    if constexpr (kAct == kRelu) {
        float x, y;
        halves(d, x, y);
        return pair_of(a > 0.f ? x : 0.f, b > 0.f ? y : 0.f);
    } else {
        const uint64_t s = pair_of(sigmoid(a), sigmoid(b));
        // s + z s (1 - s)
        const uint64_t t = fma2(mul2(z, s), add2(both(1.0f), s ^ 0x8000000080000000ull), s);
        return mul2(t, d);
    }
}

// A block's threads over `columns` lanes of channels.
struct Lay {
    int columns, lanes, rows, lane, row, blocks;
    __device__ __forceinline__ explicit Lay(int columns_)
    {
        const int threads = blockDim.x;
        columns = columns_;
        blocks = (columns + threads - 1) / threads;
        lanes = (columns + blocks - 1) / blocks;
        rows = threads / lanes;
        row = threadIdx.x / lanes;
        lane = threadIdx.x - row * lanes;
    }
    __device__ __forceinline__ bool at(int block) const { return row < rows && block * lanes + lane < columns; }
};

// Sums of runs of a group's entries, by as many neighbouring lanes as they are worth.
struct Team {
    int size, rank, first, step;      // lanes of a group; this thread's; its first group, and how many groups the block works on at a time
    __device__ __forceinline__ explicit Team(int entries)
    {
        size = 1;
        while (size < 32 && size * 4 < entries) size *= 2;
        rank = threadIdx.x & (size - 1);
        first = threadIdx.x / size;
        step = blockDim.x / size;
    }
    __device__ __forceinline__ float sum(float v) const
    {
        for (int d = size / 2; d; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
        return v;
    }
};

// Adds, for each group, what the threads hold for its channels in column block `block`: to(group, total), by one thread, blocks in their order.
// `red`: blockDim x V floats of shared memory.
template <int V, typename F>
__device__ __forceinline__ void add_groups(const Lay &lay, int block, int per_group, int group_count, const Pairs<V> &v, float *red, F to)
{
    const bool whole = V > 1 && per_group % V == 0;           // a thread's channels are of one group
    const int per_lane = whole ? 1 : V, pitch = lay.lanes * per_lane;
    __syncthreads();                                          // the readers of the last sums
    if (lay.at(block)) {
        float f[2 * kPairs<V>];
#pragma unroll
        for (int i = 0; i < kPairs<V>; ++i) halves(v[i], f[2 * i], f[2 * i + 1]);
        float *const at = red + lay.row * pitch + lay.lane * per_lane;
        if (whole) {
            float s = f[0];
#pragma unroll
            for (int i = 1; i < V; ++i) s += f[i];
            at[0] = s;
        } else
#pragma unroll
            for (int i = 0; i < V; ++i) at[i] = f[i];
    }
    __syncthreads();
    const int per = whole ? per_group / V : per_group;        // entries of a group in a row
    const int c0 = block * pitch, c1 = min(c0 + pitch, whole ? lay.columns : lay.columns * V);
    const int g0 = c0 / per, g1 = min(group_count, (c1 + per - 1) / per);
    const Team team(lay.rows * per);
    for (int base = g0; base < g1; base += team.step) {       // (all threads go round together: the sums are taken by whole warps)
        const int g = base + team.first;
        float s = 0.f;
        if (g < g1) {
            const int from = max(g * per, c0) - c0, count = min((g + 1) * per, c1) - c0 - from;
            if (count == 1) for (int r = team.rank; r < lay.rows; r += team.size) s += red[r * pitch + from];
            else
                for (int i = team.rank; i < lay.rows * count; i += team.size) {
                    const int r = i / count;
                    s += red[r * pitch + from + i - r * count];
                }
        }
        s = team.sum(s);
        if (g < g1 && team.rank == 0) to(g, s);
    }
}

}  // namespace groups
