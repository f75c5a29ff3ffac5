// What the kernels of the group norm and of its gradient share: values as pairs of fp32, the way threads are laid over pixels and channels,
// sums over a group's channels and a block's pixels.
//
// Maps have their channels as neighbours in memory.  A block works on a run of a map's pixels with all their channels, contiguous in memory.
// Its threads are laid as `rows` x `lanes`: a lane holds V neighbouring channels (16 bytes, or two values or one where rows do not begin
// at 16 bytes), a row every rows-th pixel, so that a thread's weights stay in registers.  More channels than threads are worked through in
// column blocks.
#pragma once

#include "block_codes.cuh"
#include "sm100_ptx.cuh"
#include "tc_internal.h"

namespace groups {

using namespace tcdev;
using namespace blk;

constexpr int kRunThreads = 256;                               // that work on a run of pixels; a ring has a warp more

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

// V values as they lie in memory, and as pairs (one value: a pair with a zero).  Loops load some vectors before they work on the first: a store between two loads
// would keep the second back, for all the compiler knows of what overlaps.
template <int V> constexpr int kPairs = (V + 1) / 2;
template <int V> using Pairs = uint64_t[kPairs<V>];
template <typename T, int V> struct Raw { uint4 v; };
template <> struct Raw<__nv_bfloat16, 2> { uint32_t v; };
template <> struct Raw<float, 2> { float2 v; };
template <typename T> struct Raw<T, 1> { float v; };

template <int V, typename T>
__device__ __forceinline__ void load_raw(Raw<T, V> &r, const T *p)
{
    if constexpr (V > 1) r.v = *reinterpret_cast<const decltype(r.v) *>(p);
    else r.v = load1(p);
}
template <int V, typename T>
__device__ __forceinline__ void pairs_of(const Raw<T, V> &r, Pairs<V> &v)
{
    if constexpr (V == 8) {
        const uint32_t w[4] = {r.v.x, r.v.y, r.v.z, r.v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = pair_of(w[i] << 16, w[i] & 0xffff0000u);
    } else if constexpr (V == 4) {
        v[0] = pair_of(r.v.x, r.v.y);
        v[1] = pair_of(r.v.z, r.v.w);
    } else if constexpr (V == 2 && sizeof(T) == 2)
        v[0] = pair_of(r.v << 16, r.v & 0xffff0000u);
    else if constexpr (V == 2)
        v[0] = pair_of(r.v.x, r.v.y);
    else
        v[0] = pair_of(r.v, 0.f);
}
template <int V, typename T>
__device__ __forceinline__ void load_pairs(const T *p, Pairs<V> &v)
{
    Raw<T, V> r;
    load_raw<V>(r, p);
    pairs_of<V>(r, v);
}
// load(place, i) and then work(place, i, i2) for pairs of the pixels i and i2 of a thread, from `first` on in steps of `rows`, kBatch (even) loaded at a time; an odd last one comes
// with i2 = -1, and the place behind it has the same pixel.
template <int kBatch, typename L, typename W>
__device__ __forceinline__ void in_batches(int first, int end, int rows, L load, W work)
{
    int i = first;
    for (; i + (kBatch - 1) * rows < end; i += kBatch * rows) {
#pragma unroll
        for (int k = 0; k < kBatch; ++k) load(k, i + k * rows);
#pragma unroll
        for (int k = 0; k < kBatch; k += 2) work(k, i + k * rows, i + (k + 1) * rows);
    }
    if (i >= end) return;
    int at[kBatch];
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
        at[k] = k == 0 || i + k * rows < end ? i + k * rows : at[k ? k - 1 : 0];
        load(k, at[k]);
    }
#pragma unroll
    for (int k = 0; k < kBatch; k += 2)
        if (k == 0 || at[k] != at[k ? k - 1 : 0]) work(k, at[k], at[k + 1] != at[k] ? at[k + 1] : -1);
}
// Vectors that a thread asks for before it works on the first, of V values from global memory.
template <int V> constexpr int kAhead = V <= 2 ? 8 : 4;
template <int V, typename T>
__device__ __forceinline__ void store_pairs(T *p, const Pairs<V> &v)
{
    float f[2 * kPairs<V>];
#pragma unroll
    for (int i = 0; i < kPairs<V>; ++i) halves(v[i], f[2 * i], f[2 * i + 1]);
    if constexpr (V == 8) *reinterpret_cast<uint4 *>(p) = make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
    else if constexpr (V == 4) *reinterpret_cast<float4 *>(p) = make_float4(f[0], f[1], f[2], f[3]);
    else if constexpr (V == 2 && sizeof(T) == 2) *reinterpret_cast<uint32_t *>(p) = pack_bf16(f[0], f[1]);
    else if constexpr (V == 2) *reinterpret_cast<float2 *>(p) = make_float2(f[0], f[1]);
    else store1(p, f[0]);
}
// A vector's values from channel c on, `other` without the vector.
template <int V>
__device__ __forceinline__ void vector_pairs(const float *p, int c, float other, Pairs<V> &v)
{
    if constexpr (V % 4 == 0) {
        if (p && ((uintptr_t)p & 15u) == 0) {
#pragma unroll
            for (int i = 0; i < V; i += 4) {
                const float4 f = *reinterpret_cast<const float4 *>(p + c + i);
                v[i / 2] = pair_of(f.x, f.y);
                v[i / 2 + 1] = pair_of(f.z, f.w);
            }
            return;
        }
    }
    float f[2 * kPairs<V>] = {};
#pragma unroll
    for (int i = 0; i < V; ++i) f[i] = p ? p[c + i] : other;
#pragma unroll
    for (int i = 0; i < kPairs<V>; ++i) v[i] = pair_of(f[2 * i], f[2 * i + 1]);
}
// First (negated) and second value of V channels' groups: of(group).
template <int V, typename F>
__device__ __forceinline__ void stats_pairs(int c, int per_group, Pairs<V> &minus, Pairs<V> &second, F of)
{
    int g = c / per_group, rest = c - g * per_group;
    float2 s = of(g);
    if (rest + V <= per_group) {
#pragma unroll
        for (int i = 0; i < kPairs<V>; ++i) {
            minus[i] = pair_of(-s.x, -s.x);
            second[i] = pair_of(s.y, s.y);
        }
        return;
    }
    float m[2 * kPairs<V>] = {}, r[2 * kPairs<V>] = {};
#pragma unroll
    for (int i = 0; i < V; ++i) {
        if (i && ++rest == per_group) {
            rest = 0;
            s = of(++g);
        }
        m[i] = -s.x;
        r[i] = s.y;
    }
#pragma unroll
    for (int i = 0; i < kPairs<V>; ++i) {
        minus[i] = pair_of(m[2 * i], m[2 * i + 1]);
        second[i] = pair_of(r[2 * i], r[2 * i + 1]);
    }
}
constexpr uint64_t kMinus = 0x8000000080000000ull;             // a pair's signs
__device__ __forceinline__ uint64_t both(float v) { return pair_of(v, v); }

__device__ __forceinline__ float max_nan(float a, float b)    // (a NaN stays one)
{
    float d;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
    return d;
}
// s = 1 / (1 + e^-z) of two pixels' pairs a and b, and rest = e^-z s = 1 - s (the difference would lose the digits that a large z needs).  Each value's two reciprocals come from one of
// their product: the functions' unit takes three operations for two values instead of four.  The two are of one channel, so a NaN stays in its group.  z is taken as -43.5 at
// least, where s is 1.3e-19: two denominators' product is 6.1e37 at most, whose reciprocal is a normal number still.  The fast exponential and reciprocal, a few
// steps of 2^-23 each.
__device__ __forceinline__ float exp2_fast(float v)
{
    float e;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(v));
    return e;
}
__device__ __forceinline__ float reciprocal_fast(float v)
{
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}
__device__ __forceinline__ uint64_t at_least(uint64_t z, float least)
{
    float x, y;
    halves(z, x, y);
    return pair_of(max_nan(x, least), max_nan(y, least));
}
__device__ __forceinline__ uint64_t exp_minus(uint64_t z)
{
    float x, y;
    halves(mul2(z, both(-1.4426950408889634f)), x, y);
    return pair_of(exp2_fast(x), exp2_fast(y));
}
__device__ __forceinline__ void sigmoids(uint64_t &za, uint64_t &zb, uint64_t &sa, uint64_t &sb, uint64_t &rest_a, uint64_t &rest_b)
{
    za = at_least(za, -43.5f);
    zb = at_least(zb, -43.5f);
    const uint64_t ea = exp_minus(za), eb = exp_minus(zb), da = add2(ea, both(1.0f)), db = add2(eb, both(1.0f));
    float x, y;
    halves(mul2(da, db), x, y);
    const uint64_t r = pair_of(reciprocal_fast(x), reciprocal_fast(y));
    sa = mul2(r, db);
    sb = mul2(r, da);
    rest_a = mul2(ea, sa);
    rest_b = mul2(eb, sb);
}
// The activation.  (Each value's reciprocal its own: memory bounds the forward pass, and a value's bits do not depend on its neighbour.)
template <int kAct>
__device__ __forceinline__ uint64_t activate2(uint64_t z)
{
    if constexpr (kAct == kNoAct) return z;
    if constexpr (kAct == kRelu) return at_least(z, 0.f);
    float x, y;
    halves(add2(exp_minus(z), both(1.0f)), x, y);             // (e^-z beyond 2^126: 0)
    return mul2(z, pair_of(reciprocal_fast(x), reciprocal_fast(y)));
}
// Its derivatives at za and zb, times da and db.
template <int kAct>
__device__ __forceinline__ void slope2(uint64_t za, uint64_t zb, uint64_t &da, uint64_t &db)
{
    if constexpr (kAct == kRelu) {
        auto one = [](uint64_t z, uint64_t &d) {
            float a, b, x, y;
            halves(z, a, b);
            halves(d, x, y);
            d = pair_of(a > 0.f ? x : 0.f, b > 0.f ? y : 0.f);
        };
        one(za, da);
        one(zb, db);
    } else if constexpr (kAct == kSilu) {
        uint64_t sa, sb, rest_a, rest_b;
        sigmoids(za, zb, sa, sb, rest_a, rest_b);
        // s (1 + z (1 - s))
        const uint64_t one = both(1.0f);
        da = mul2(da, mul2(sa, fma2(za, rest_a, one)));
        db = mul2(db, mul2(sb, fma2(zb, rest_b, one)));
    }
}

// Moments or totals of group `g` that the blocks of a cluster left at `mine` in their shared memory, asked for all at once (one after the other they cost
// a microsecond for each two blocks).
constexpr int kMostShares = 16;
__device__ __forceinline__ void of_cluster(const float2 *mine, int shares, float2 (&m)[kMostShares])
{
#pragma unroll
    for (int i = 0; i < kMostShares; ++i)
        if (i < shares)
            asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(m[i].x), "=f"(m[i].y) : "r"(peer_address(mine, (uint32_t)i)));
}

// A block's first `threads` threads over `columns` lanes of channels.
struct Lay {
    int threads, columns, lanes, rows, lane, row, blocks;
    __device__ __forceinline__ explicit Lay(int columns_, int threads_)
    {
        threads = threads_;
        columns = columns_;
        blocks = (columns + threads - 1) / threads;
        lanes = (columns + blocks - 1) / blocks;
        rows = threads / lanes;
        row = threadIdx.x / lanes;
        lane = threadIdx.x - row * lanes;
    }
    __device__ __forceinline__ bool at(int block) const { return row < rows && block * lanes + lane < columns; }
    __device__ __forceinline__ void sync() const { sm100::named_bar_sync(1, threads); }
};

// A block's pixels, a piece after the other: piece i has the pixels first(i) to end(i), the first of which lies `at(i)` pixels behind the source's address once wait(i) is over, until
// done(i), both by whole warps.  (A wait that runs out is reported; the values are wrong then, nothing else.)
// All of them are where they are:
struct InPlace {
    int pixels;
    __device__ __forceinline__ int count() const { return 1; }
    __device__ __forceinline__ int first(int) const { return 0; }
    __device__ __forceinline__ int end(int) const { return pixels; }
    __device__ __forceinline__ int at(int) const { return 0; }
    __device__ __forceinline__ void wait(int) {}
    __device__ __forceinline__ void done(int) {}
};
__device__ __forceinline__ bool arrived(unsigned long long *barrier, uint32_t parity)
{
    const uint32_t bar = sm100::smem_u32(barrier);
    return sm100::mbar_try_wait(bar, parity, 1000u) || sm100::mbar_wait_soon(bar, parity) || sm100::mbar_wait_soon(bar, parity);
}
// On their way to shared memory, so that the first can be worked on while the others come: pieces of whole rounds of the block's rows.
constexpr int kPieces = 4;
struct Pieces {
    int pixels, each;
    unsigned long long *full;
    unsigned int *status;
    __device__ __forceinline__ Pieces(int pixels_, int rows, unsigned long long *full_, unsigned int *status_)
    {
        pixels = pixels_;
        each = ((pixels + kPieces - 1) / kPieces + rows - 1) / rows * rows;
        full = full_;
        status = status_;
    }
    __device__ __forceinline__ int first(int piece) const { return min(piece * each, pixels); }
    __device__ __forceinline__ int end(int piece) const { return min((piece + 1) * each, pixels); }
    __device__ __forceinline__ int at(int piece) const { return first(piece); }
    __device__ __forceinline__ int count() const { return kPieces; }
    __device__ __forceinline__ void wait(int piece) const
    {
        if (first(piece) != end(piece) && !arrived(&full[piece], 0)) tc_dev_set_status(status, TC_ERR_TIMEOUT);
    }
    __device__ __forceinline__ void done(int) const {}
};
// Of a run that is longer than its block's shared memory: pieces of kRounds rounds of the rows through a ring of kSlots, that a warp of its own fills by bulk copies.  Loads of the threads
// keep too little on its way (gradient of silu, 128x56x56 x 128 bf16: 144 us, ring 116; 256x56x56 x 128 forward 116 and 105).  Few long pieces: more and shorter ones, of the
// same bytes, cost more waits than their earlier refills are worth (123 and 107).
template <int kSlots_, int kRounds, int kTensors>
struct Ring {
    static constexpr int kSlots = kSlots_, kRows = kTensors * kSlots * kRounds;
    int pixels, each;                 // of the run; of a piece
    unsigned long long *full, *empty;
    unsigned int *status;
    bool lost;
    __device__ __forceinline__ Ring(int pixels_, int rows, unsigned long long *barriers, unsigned int *status_)
    {
        pixels = pixels_;
        each = kRounds * rows;
        full = barriers;
        empty = barriers + kSlots;
        status = status_;
        lost = false;
    }
    __device__ __forceinline__ int count() const { return (pixels + each - 1) / each; }
    __device__ __forceinline__ int first(int piece) const { return piece * each; }
    __device__ __forceinline__ int end(int piece) const { return min((piece + 1) * each, pixels); }
    __device__ __forceinline__ int at(int piece) const { return piece % kSlots * each; }
    __device__ __forceinline__ void wait(int piece)
    {
        if (lost || arrived(&full[piece % kSlots], piece / kSlots & 1)) return;
        lost = true;
        tc_dev_set_status(status, TC_ERR_TIMEOUT);
    }
    __device__ __forceinline__ void done(int piece) const
    {
        __syncwarp();
        if ((threadIdx.x & 31) == 0) sm100::mbar_arrive(sm100::smem_u32(&empty[piece % kSlots]));
    }
    __device__ __forceinline__ static void init(unsigned long long *barriers)
    {
        for (int i = 0; i < 2 * kSlots; ++i) sm100::mbar_init(sm100::smem_u32(&barriers[i]), i < kSlots ? 1 : kRunThreads / 32);
        sm100::mbar_fence_init();
    }
    // By one thread: the run's pixels of `row` bytes from each of the tensors, to rings that follow one another.
    __device__ __forceinline__ void fill(unsigned char *ring, const void *x, const void *dy, int row) const
    {
        const int pieces = count(), room = each * row;
        int i = 0;
        for (; i < pieces; ++i) {
            const int slot = i % kSlots;
            if (i >= kSlots && !arrived(&empty[slot], (i / kSlots + 1) & 1)) {
                tc_dev_set_status(status, TC_ERR_TIMEOUT);
                break;
            }
            const uint32_t bytes = (uint32_t)(end(i) - first(i)) * row, bar = sm100::smem_u32(&full[slot]), to = sm100::smem_u32(ring) + slot * room;
            const size_t from = (size_t)first(i) * row;
            sm100::mbar_arrive_expect_tx(bar, kTensors * bytes);
            sm100::bulk_load(to, (const char *)x + from, bytes, bar);
            if (kTensors > 1) sm100::bulk_load(to + kSlots * room, (const char *)dy + from, bytes, bar);
        }
        // The copies in flight land before the block's shared memory goes to another, whoever's wait ran out.
        for (int last = max(i - kSlots, 0); last < i; ++last) arrived(&full[last % kSlots], last / kSlots & 1);
    }
};
// A ring's bytes.  (Rows of a block: as Lay's.)
template <typename R>
size_t ring_bytes(int columns) { return (size_t)R::kRows * (kRunThreads / columns) * columns * 16; }
// Rings are for rows whose vectors have a thread each.
inline bool ring_takes(int c, int v, int element) { return v * element == 16 && c / v <= kRunThreads; }
// Neighbouring channels that a lane holds: of 16 bytes, else two, else one.
inline int vector_of(int c, int element, bool aligned) { return !aligned ? 1 : c * element % 16 == 0 ? 16 / element : c % 2 == 0 ? 2 : 1; }

// The run of pixels that a block works on.
struct Run {
    unsigned int index;               // of all maps' runs
    long long map;
    int run, pixels;
    long long first;                  // pixel of the tensor
    __device__ __forceinline__ Run(const GroupArgs &a, unsigned int index_)
    {
        index = index_;
        const unsigned int m = index / (unsigned int)a.shares;
        run = (int)(index - m * (unsigned int)a.shares);
        map = m;
        pixels = min(a.share, a.hw - run * a.share);
        first = map * a.hw + run * a.share;
    }
};

// What a kernel on runs does: work(x, dy, pieces) on its block's run, by the threads up to kRunThreads.  With a ring a block has a warp more, and the ring lies first in shared memory, x's
// and then dy's.
template <typename T, typename R, bool kRing, typename F>
__device__ __forceinline__ void with_run(const GroupArgs &a, const Run &run, const Lay &lay, unsigned char *smem, int ring_size, F work)
{
    const T *const x = (const T *)a.x + run.first * a.c, *const dy = a.dy ? (const T *)a.dy + run.first * a.c : nullptr;
    if constexpr (kRing) {
        __shared__ __align__(8) unsigned long long s_ring[2 * R::kSlots];
        if (threadIdx.x == 0) R::init(s_ring);
        __syncthreads();
        chain_next();
        chain_wait();
        R ring(run.pixels, lay.rows, s_ring, a.status);
        if (threadIdx.x < kRunThreads) work(reinterpret_cast<const T *>(smem), reinterpret_cast<const T *>(smem + ring_size / 2), ring);
        else if (threadIdx.x == kRunThreads) ring.fill(smem, x, dy, a.c * (int)sizeof(T));
    } else {
        chain_next();
        chain_wait();
        InPlace pieces{run.pixels};
        work(x, dy, pieces);
    }
}

// Room that channel_sums takes: of the lower half of the rows.
__host__ __device__ inline int red_values(int columns, int threads, int v)
{
    const int blocks = (columns + threads - 1) / threads, lanes = (columns + blocks - 1) / blocks, rows = threads / lanes;
    return ((rows + 1) / 2 * lanes * v + 1) / 2 * 2;
}

// Sums of runs of a group's entries, by as many neighbouring lanes as they are worth.
struct Team {
    int size, rank, first, step;      // lanes of a group; this thread's; its first group, and how many groups the block works on at a time
    __device__ __forceinline__ Team(int entries, int threads)
    {
        size = 1;
        while (size < 32 && size * 4 < entries) size *= 2;
        rank = threadIdx.x & (size - 1);
        first = threadIdx.x / size;
        step = threads / size;
    }
    __device__ __forceinline__ float sum(float v) const
    {
        for (int d = size / 2; d; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
        return v;
    }
};

// Sums over the block's rows of what its threads hold for V channels each (a[i], b[i]); each(channel, a, b) by one thread for each of column block `block`, by
// neighbouring threads for neighbouring channels, whole warps together (channel -1: none).  red: red_values() float2.
template <int V, typename F>
__device__ __forceinline__ void channel_sums(const Lay &lay, int block, const float (&a)[2 * kPairs<V>], const float (&b)[2 * kPairs<V>], float2 *red, F each)
{
    // the upper half of the rows leaves its values, the lower half adds its own
    constexpr int kPer = V > 1 ? V / 2 : 1;
    const int half = (lay.rows + 1) / 2, lanes = lay.lanes;
    const bool here = lay.at(block);
    lay.sync();                                               // the last sums' readers
    float4 *const at = reinterpret_cast<float4 *>(red) + (lay.row >= half ? lay.row - half : lay.row) * kPer * lanes + lay.lane;
    float2 *const at1 = red + (lay.row >= half ? lay.row - half : lay.row) * lanes + lay.lane;
    if (here && lay.row >= half) {
        if constexpr (V > 1)
#pragma unroll
            for (int i = 0; i < kPer; ++i) at[i * lanes] = make_float4(a[2 * i], b[2 * i], a[2 * i + 1], b[2 * i + 1]);
        else *at1 = make_float2(a[0], b[0]);
    }
    lay.sync();
    if (here && lay.row < half) {
        const bool two = lay.row + half < lay.rows;
        if constexpr (V > 1) {
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                const float4 t = two ? at[i * lanes] : make_float4(0.f, 0.f, 0.f, 0.f);
                at[i * lanes] = make_float4(a[2 * i] + t.x, b[2 * i] + t.y, a[2 * i + 1] + t.z, b[2 * i + 1] + t.w);
            }
        } else {
            const float2 t = two ? *at1 : make_float2(0.f, 0.f);
            *at1 = make_float2(a[0] + t.x, b[0] + t.y);
        }
    }
    lay.sync();
    const int first = block * lanes, channels = min(lanes, lay.columns - first) * V;
    for (int base = 0; base < channels; base += lay.threads) {
        const int j = base + threadIdx.x;
        float2 s = make_float2(0.f, 0.f);
        if (j < channels) {
            const float2 *from = red + (V > 1 ? 2 * (((j % V) / 2) * lanes + j / V) + (j & 1) : j);
            const int pitch = V * lanes;
#pragma unroll 4
            for (int r = 0; r < half; ++r) {
                const float2 t = from[r * pitch];
                s.x += t.x;
                s.y += t.y;
            }
        }
        each(j < channels ? first * V + j : -1, s.x, s.y);
    }
}
// Where a block's channels have a thread each and a group's are a power of two that a warp holds, sums over groups need no shared memory.
__device__ __forceinline__ bool groups_in_warps(const Lay &lay, int per_group) { return lay.blocks == 1 && per_group <= 32 && (per_group & (per_group - 1)) == 0; }
__device__ __forceinline__ float sum_over(float v, int lanes)
{
    for (int d = lanes / 2; d; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    return v;
}

}  // namespace groups

// Clusters of `shares` blocks that run at a time with a block an SM.  Clusters lie within a GPC, and one of the GPCs has fewer than 16 SMs: eight clusters of 16 blocks, or sixteen of 8, take
// two turns (gradient of 832x19x19 x 8 bf16 in clusters of 16: 26 us, of 8: 19).
inline long long clusters_at_once(int shares, int sm_count) { return shares <= 4 ? sm_count / shares : sm_count * (shares == 8 ? 14 : 7) / 148; }
// Blocks of a map where all maps lie in clusters' shared memory at one time, `per_sm` blocks an SM where two fit; 0: they do not.  As few as let two share an SM, then as few as fit one, and
// more where SMs would be idle.  More maps than find a place at a time take the other kernels: a block's phases (wait, sums, cluster, values) follow one another, and little of the
// next one's waiting falls into them.
template <typename F>
int shares_on_chip(long long n, int hw, int per_sm, int sm_count, F bytes)
{
    for (const size_t room : {kTwoBlocks, kMostShared}) {
        int shares = 1;
        while (shares < groups::kMostShares && bytes(shares) > room) shares *= 2;
        if (bytes(shares) > room || n > clusters_at_once(shares, sm_count) * (room == kTwoBlocks ? per_sm : 1)) continue;
        while (shares < groups::kMostShares && n <= clusters_at_once(2 * shares, sm_count) && hw / shares >= 12) shares *= 2;
        return shares;
    }
    return 0;
}
// Runs of pixels (of `columns` vectors, `row` bytes in each of `tensors`) of a map; ring_blocks: blocks of an SM that take them through rings, 0: none do.
void cut_runs(GroupPlan &p, long long n, int hw, int columns, long long row, int tensors, int ring_blocks, int sm_count);
