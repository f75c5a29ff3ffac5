// tc_group_norm: of maps whose channels are neighbours in memory,
//
//   y = act((x - mean) rstd w + b),   mean and rstd = 1 / sqrt(var + eps) over a map's pixels and a group's channels
//
// Bound by the bytes moved, x once and y once.  A map or two, and maps that a block holds, are read once: each of a cluster's blocks (up to sixteen)
// takes its pixels to shared memory by bulk copies, finds its moments, they are put together through the cluster's shared memory, and the values leave from where
// they lie.  Others take two kernels: moments of runs of pixels, and the values, the pixels through a ring in shared memory where their rows begin at 16 bytes.
// 256x56x56 x 128 bf16: 105 us, 5.9 TB/s with the second reading of x; one map of 256x14x14: 6.7 us.
//
// Moments are put together as (n, mean, M2): no sum of squares is taken about a mean far from its own.
#include "group_norm.cuh"
#include "integer_codes.cuh"

#include <type_traits>

namespace {

using namespace groups;
using rowcodes::Coder;

using NormRing = Ring<2, 8, 1>;                               // 64 KB
constexpr int kNormBlocks = 3;                                // an SM

// A whole run where it is, in steps: each as long as all before it.
constexpr int kStepRounds = 16;                               // of the block's rows, the first two steps
struct InSteps {
    int pixels, each;
    __device__ __forceinline__ int count() const
    {
        int n = 1;
        while (each << (n - 1) < pixels) ++n;
        return n;
    }
    __device__ __forceinline__ int first(int step) const { return step ? each << (step - 1) : 0; }
    __device__ __forceinline__ int end(int step) const { return min(each << step, pixels); }
    __device__ __forceinline__ int at(int step) const { return first(step); }
    __device__ __forceinline__ void wait(int) {}
    __device__ __forceinline__ void done(int) {}
};
__device__ __forceinline__ InSteps in_steps(InPlace &p, const Lay &lay) { return {p.pixels, kStepRounds * lay.rows}; }
template <typename P>
__device__ __forceinline__ P &in_steps(P &p, const Lay &) { return p; }

// Moments that are put together about the first one's mean: what is taken away in the end is at most so many times what stays.
constexpr int kFew = 8;

// The pixels of a block's rows.
struct RowCounts {
    int rows, rest;
    float full, per_pixel;
    __device__ __forceinline__ RowCounts(int pixels, const Lay &lay)
    {
        rows = lay.rows;
        rest = pixels % rows;
        full = (float)(pixels / rows);
        per_pixel = pixels ? reciprocal_fast((float)pixels) : 0.f;
    }
    __device__ __forceinline__ float operator()(int row) const { return row < rest ? full + 1.f : row < rows ? full : 0.f; }
};
// Mean and M2 (sum of squares about it) over the block's pixels of column block `block` from its threads' moments of V channels each, as channel_sums hands them out.
template <int V, typename F>
__device__ __forceinline__ void channel_moments(const Lay &lay, int block, const RowCounts &count, const float (&mean)[2 * kPairs<V>], const float (&m2)[2 * kPairs<V>], float2 *red, F each)
{
    constexpr int kPer = V > 1 ? V / 2 : 1;
    const int half = (lay.rows + 1) / 2, lanes = lay.lanes;
    const bool here = lay.at(block);
    const int place = lay.row >= half ? lay.row - half : lay.row;
    lay.sync();                                               // the last moments' readers
    float4 *const at = reinterpret_cast<float4 *>(red) + place * kPer * lanes + lay.lane;
    float2 *const at1 = red + place * lanes + lay.lane;
    if (here && lay.row >= half) {
        if constexpr (V > 1)
#pragma unroll
            for (int i = 0; i < kPer; ++i) at[i * lanes] = make_float4(mean[2 * i], m2[2 * i], mean[2 * i + 1], m2[2 * i + 1]);
        else *at1 = make_float2(mean[0], m2[0]);
    }
    lay.sync();
    if (here && lay.row < half) {
        // the upper half's row added to the lower half's
        const float n = count(lay.row), more = count(lay.row + half), share = more > 0.f ? more * reciprocal_fast(n + more) : 0.f, weight = n * share;
        auto joined = [&](float mean_a, float m2_a, float mean_b, float m2_b) {
            const float d = more > 0.f ? mean_b - mean_a : 0.f;
            return make_float2(fmaf(d, share, mean_a), more > 0.f ? fmaf(__fmul_rn(d, weight), d, __fadd_rn(m2_a, m2_b)) : m2_a);
        };
        if constexpr (V > 1) {
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                const float4 t = at[i * lanes];
                const float2 x = joined(mean[2 * i], m2[2 * i], t.x, t.y), y = joined(mean[2 * i + 1], m2[2 * i + 1], t.z, t.w);
                at[i * lanes] = make_float4(x.x, x.y, y.x, y.y);
            }
        } else {
            const float2 t = *at1;
            *at1 = joined(mean[0], m2[0], t.x, t.y);
        }
    }
    lay.sync();
    const int first = block * lanes, channels = min(lanes, lay.columns - first) * V;
    for (int base = 0; base < channels; base += lay.threads) {
        const int j = base + threadIdx.x;
        float about = 0.f, off = 0.f, squares = 0.f;
        if (j < channels) {
            const float2 *from = red + (V > 1 ? 2 * (((j % V) / 2) * lanes + j / V) + (j & 1) : j);
            const int pitch = V * lanes;
            // about the first row's mean, or the mean where there are more than a few: then the squares, and what the mean is off
            about = from[0].x;
            if (half > kFew) {
                about = 0.f;
#pragma unroll 4
                for (int r = 0; r < half; ++r) about = fmaf(count(r) + count(r + half), from[r * pitch].x, about);
                about = __fmul_rn(about, count.per_pixel);
            }
#pragma unroll 4
            for (int r = 0; r < half; ++r) {
                const float2 t = from[r * pitch];
                const float d = t.x - about, weighted = __fmul_rn(count(r) + count(r + half), d);
                off = __fadd_rn(off, weighted);
                squares = __fadd_rn(squares, fmaf(weighted, d, t.y));
            }
        }
        const float step = __fmul_rn(off, count.per_pixel);
        each(j < channels ? first * V + j : -1, __fadd_rn(about, step), max_nan(fmaf(-off, step, squares), 0.f));
    }
}

// Mean and M2 of each group over the pixels at `src`, in one pass.  A thread sums the distances d of its pixels from a value p and their squares; p is the first of them and moves to the mean of those so far after
// the first piece and whenever there are twice as many (by t, what the sums are corrected by: sum d - n t, sum d^2 - t (2 sum d - n t)).  (p - mean)^2 of one of n pixels is at most their sum
// of squares, so what the first correction takes away is no more than n times what stays, n being up to kStepRounds; later ones take away at most as much as stays: no sum of squares is
// taken about a value far from its values' mean, wherever the pixels lie that are far from the rest.
// kNear (few_pixels): p is the first pixel's value in all rows, whose sums are simply added; what is taken away in the end is no more than the block's pixels times what stays.
// to(group, (mean, M2)) by one thread each.  red: red_values() float2; channels: c float2.
template <typename T, int V, bool kNear, typename P, typename F>
__device__ __forceinline__ void block_moments(const T *src, P &given, const GroupArgs &a, const Lay &lay, float2 *red, float2 *channels, F to)
{
    decltype(auto) pieces = in_steps(given, lay);
    const int per_group = a.c / a.groups, pixels = pieces.pixels;
    const float per_channel = 1.0f / (float)per_group, n = (float)pixels;
    const bool in_warps = groups_in_warps(lay, per_group), moves = !kNear && pixels > kStepRounds * lay.rows;
    // a channel's mean and squares, and in warps its group's.  (Products that are not left to be fused: the statistics' bits are the same in every variant of the kernels.)
    auto channel = [&](int ch, float mean, float m2) {
        if (in_warps) {
            const float m = __fmul_rn(sum_over(mean, per_group), per_channel);
            m2 = sum_over(fmaf(__fmul_rn(n, mean - m), mean - m, m2), per_group);
            if (ch >= 0 && (ch & (per_group - 1)) == 0) to(ch / per_group, make_float2(m, m2));
        } else if (ch >= 0)
            channels[ch] = make_float2(mean, m2);
    };
    for (int b = 0; b < lay.blocks; ++b) {
        Pairs<V> from = {}, sum = {}, squares = {};           // (-p)
        const bool here = lay.at(b) && lay.row < pixels;
        const int c = (b * lay.lanes + lay.lane) * V;
        int seen = 0;
        for (int piece = 0; piece < pieces.count(); ++piece) {
            pieces.wait(piece);
            if (here) {
                const T *const p = src + pieces.at(piece) * a.c + c;
                if (piece == 0) {                             // (each row has a pixel in the first piece)
                    load_pairs<V>(kNear ? p : p + lay.row * a.c, from);
#pragma unroll
                    for (int k = 0; k < kPairs<V>; ++k) {
                        float x, y;
                        halves(from[k], x, y);
                        if (kNear && lay.row == 0) {          // (a ring's first pixel may be gone when the mean is computed)
                            channels[c + 2 * k].x = x;
                            if (V > 1) channels[c + 2 * k + 1].x = y;
                        }
                        from[k] ^= kMinus;
                    }
                }
                Raw<T, V> raw[kAhead<V>];
                in_batches<kAhead<V>>(
                    lay.row, pieces.end(piece) - pieces.first(piece), lay.rows, [&](int k, int i) { load_raw<V>(raw[k], p + i * a.c); },
                    [&](int k, int, int second) {
                        seen += second < 0 ? 1 : 2;
                        for (int h = 0; h < (second < 0 ? 1 : 2); ++h) {
                            Pairs<V> v;
                            pairs_of<V>(raw[k + h], v);
#pragma unroll
                            for (int j = 0; j < kPairs<V>; ++j) {
                                const uint64_t d = add2(v[j], from[j]);
                                sum[j] = add2(sum[j], d);
                                squares[j] = fma2(d, d, squares[j]);
                            }
                        }
                    });
                if (moves && ((piece & (piece + 1)) == 0 || std::is_same_v<P, InPlace>) && piece + 1 < pieces.count()) {
                    const uint64_t minus = both(-(float)seen), per = both(reciprocal_fast((float)seen));
#pragma unroll
                    for (int j = 0; j < kPairs<V>; ++j) {
                        const uint64_t moved = fma2(sum[j] ^ kMinus, per, from[j]), t = add2(from[j], moved ^ kMinus), left = fma2(minus, t, sum[j]);          // (t as p moved, rounded)
                        squares[j] = fma2(t ^ kMinus, add2(sum[j], left), squares[j]);
                        sum[j] = left;
                        from[j] = moved;
                    }
                }
            }
            pieces.done(piece);
        }
        float mean[2 * kPairs<V>] = {}, m2[2 * kPairs<V>] = {};
        if constexpr (kNear) {
            // the sums
            const float per_pixel = pixels ? 1.0f / (float)pixels : 0.f;
#pragma unroll
            for (int k = 0; k < kPairs<V>; ++k) {
                halves(sum[k], mean[2 * k], mean[2 * k + 1]);
                halves(squares[k], m2[2 * k], m2[2 * k + 1]);
            }
            channel_sums<V>(lay, b, mean, m2, red, [&](int ch, float s, float q) {
                const float d = __fmul_rn(s, per_pixel);
                channel(ch, ch >= 0 && pixels > 0 ? __fadd_rn(channels[ch].x, d) : 0.f, max_nan(fmaf(-s, d, q), 0.f));
            });
        } else {
            // the thread's mean, p + s / n, and M2
            const RowCounts count(pixels, lay);
            if (here) {
                const uint64_t per = both(reciprocal_fast(count(lay.row)));
#pragma unroll
                for (int k = 0; k < kPairs<V>; ++k) {
                    const uint64_t step = mul2(sum[k], per);
                    halves(add2(step, from[k] ^ kMinus), mean[2 * k], mean[2 * k + 1]);
                    halves(fma2(sum[k] ^ kMinus, step, squares[k]), m2[2 * k], m2[2 * k + 1]);
                }
            }
            channel_moments<V>(lay, b, count, mean, m2, red, channel);
        }
    }
    if (in_warps) return;
    lay.sync();
    // groups of so many channels: their means' mean, and what the channels' means are off it
    const Team team(per_group, lay.threads);
    for (int base = 0; base < a.groups; base += team.step) {
        const int g = base + team.first;
        const float2 *const at = channels + g * per_group;
        const int count = g < a.groups ? per_group : 0;
        float mean = 0.f, m2 = 0.f;
        for (int i = team.rank; i < count; i += team.size) mean += at[i].x;
        mean = __fmul_rn(team.sum(mean), per_channel);
        for (int i = team.rank; i < count; i += team.size) {
            const float2 t = at[i];
            m2 = __fadd_rn(m2, fmaf(n * (t.x - mean), t.x - mean, t.y));
        }
        m2 = team.sum(m2);
        if (g < a.groups && team.rank == 0) to(g, make_float2(mean, m2));
    }
}

// What a thread's values are computed with: y = act((x + minus) slope + bias).
template <int V> struct Affine {
    Pairs<V> minus, slope, bias;
    // stats(group): mean and 1 / deviation
    template <typename F>
    __device__ __forceinline__ Affine(const GroupArgs &a, int c, F stats)
    {
        Pairs<V> w;
        vector_pairs<V>(a.weight, c, 1.f, w);
        vector_pairs<V>(a.bias, c, 0.f, bias);
        stats_pairs<V>(c, a.c / a.groups, minus, slope, stats);
#pragma unroll
        for (int k = 0; k < kPairs<V>; ++k) slope[k] = mul2(slope[k], w[k]);
    }
};
// The values of the pixels at `src`, the first of them pixel `first` of the tensor.
template <typename T, int V, int kAct, typename P, typename F>
__device__ __forceinline__ void write_values(const T *src, P &pieces, long long first, const GroupArgs &a, const Lay &lay, F stats)
{
    for (int b = 0; b < lay.blocks; ++b) {
        const bool here = lay.at(b);
        const int c = here ? (b * lay.lanes + lay.lane) * V : 0;
        const Affine<V> f(a, c, stats);
        T *const to = (T *)a.out + first * a.c + c;
        for (int piece = 0; piece < pieces.count(); ++piece) {
            pieces.wait(piece);
            if (here) {
                const T *const p = src + pieces.at(piece) * a.c + c;
                T *const q = to + pieces.first(piece) * a.c;
                Raw<T, V> raw[kAhead<V>];
                in_batches<kAhead<V>>(
                    lay.row, pieces.end(piece) - pieces.first(piece), lay.rows, [&](int k, int i) { load_raw<V>(raw[k], p + i * a.c); },
                    [&](int k, int i, int second) {
                        Pairs<V> v, w;
                        pairs_of<V>(raw[k], v);
                        pairs_of<V>(raw[k + 1], w);
#pragma unroll
                        for (int j = 0; j < kPairs<V>; ++j) {
                            v[j] = activate2<kAct>(fma2(add2(v[j], f.minus[j]), f.slope[j], f.bias[j]));
                            w[j] = activate2<kAct>(fma2(add2(w[j], f.minus[j]), f.slope[j], f.bias[j]));
                        }
                        store_pairs<V>(q + i * a.c, v);
                        if (second >= 0) store_pairs<V>(q + second * a.c, w);
                    });
            }
            pieces.done(piece);
        }
    }
}

// The same as codes, and as values too where they are wanted: a team of lanes a pixel, its largest magnitude first.  A pixel's values stay in registers
// until the codes where a lane has no more than kKeep vectors of them (256x14x14 x 1024 bf16, silu: 114 us, 140 where they are computed again), else they are computed again.  `table`: [3][c] floats of shared memory.
template <int V> constexpr int kKeep = V == 8 ? 2 : V == 4 ? 4 : 8;
template <typename T, int V, int kAct, bool kKeeps, typename P, typename F>
__device__ __forceinline__ void codes_of_run(const T *src, P &pieces, long long first, const GroupArgs &a, const Lay &lay, F stats, float *table)
{
    const int per_group = a.c / a.groups;
    lay.sync();                                               // the last table's readers
    for (int c = threadIdx.x; c < a.c; c += lay.threads) {
        const float2 s = stats(c / per_group);
        table[c] = -s.x;
        table[a.c + c] = s.y * (a.weight ? a.weight[c] : 1.f);
        table[2 * a.c + c] = a.bias ? a.bias[c] : 0.f;
    }
    lay.sync();
    const int columns = a.c / V;
    int size = 1;
    while (size < 32 && size < columns) size *= 2;
    const int rank = threadIdx.x & (size - 1), step = lay.threads / size;
    auto values = [&](int pixel, int c, Pairs<V> &v) {
        load_pairs<V>(src + (long long)pixel * a.c + c, v);   // (pixels as they lie at src)
        Pairs<V> minus, slope, bias;
        vector_pairs<V>(table, c, 0.f, minus);
        vector_pairs<V>(table, a.c + c, 0.f, slope);
        vector_pairs<V>(table, 2 * a.c + c, 0.f, bias);
#pragma unroll
        for (int k = 0; k < kPairs<V>; ++k) v[k] = activate2<kAct>(fma2(add2(v[k], minus[k]), slope[k], bias[k]));
    };
    auto magnitude = [](const Pairs<V> &v, uint32_t most) {
#pragma unroll
        for (int k = 0; k < kPairs<V>; ++k) {
            float x, y;
            halves(v[k], x, y);
            most = max(most, max(abs_bits(x), V > 1 ? abs_bits(y) : 0u));
        }
        return most;
    };
    auto write = [](uint8_t *to, const Pairs<V> &v, const Coder &coder) {
        float f[2 * kPairs<V>];
#pragma unroll
        for (int k = 0; k < kPairs<V>; ++k) halves(v[k], f[2 * k], f[2 * k + 1]);
        if constexpr (V == 8) *reinterpret_cast<uint2 *>(to) = make_uint2(rowcodes::codes_of4(f, coder), rowcodes::codes_of4(f + 4, coder));
        else if constexpr (V == 4) *reinterpret_cast<uint32_t *>(to) = rowcodes::codes_of4(f, coder);
        else if constexpr (V == 2) {
            const float two[4] = {f[0], f[1], 0.f, 0.f};
            *reinterpret_cast<uint16_t *>(to) = (uint16_t)rowcodes::codes_of4(two, coder);
        } else
            *to = rowcodes::code_of(f[0], coder);
    };
    // pixel p of the run is team p % step's, whatever piece it comes in; whole warps go round together
    for (int piece = 0; piece < pieces.count(); ++piece) {
        pieces.wait(piece);
        const int from = pieces.first(piece), end = pieces.end(piece), place = pieces.at(piece) - from;
        for (int base = from / step * step; base < end; base += step) {
            const int pixel = base + threadIdx.x / size;
            const bool here = pixel >= from && pixel < end;
            if (!__any_sync(0xffffffffu, here)) continue;
            T *const out = a.out ? (T *)a.out + (first + pixel) * a.c : nullptr;
            uint8_t *const to = a.codes.codes + (first + pixel) * a.codes.ld;
            uint32_t most = 0;
            Pairs<V> kept[kKeeps ? kKeep<V> : 1];
            if constexpr (kKeeps) {
#pragma unroll
                for (int i = 0; i < kKeep<V>; ++i) {
                    const int c = (i * size + rank) * V;
                    if (!here || c >= a.c) break;
                    values(place + pixel, c, kept[i]);
                    if (out) store_pairs<V>(out + c, kept[i]);
                    most = magnitude(kept[i], most);
                }
            } else if (here)
                for (int c = rank * V; c < a.c; c += size * V) {
                    Pairs<V> v;
                    values(place + pixel, c, v);
                    if (out) store_pairs<V>(out + c, v);
                    most = magnitude(v, most);
                }
            for (int d = size / 2; d; d >>= 1) most = max(most, __shfl_xor_sync(0xffffffffu, most, d));
            const Coder coder(rowcodes::row_scale(most));
            if (!here) continue;
            if (rank == 0) a.codes.scales[first + pixel] = coder.scale;
            if constexpr (kKeeps) {
#pragma unroll
                for (int i = 0; i < kKeep<V>; ++i) {
                    const int c = (i * size + rank) * V;
                    if (c >= a.c) break;
                    write(to + c, kept[i], coder);
                }
            } else
                for (int c = rank * V; c < a.c; c += size * V) {
                    Pairs<V> v;
                    values(place + pixel, c, v);
                    write(to + c, v, coder);
                }
        }
        pieces.done(piece);
    }
}
template <typename T, int V, int kAct, typename P, typename F>
__device__ __forceinline__ void write_codes(const T *src, P &pieces, long long first, const GroupArgs &a, const Lay &lay, F stats, float *table)
{
    if (a.c <= 32 * V * kKeep<V>) codes_of_run<T, V, kAct, true>(src, pieces, first, a, lay, stats, table);
    else codes_of_run<T, V, kAct, false>(src, pieces, first, a, lay, stats, table);
}

// ---- maps in a cluster's shared memory --------------------------------------------------------
// [data, to 16 bytes][red: red_values() float2][moments: groups float2][stats: groups float2][table of the codes: 3 c floats, room for which there
// always is: a map is cut the same way, and has the same statistics to the last bit, whatever is asked for; before it, the channels' c float2]
size_t shared_bytes(const GroupArgs &a, int pixels, int element, int v, int threads)
{
    return ((size_t)pixels * a.c * element + 15) / 16 * 16 + 8 * (size_t)red_values(a.c / v, threads, v) + 16 * (size_t)a.groups + 12 * (size_t)a.c;
}

template <typename T, int V, int kAct, bool kCodes, bool kNear>
__global__ void __launch_bounds__(512, 2) group_norm_map_kernel(const __grid_constant__ GroupArgs a)
{
    using namespace sm100;
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ __align__(8) unsigned long long s_full[kPieces];
    T *const data = reinterpret_cast<T *>(smem);
    float2 *const red = reinterpret_cast<float2 *>(smem + ((size_t)a.share * a.c * sizeof(T) + 15) / 16 * 16);
    float2 *const moments = red + red_values(a.c / V, blockDim.x, V), *const stats = moments + a.groups, *const table = stats + a.groups;
    if (threadIdx.x == 0) {
        for (int i = 0; i < kPieces; ++i) mbar_init(smem_u32(&s_full[i]), 1);
        mbar_fence_init();
    }
    __syncthreads();
    chain_next();
    chain_wait();
    const int rank = blockIdx.x % a.shares;
    const long long map = blockIdx.x / a.shares;
    const int p0 = rank * a.share, pixels = max(0, min(a.share, a.hw - p0)), per_group = a.c / a.groups;
    const long long first = map * a.hw + p0;
    const Lay lay(a.c / V, blockDim.x);
    Pieces pieces(pixels, lay.rows, s_full, a.status);
    if (threadIdx.x == 0) {
        const char *const src = (const char *)((const T *)a.x + first * a.c);
        const uint32_t row = (uint32_t)a.c * sizeof(T);
        for (int i = 0; i < kPieces; ++i) {
            const uint32_t from = pieces.first(i) * row, to = pieces.end(i) * row;
            if (from == to) break;
            mbar_arrive_expect_tx(smem_u32(&s_full[i]), to - from);
            for (uint32_t at = from; at < to; at += 16384) bulk_load(smem_u32(smem) + at, src + at, min(16384u, to - at), smem_u32(&s_full[i]));
        }
    }
    block_moments<T, V, kNear>(data, pieces, a, lay, red, table, [&](int g, float2 m) { moments[g] = m; });
    if (a.shares > 1) cluster_sync();
    else __syncthreads();
    const float count = (float)a.hw * (float)per_group;
    for (int g = threadIdx.x; g < a.groups; g += blockDim.x) {
        float2 m[kMostShares];
        if (a.shares > 1) of_cluster(&moments[g], a.shares, m);
        else m[0] = moments[g];
        float mean = 0.f, m2 = 0.f;
#pragma unroll
        for (int i = 0; i < kMostShares; ++i)
            if (i < a.shares) mean = fmaf(m[i].x, (float)max(0, min(a.share, a.hw - i * a.share)) * (float)per_group / count, mean);
#pragma unroll
        for (int i = 0; i < kMostShares; ++i)
            if (i < a.shares) {
                const float d = m[i].x - mean;
                m2 = __fadd_rn(m2, fmaf((float)max(0, min(a.share, a.hw - i * a.share)) * (float)per_group * d, d, m[i].y));
            }
        const float2 s = make_float2(mean, 1.0f / sqrtf(__fadd_rn(m2 / count, a.eps)));
        stats[g] = s;
        if (rank == 0 && a.stats) a.stats[map * a.groups + g] = s;
    }
    __syncthreads();
    if (a.shares > 1) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    auto of = [&](int g) { return stats[g]; };
    InPlace all{pixels};
    if constexpr (kCodes) write_codes<T, V, kAct>(data, all, first, a, lay, of, reinterpret_cast<float *>(table));
    else write_values<T, V, kAct>(data, all, first, a, lay, of);
    if (a.shares > 1) {
        __syncwarp();
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");       // the others have read this block's moments
    }
}

// ---- maps in runs of pixels ----------------------------------------------------------------------
// A group's mean and 1 / deviation from its runs' moments, by a team of `size` lanes, as channel_moments.  A lane has kHeld runs, or more of them (kMore).
constexpr int kHeld = 4;
static_assert(kInlineRuns <= 32 * kHeld, "a team of 32 lanes holds all runs that are joined inline");
template <bool kMore>
__device__ __forceinline__ float2 join_runs(const GroupArgs &a, long long map, int g, int rank, int size)
{
    const int per_group = a.c / a.groups;
    const float2 *const at = a.part + map * a.shares * a.groups + g;
    auto pixels_of = [&](int r) { return (float)min(a.share, a.hw - r * a.share); };
    auto run = [&](int r) { return r < a.shares ? at[(long long)r * a.groups] : make_float2(0.f, 0.f); };
    const float per_pixel = reciprocal_fast((float)a.hw);
    float2 held[kHeld];
#pragma unroll
    for (int i = 0; i < kHeld; ++i) held[i] = run(rank + i * size);
    float about = at->x, off = 0.f, squares = 0.f;
    if (a.shares > kFew) {
        about = 0.f;
#pragma unroll
        for (int i = 0; i < kHeld; ++i)
            if (rank + i * size < a.shares) about = fmaf(pixels_of(rank + i * size), held[i].x, about);
        if constexpr (kMore)
            for (int r = rank + kHeld * size; r < a.shares; r += size) about = fmaf(pixels_of(r), run(r).x, about);
        about = __fmul_rn(sum_over(about, size), per_pixel);
    }
    auto add = [&](int r, float2 m) {
        const float d = m.x - about, weighted = __fmul_rn(pixels_of(r), d);
        off = __fadd_rn(off, weighted);
        squares = __fadd_rn(squares, fmaf(__fmul_rn(weighted, (float)per_group), d, m.y));
    };
#pragma unroll
    for (int i = 0; i < kHeld; ++i)
        if (rank + i * size < a.shares) add(rank + i * size, held[i]);
    if constexpr (kMore)
        for (int r = rank + kHeld * size; r < a.shares; r += size) add(r, run(r));
    off = sum_over(off, size);
    squares = sum_over(squares, size);
    const float step = __fmul_rn(off, per_pixel);
    squares = max_nan(fmaf(__fmul_rn(-off, (float)per_group), step, squares), 0.f);
    return make_float2(__fadd_rn(about, step), 1.0f / sqrtf(__fadd_rn(squares / ((float)a.hw * (float)per_group), a.eps)));
}

// Maps of many runs: sums[map][group], a warp each.
__global__ void __launch_bounds__(256) group_join_kernel(const __grid_constant__ GroupArgs a)
{
    chain_next();
    chain_wait();
    const long long i = ((long long)blockIdx.x * 256 + threadIdx.x) / 32;
    if (i >= a.n * a.groups) return;
    const float2 v = join_runs<true>(a, i / a.groups, (int)(i % a.groups), threadIdx.x & 31, 32);
    if (threadIdx.x & 31) return;
    a.sums[i] = v;
    if (a.stats) a.stats[i] = v;
}

// part[map][run][group]: moments of a run of pixels.  [ring][red: red_values() float2][channels: c float2]
template <typename T, int V, bool kRing, bool kNear>
__global__ void __launch_bounds__(kRing ? kRunThreads + 32 : kRunThreads, kRing ? kNormBlocks : 4) group_moments_kernel(const __grid_constant__ GroupArgs a, int ring_size)
{
    extern __shared__ __align__(128) unsigned char smem[];
    float2 *const red = reinterpret_cast<float2 *>(smem + ring_size), *const channels = red + red_values(a.c / V, kRunThreads, V);
    const Lay lay(a.c / V, kRunThreads);
    const Run run(a, blockIdx.x);
    float2 *const part = a.part + (long long)run.index * a.groups;
    with_run<T, NormRing, kRing>(a, run, lay, smem, ring_size, [&](const T *src, const T *, auto &pieces) {
        block_moments<T, V, kNear>(src, pieces, a, lay, red, channels, [&](int g, float2 m) { part[g] = m; });
    });
}

// The values, the last runs first: they are the likeliest to be in L2 still.  [ring][stats: groups float2][table of the codes: 3 c floats]
template <typename T, int V, int kAct, bool kCodes, bool kRing>
__global__ void __launch_bounds__(kRing ? kRunThreads + 32 : kRunThreads, kRing ? kNormBlocks : 4) group_values_kernel(const __grid_constant__ GroupArgs a, int ring_size)
{
    extern __shared__ __align__(128) unsigned char smem[];
    float2 *const own = reinterpret_cast<float2 *>(smem + ring_size);
    const Lay lay(a.c / V, kRunThreads);
    const Run run(a, gridDim.x - 1 - blockIdx.x);
    with_run<T, NormRing, kRing>(a, run, lay, smem, ring_size, [&](const T *src, const T *, auto &pieces) {
        if (a.sums)
            for (int g = threadIdx.x; g < a.groups; g += kRunThreads) own[g] = a.sums[run.map * a.groups + g];
        else {
            const Team team(a.shares, kRunThreads);
            for (int base = 0; base < a.groups; base += team.step) {
                const int g = base + team.first;
                const float2 v = join_runs<false>(a, run.map, min(g, a.groups - 1), team.rank, team.size);
                if (g < a.groups && team.rank == 0) {
                    own[g] = v;
                    if (a.stats && run.run == 0) a.stats[run.map * a.groups + g] = v;
                }
            }
        }
        lay.sync();
        auto stats = [&](int g) { return own[g]; };
        if constexpr (kCodes) write_codes<T, V, kAct>(src, pieces, run.first, a, lay, stats, reinterpret_cast<float *>(own + a.groups));
        else write_values<T, V, kAct>(src, pieces, run.first, a, lay, stats);
    });
}

// Whether a block's `pixels` are so few that their squares can be summed about the first one's value.  Sums of n squares, of which a thread has n / rows and a channel's last sum half of the rows' one
// after the other, are off by half as many roundings each, and by n times that where the first pixel is as far from the rest as it can be: 512 roundings of 2^-24 of the variance at most, and
// in all ordinary cases a few.  (The general way has longer code, which small calls wait for: one map of 256x14x14 6.7 us and 7.2, 290 of 64x7x7 8.3 and 9.2.)
bool few_pixels(int pixels, int columns, int threads)
{
    const int blocks = (columns + threads - 1) / threads, rows = threads / ((columns + blocks - 1) / blocks);
    return (long long)pixels * ((pixels + rows - 1) / rows + std::min(pixels, rows) / 2) <= 1024;
}

template <typename T, int V, int kAct, bool kCodes, bool kNear>
tc_status launch_map(int device, const GroupArgs &a, int threads, size_t smem, cudaStream_t s)
{
    constexpr auto kernel = group_norm_map_kernel<T, V, kAct, kCodes, kNear>;
    if (!allow_shared<kernel>(device, kMostShared) || !allow_large_clusters<kernel>(device)) return TC_ERR_CUDA;
    return launch_first_cluster(a.shares, kernel, dim3((unsigned int)(a.n * a.shares)), dim3(threads), smem, s, a) == cudaSuccess ? TC_OK : TC_ERR_CUDA;
}
template <typename T, int V, int kAct, bool kCodes, bool kRing>
tc_status launch_runs(int device, const GroupArgs &a, cudaStream_t s)
{
    constexpr auto general = group_moments_kernel<T, V, kRing, false>, near = group_moments_kernel<T, V, kRing, true>;
    constexpr auto values = group_values_kernel<T, V, kAct, kCodes, kRing>;
    const size_t ring = kRing ? ring_bytes<NormRing>(a.c / V) : 0;
    const size_t first = ring + 8 * (size_t)red_values(a.c / V, kRunThreads, V) + 8 * (size_t)a.c, last = ring + 8 * (size_t)a.groups + (kCodes ? 12 * (size_t)a.c : 0);
    if (!allow_shared<general>(device, kMostShared) || !allow_shared<near>(device, kMostShared) || !allow_shared<values>(device, kMostShared)) return TC_ERR_CUDA;
    const dim3 grid((unsigned int)(a.n * a.shares)), block(kRing ? kRunThreads + 32 : kRunThreads);
    if (launch_first(true, few_pixels(a.share, a.c / V, kRunThreads) ? near : general, grid, block, first, s, a, (int)ring) != cudaSuccess) return TC_ERR_CUDA;
    if (a.sums && launch_chained(true, group_join_kernel, dim3((unsigned int)((a.n * a.groups + 7) / 8)), dim3(256), 0, s, a) != cudaSuccess) return TC_ERR_CUDA;
    return launch_chained(true, values, grid, block, last, s, a, (int)ring) == cudaSuccess ? TC_OK : TC_ERR_CUDA;
}

template <typename T, int V>
tc_status launch(int device, const GroupArgs &a, const GroupPlan &p, int act, cudaStream_t s)
{
    // (maps of other vectors never lie in shared memory: bulk copies begin at 16 bytes)
#define TC_NORM(kAct, kCodes) \
    do { \
        if constexpr (V * sizeof(T) == 16) { \
            if (p.shared) \
                return few_pixels(a.share, a.c / V, p.threads) ? launch_map<T, V, kAct, kCodes, true>(device, a, p.threads, p.shared, s) \
                                                               : launch_map<T, V, kAct, kCodes, false>(device, a, p.threads, p.shared, s); \
            if (ring_takes(a.c, V, sizeof(T))) return launch_runs<T, V, kAct, kCodes, true>(device, a, s); \
        } \
        return launch_runs<T, V, kAct, kCodes, false>(device, a, s); \
    } while (0)
    if (a.codes.codes) {
        if (act == kRelu) TC_NORM(kRelu, true);
        if (act == kSilu) TC_NORM(kSilu, true);
        TC_NORM(kNoAct, true);
    }
    if (act == kRelu) TC_NORM(kRelu, false);
    if (act == kSilu) TC_NORM(kSilu, false);
    TC_NORM(kNoAct, false);
#undef TC_NORM
}

}  // namespace

int tc_group_threads(int columns)
{
    // the number of threads of which the fewest are idle, few of them where that is all the same
    int best = 256, idle = 1 << 30;
    for (int threads = 256; threads <= 512; threads += 32) {
        const int blocks = (columns + threads - 1) / threads, lanes = (columns + blocks - 1) / blocks, rest = (threads - threads / lanes * lanes) * 512 / threads;
        if (rest < idle) { idle = rest; best = threads; }
    }
    return best;
}

void cut_runs(GroupPlan &p, long long n, int hw, int columns, long long row, int tensors, int ring_blocks, int sm_count)
{
    // a thread's sums stay short: so many pixels of a block's rows
    const int blocks_of_columns = (columns + kRunThreads - 1) / kRunThreads, rows = kRunThreads / ((columns + blocks_of_columns - 1) / blocks_of_columns);
    const long long longest = (long long)kMostRounds * rows;
    // in all 2^29 runs at most
    const long long least = std::max(((long long)hw * n + (1ll << 29) - 1) >> 29, 1ll);
    long long share;
    if (ring_blocks) {
        // So many that the blocks' work is least: a run costs as much as kRunCost more of each tensor, and the last ones leave half of the blocks idle.  (Fitted: 128x56x56 x 128 bf16,
        // gradient, in runs of 128, 242, 349, 448 and 628 pixels: 174, 131, 115, 117 and 116 us; 256x56x56 x 128 forward, 126, 349 and 628: 107, 105 and 109.)
        const double blocks = (double)ring_blocks * sm_count;
        const long long shortest = std::max(least, kRunLeast / (row * tensors));
        double best_cost = 0.0;
        share = 0;
        for (long long runs = std::max((hw * row + kRunMost - 1) / kRunMost, (hw + longest - 1) / longest), more; runs <= hw; runs += more) {
            more = std::max(1ll, runs / 8);
            const long long of = std::max(shortest, (hw + runs - 1) / runs);
            const double cost = ((double)n * ((hw + of - 1) / of) / blocks + 0.5) * (double)((of * row + kRunCost) * tensors);
            if (!share || cost < best_cost) { share = of; best_cost = cost; }
            if (of == shortest) break;
        }
    } else {
        // of eight pixels at least where their channels' sums are written too; shorter than kRunBytes where SMs would be idle
        share = std::max(tensors > 1 ? 8ll : 1ll, std::min(longest, kRunBytes / (row * tensors)));
        while (share > 1 && n * ((hw + share - 1) / share) < 2ll * sm_count) share = (share + 1) / 2;
        share = std::max(share, least);
    }
    const long long runs = (hw + std::min<long long>(share, hw) - 1) / std::min<long long>(share, hw);
    p.share = (int)((hw + runs - 1) / runs);                  // (of one size but for the last)
    p.shares = (hw + p.share - 1) / p.share;
    p.join = p.shares > kInlineRuns;
}

GroupPlan tc_plan_group_norm(const GroupNormArgs &m, int sm_count)
{
    GroupPlan p;
    const int element = m.dtype == TC_BF16 ? 2 : 4;
    p.vector = vector_of(m.c, element, m.aligned);
    p.threads = tc_group_threads(m.c / p.vector);
    GroupArgs a{};
    a.c = m.c;
    a.groups = m.groups;
    auto bytes = [&](int shares) { return shared_bytes(a, (m.hw + shares - 1) / shares, element, p.vector, p.threads); };
    if (p.vector * element == 16) {
        // On chip where a block has a map of some size, or for a map or two.  (Others read x a second time from L2, which costs less than waiting for clusters: 256x14x14 bf16 x 1, 2, 8, 30: 6.8,
        // 6.9, 8.7 and 12.8 us on chip, 7.2, 7.1, 7.1 and 10.0 by runs; 832x19x19 x 2: 10.2 and 9.5; without clusters, 256x14x14 x 290: 22 and 26, 64x7x7 x 290: 9.4 and 8.4.)
        const int shares = shares_on_chip(m.n, m.hw, 2, sm_count, bytes);
        if (shares && (m.n <= 2 || (shares == 1 && (long long)m.hw * m.c * element >= kWorthKeeping))) {
            p.shares = shares;
            p.share = (m.hw + shares - 1) / shares;
            p.shared = bytes(shares);
            return p;
        }
    }
    cut_runs(p, m.n, m.hw, m.c / p.vector, (long long)m.c * element, 1, ring_takes(m.c, p.vector, element) ? kNormBlocks : 0, sm_count);
    p.workspace = (size_t)m.n * m.groups * sizeof(float2) * (p.shares + (p.join ? 1 : 0));
    return p;
}

tc_status tc_launch_group_norm(int device, const GroupNormArgs &m, const GroupPlan &p, void *workspace, cudaStream_t s)
{
    GroupArgs a{};
    a.x = m.x;
    a.weight = m.weight;
    a.bias = m.bias;
    a.out = m.y;
    a.codes = m.codes;
    a.stats = (float2 *)m.stats;
    a.eps = m.eps;
    a.n = m.n;
    a.c = m.c;
    a.hw = m.hw;
    a.groups = m.groups;
    a.share = p.share;
    a.shares = p.shares;
    a.status = m.status;
    if (!p.shared) {
        a.part = (float2 *)workspace;
        if (p.join) a.sums = a.part + (long long)a.n * a.groups * a.shares;
    }
    if (m.dtype == TC_BF16) return p.vector == 8 ? launch<__nv_bfloat16, 8>(device, a, p, m.act, s) : p.vector == 2 ? launch<__nv_bfloat16, 2>(device, a, p, m.act, s) : launch<__nv_bfloat16, 1>(device, a, p, m.act, s);
    return p.vector == 4 ? launch<float, 4>(device, a, p, m.act, s) : p.vector == 2 ? launch<float, 2>(device, a, p, m.act, s) : launch<float, 1>(device, a, p, m.act, s);
}
