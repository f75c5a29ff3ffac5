// tc_group_norm_backward: gradients of y = act(z), z = n w + b, n = (x - mean) rstd.  With dz = dy act'(z), sums over a map's pixels
//
//   A_c = sum dz, B_c = sum dz n   ->   db = sum over the maps of A, dw = of B,   s1 = sum over a group's channels of w A, s2 = of w B,
//   dx = rstd (w dz - (s1 + n s2) / m),   m values a group
//
// Bound by the bytes moved, x and dy once and dx once.  As the forward pass: where a map's x and dy fit the shared memory of a cluster's
// blocks they are read once, else by two kernels; dz is computed for the sums and again for dx (it does not fit beside them).  Each block leaves its
// A and B, which the last kernel adds over maps in a fixed order.
// 128x56x56 x 128 bf16, SiLU: 118 us (instructions and memory, x and dy twice); 256x14x14 x 37 f32: 13.5 us.
#include "group_norm.cuh"

#include <type_traits>

namespace {

using namespace groups;

// Blocks an SM: registers enough for both pixels' values.
constexpr int kGradientBlocks = 2;
using GradientRing = Ring<2, 4, 2>;                           // 64 KB
// Vectors that a thread asks for before it works on the first: from shared memory two.
template <typename P, int V> constexpr int kBatch = std::is_same_v<P, InPlace> ? kAhead<V> : 2;

// What a thread needs of its channels: z = (x + minus) slope + b, slope = rstd w.
template <int V> struct Channel {
    Pairs<V> minus, slope, b, rstd;
    template <typename S>
    __device__ __forceinline__ Channel(const GroupArgs &a, S stats, int c)
    {
        stats_pairs<V>(c, a.c / a.groups, minus, rstd, stats);
        vector_pairs<V>(a.weight, c, 1.f, slope);
        vector_pairs<V>(a.bias, c, 0.f, b);
#pragma unroll
        for (int k = 0; k < kPairs<V>; ++k) slope[k] = mul2(slope[k], rstd[k]);
    }
};

// A and B of the channels over the pixels at `src` and `grad`, to part[c] (or null), and to(group, (s1, s2)) by one thread each.  stats(group): the map's.
// red: red_values() float2; sums: c float2.
template <typename T, int V, int kAct, typename P, typename S, typename F>
__device__ __forceinline__ void block_sums(const T *src, const T *grad, P &pieces, const GroupArgs &a, const Lay &lay, S stats, float2 *red, float2 *sums, float2 *part, F to)
{
    const int per_group = a.c / a.groups;
    const bool in_warps = groups_in_warps(lay, per_group);
    for (int b = 0; b < lay.blocks; ++b) {
        Pairs<V> sum_a = {}, sum_b = {};
        const int c = (b * lay.lanes + lay.lane) * V;
        const bool here = lay.at(b);
        const Channel<V> ch(a, stats, here ? c : 0);
        for (int piece = 0; piece < pieces.count(); ++piece) {
            pieces.wait(piece);
            if (here) {
                const T *const p = src + pieces.at(piece) * a.c + c, *const q = grad + pieces.at(piece) * a.c + c;
                constexpr int kMany = kBatch<P, V>;
                Raw<T, V> x[kMany], dy[kMany];
                in_batches<kMany>(
                    lay.row, pieces.end(piece) - pieces.first(piece), lay.rows,
                    [&](int k, int i) {
                        load_raw<V>(x[k], p + i * a.c);
                        load_raw<V>(dy[k], q + i * a.c);
                    },
                    [&](int k, int, int second) {
                        Pairs<V> v, w, d, e;
                        pairs_of<V>(x[k], v);
                        pairs_of<V>(x[k + 1], w);
                        pairs_of<V>(dy[k], d);
                        pairs_of<V>(dy[k + 1], e);
#pragma unroll
                        for (int j = 0; j < kPairs<V>; ++j) {
                            if (second < 0) e[j] = 0;         // (adds nothing, and with the first one's x nothing that is not there already)
                            v[j] = add2(v[j], ch.minus[j]);
                            w[j] = add2(w[j], ch.minus[j]);
                            slope2<kAct>(fma2(v[j], ch.slope[j], ch.b[j]), fma2(w[j], ch.slope[j], ch.b[j]), d[j], e[j]);
                            sum_a[j] = add2(sum_a[j], add2(d[j], e[j]));
                            sum_b[j] = fma2(d[j], v[j], fma2(e[j], w[j], sum_b[j]));
                        }
                    });
            }
            pieces.done(piece);
        }
        // the distances from the mean in units of the deviation
#pragma unroll
        for (int j = 0; j < kPairs<V>; ++j) sum_b[j] = mul2(sum_b[j], ch.rstd[j]);
        float fa[2 * kPairs<V>], fb[2 * kPairs<V>];
#pragma unroll
        for (int k = 0; k < kPairs<V>; ++k) {
            halves(sum_a[k], fa[2 * k], fa[2 * k + 1]);
            halves(sum_b[k], fb[2 * k], fb[2 * k + 1]);
        }
        channel_sums<V>(lay, b, fa, fb, red, [&](int ch, float sa, float sb) {
            if (ch >= 0 && part) part[ch] = make_float2(sa, sb);
            const float w = ch >= 0 && a.weight ? a.weight[ch] : 1.f;
            sa *= w;
            sb *= w;
            if (in_warps) {
                sa = sum_over(sa, per_group);
                sb = sum_over(sb, per_group);
                if (ch >= 0 && (ch & (per_group - 1)) == 0) to(ch / per_group, make_float2(sa, sb));
            } else if (ch >= 0)
                sums[ch] = make_float2(sa, sb);
        });
    }
    if (in_warps) return;
    lay.sync();
    const Team team(per_group, lay.threads);
    for (int base = 0; base < a.groups; base += team.step) {
        const int g = base + team.first;
        float s1 = 0.f, s2 = 0.f;
        if (g < a.groups)
            for (int i = team.rank; i < per_group; i += team.size) {
                s1 += sums[g * per_group + i].x;
                s2 += sums[g * per_group + i].y;
            }
        s1 = team.sum(s1);
        s2 = team.sum(s2);
        if (g < a.groups && team.rank == 0) to(g, make_float2(s1, s2));
    }
}

// dx of the pixels; totals(group) = (s1, s2) / m.
template <typename T, int V, int kAct, typename P, typename S, typename F>
__device__ __forceinline__ void write_gradients(const T *src, const T *grad, P &pieces, long long first, const GroupArgs &a, const Lay &lay, S stats, F totals)
{
    for (int b = 0; b < lay.blocks; ++b) {
        const bool here = lay.at(b);
        const int c = here ? (b * lay.lanes + lay.lane) * V : 0;
        const Channel<V> ch(a, stats, c);
        // dx = w rstd dz - rstd s1 - (x - mean) rstd (rstd s2)
        Pairs<V> by_one, by_x;
        stats_pairs<V>(c, a.c / a.groups, by_one, by_x, totals);
#pragma unroll
        for (int j = 0; j < kPairs<V>; ++j) {
            by_one[j] = mul2(by_one[j], ch.rstd[j]);
            by_x[j] = mul2(mul2(by_x[j], ch.rstd[j]), ch.rstd[j]) ^ kMinus;
        }
        T *const out = (T *)a.out + first * a.c + c;
        for (int piece = 0; piece < pieces.count(); ++piece) {
            pieces.wait(piece);
            if (here) {
                const T *const p = src + pieces.at(piece) * a.c + c, *const q = grad + pieces.at(piece) * a.c + c;
                T *const to = out + pieces.first(piece) * a.c;
                constexpr int kMany = kBatch<P, V>;
                Raw<T, V> x[kMany], dy[kMany];
                in_batches<kMany>(
                    lay.row, pieces.end(piece) - pieces.first(piece), lay.rows,
                    [&](int k, int i) {
                        load_raw<V>(x[k], p + i * a.c);
                        load_raw<V>(dy[k], q + i * a.c);
                    },
                    [&](int k, int i, int second) {
                        Pairs<V> v, w, d, e;
                        pairs_of<V>(x[k], v);
                        pairs_of<V>(x[k + 1], w);
                        pairs_of<V>(dy[k], d);
                        pairs_of<V>(dy[k + 1], e);
#pragma unroll
                        for (int j = 0; j < kPairs<V>; ++j) {
                            v[j] = add2(v[j], ch.minus[j]);
                            w[j] = add2(w[j], ch.minus[j]);
                            slope2<kAct>(fma2(v[j], ch.slope[j], ch.b[j]), fma2(w[j], ch.slope[j], ch.b[j]), d[j], e[j]);
                            v[j] = fma2(d[j], ch.slope[j], fma2(v[j], by_x[j], by_one[j]));
                            w[j] = fma2(e[j], ch.slope[j], fma2(w[j], by_x[j], by_one[j]));
                        }
                        store_pairs<V>(to + i * a.c, v);
                        if (second >= 0) store_pairs<V>(to + second * a.c, w);
                    });
            }
            pieces.done(piece);
        }
    }
}

// ---- maps in a cluster's shared memory --------------------------------------------------------
// [x][dy][red: red_values() float2][sums: c float2][own: groups float2][totals: groups float2]
size_t shared_bytes(const GroupArgs &a, int pixels, int element, int v, int threads)
{
    return 2 * (((size_t)pixels * a.c * element + 15) / 16 * 16) + 8 * (size_t)red_values(a.c / v, threads, v) + 8 * (size_t)a.c + 16 * (size_t)a.groups;
}

template <typename T, int V, int kAct>
__global__ void __launch_bounds__(512) group_gradient_map_kernel(const __grid_constant__ GroupArgs a)
{
    using namespace sm100;
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ __align__(8) unsigned long long s_full[kPieces];
    const size_t room = ((size_t)a.share * a.c * sizeof(T) + 15) / 16 * 16;
    const T *const data = reinterpret_cast<const T *>(smem), *const grad = reinterpret_cast<const T *>(smem + room);
    float2 *const red = reinterpret_cast<float2 *>(smem + 2 * room), *const sums = red + red_values(a.c / V, blockDim.x, V);
    float2 *const own = sums + a.c, *const totals = own + a.groups;
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
        const char *const src = (const char *)((const T *)a.x + first * a.c), *const dy = (const char *)((const T *)a.dy + first * a.c);
        const uint32_t row = (uint32_t)a.c * sizeof(T);
        for (int i = 0; i < kPieces; ++i) {
            const uint32_t from = pieces.first(i) * row, to = pieces.end(i) * row;
            if (from == to) break;
            mbar_arrive_expect_tx(smem_u32(&s_full[i]), 2 * (to - from));
            for (uint32_t at = from; at < to; at += 16384) {
                bulk_load(smem_u32(smem) + at, src + at, min(16384u, to - at), smem_u32(&s_full[i]));
                bulk_load(smem_u32(smem) + (uint32_t)room + at, dy + at, min(16384u, to - at), smem_u32(&s_full[i]));
            }
        }
    }
    auto stats = [&](int g) { return a.stats[map * a.groups + g]; };
    block_sums<T, V, kAct>(data, grad, pieces, a, lay, stats, red, sums, a.part ? a.part + (long long)blockIdx.x * a.c : nullptr, [&](int g, float2 t) { own[g] = t; });
    if (a.shares > 1) cluster_sync();
    else __syncthreads();
    const float per_value = 1.0f / ((float)a.hw * (float)per_group);
    for (int g = threadIdx.x; g < a.groups; g += blockDim.x) {
        float2 m[kMostShares], t = make_float2(0.f, 0.f);
        if (a.shares > 1) of_cluster(&own[g], a.shares, m);
        else m[0] = own[g];
#pragma unroll
        for (int i = 0; i < kMostShares; ++i)
            if (i < a.shares) {
                t.x += m[i].x;
                t.y += m[i].y;
            }
        totals[g] = make_float2(t.x * per_value, t.y * per_value);
    }
    __syncthreads();
    if (a.shares > 1) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    InPlace all{pixels};
    write_gradients<T, V, kAct>(data, grad, all, first, a, lay, stats, [&](int g) { return totals[g]; });
    if (a.shares > 1) {
        __syncwarp();
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");       // the others have read this block's totals
    }
}

// ---- maps in runs of pixels ----------------------------------------------------------------------
// A group's (s1, s2) / m from its runs', by a team of `size` lanes.
__device__ __forceinline__ float2 join_runs(const GroupArgs &a, long long map, int g, int rank, int size)
{
    const float2 *const at = a.runs + map * a.shares * a.groups + g;
    float s1 = 0.f, s2 = 0.f;
#pragma unroll 4
    for (int r = rank; r < a.shares; r += size) {
        const float2 t = at[(long long)r * a.groups];
        s1 += t.x;
        s2 += t.y;
    }
    const float per_value = 1.0f / ((float)a.hw * (float)(a.c / a.groups));
    return make_float2(sum_over(s1, size) * per_value, sum_over(s2, size) * per_value);
}

// Maps of many runs: sums[map][group], a warp each.
__global__ void __launch_bounds__(256) group_totals_kernel(const __grid_constant__ GroupArgs a)
{
    chain_next();
    chain_wait();
    const long long i = ((long long)blockIdx.x * 256 + threadIdx.x) / 32;
    if (i >= a.n * a.groups) return;
    const float2 v = join_runs(a, i / a.groups, (int)(i % a.groups), threadIdx.x & 31, 32);
    if ((threadIdx.x & 31) == 0) a.sums[i] = v;
}

// part[map][run][channel]: A and B of a run of pixels; runs[map][run][group]: its s1 and s2.  [ring of x][ring of dy][red: red_values() float2][sums: c float2]
template <typename T, int V, int kAct, bool kRing>
__global__ void __launch_bounds__(kRing ? kRunThreads + 32 : kRunThreads, kGradientBlocks) group_sums_kernel(const __grid_constant__ GroupArgs a, int ring_size)
{
    extern __shared__ __align__(128) unsigned char smem[];
    float2 *const red = reinterpret_cast<float2 *>(smem + ring_size), *const sums = red + red_values(a.c / V, kRunThreads, V);
    const Lay lay(a.c / V, kRunThreads);
    const Run run(a, blockIdx.x);
    auto stats = [&](int g) { return a.stats[run.map * a.groups + g]; };
    float2 *const to = a.runs + (long long)run.index * a.groups;
    with_run<T, GradientRing, kRing>(a, run, lay, smem, ring_size, [&](const T *x, const T *dy, auto &pieces) {
        block_sums<T, V, kAct>(x, dy, pieces, a, lay, stats, red, sums, a.part ? a.part + (long long)run.index * a.c : nullptr, [&](int g, float2 t) { to[g] = t; });
    });
}

// dx, the last runs first: they are the likeliest to be in L2 still.  [ring of x][ring of dy][totals: groups float2]
template <typename T, int V, int kAct, bool kRing>
__global__ void __launch_bounds__(kRing ? kRunThreads + 32 : kRunThreads, kGradientBlocks) group_gradients_kernel(const __grid_constant__ GroupArgs a, int ring_size)
{
    extern __shared__ __align__(128) unsigned char smem[];
    float2 *const own = reinterpret_cast<float2 *>(smem + ring_size);
    const Lay lay(a.c / V, kRunThreads);
    const Run run(a, gridDim.x - 1 - blockIdx.x);
    with_run<T, GradientRing, kRing>(a, run, lay, smem, ring_size, [&](const T *x, const T *dy, auto &pieces) {
        if (a.sums)
            for (int g = threadIdx.x; g < a.groups; g += kRunThreads) own[g] = a.sums[run.map * a.groups + g];
        else {
            const Team team(a.shares, kRunThreads);
            for (int base = 0; base < a.groups; base += team.step) {
                const int g = base + team.first;
                const float2 v = join_runs(a, run.map, min(g, a.groups - 1), team.rank, team.size);
                if (g < a.groups && team.rank == 0) own[g] = v;
            }
        }
        lay.sync();
        write_gradients<T, V, kAct>(x, dy, pieces, run.first, a, lay, [&](int g) { return a.stats[run.map * a.groups + g]; }, [&](int g) { return own[g]; });
    });
}

// db and dw: sums over the blocks' A and B, 8 channels a block, in 64 bits (there may be many).
constexpr int kVectorThreads = 1024, kVectorChannels = 8;
__global__ void __launch_bounds__(kVectorThreads) group_vectors_kernel(const __grid_constant__ GroupArgs a, long long rows)
{
    chain_next();
    chain_wait();
    __shared__ double2 s_sum[kVectorChannels][kVectorThreads / 32 + 1];
    const int c = blockIdx.x * kVectorChannels + (threadIdx.x & (kVectorChannels - 1)), warp = threadIdx.x / 32, lane = threadIdx.x & 31;
    double2 s = make_double2(0.0, 0.0);
    if (c < a.c)
#pragma unroll 8
        for (long long r = threadIdx.x / kVectorChannels; r < rows; r += kVectorThreads / kVectorChannels) {
            const float2 t = a.part[r * a.c + c];
            s.x += t.x;
            s.y += t.y;
        }
    auto over_lanes = [&](int least) {
        for (int d = 16; d >= least; d >>= 1) {
            s.x += __shfl_xor_sync(0xffffffffu, s.x, d);
            s.y += __shfl_xor_sync(0xffffffffu, s.y, d);
        }
    };
    over_lanes(kVectorChannels);
    if (lane < kVectorChannels) s_sum[lane][warp] = s;
    __syncthreads();
    // a channel's 32 warps' sums: a warp each
    const int mine = blockIdx.x * kVectorChannels + warp;
    if (warp >= kVectorChannels || mine >= a.c) return;
    s = s_sum[warp][lane];
    over_lanes(1);
    if (lane) return;
    if (a.dbias) a.dbias[mine] = (float)s.x;
    if (a.dweight) a.dweight[mine] = (float)s.y;
}

template <typename T, int V, int kAct>
tc_status launch_map(int device, const GroupArgs &a, int threads, size_t smem, cudaStream_t s)
{
    constexpr auto kernel = group_gradient_map_kernel<T, V, kAct>;
    if (!allow_shared<kernel>(device, kMostShared) || !allow_large_clusters<kernel>(device)) return TC_ERR_CUDA;
    return launch_first_cluster(a.shares, kernel, dim3((unsigned int)(a.n * a.shares)), dim3(threads), smem, s, a) == cudaSuccess ? TC_OK : TC_ERR_CUDA;
}
template <typename T, int V, int kAct, bool kRing>
tc_status launch_runs(int device, const GroupArgs &a, cudaStream_t s)
{
    constexpr auto sums = group_sums_kernel<T, V, kAct, kRing>;
    constexpr auto gradients = group_gradients_kernel<T, V, kAct, kRing>;
    const size_t ring = kRing ? ring_bytes<GradientRing>(a.c / V) : 0;
    const size_t first = ring + 8 * (size_t)red_values(a.c / V, kRunThreads, V) + 8 * (size_t)a.c, last = ring + 8 * (size_t)a.groups;
    if (!allow_shared<sums>(device, kMostShared) || !allow_shared<gradients>(device, kMostShared)) return TC_ERR_CUDA;
    const dim3 grid((unsigned int)(a.n * a.shares)), block(kRing ? kRunThreads + 32 : kRunThreads);
    if (launch_first(true, sums, grid, block, first, s, a, (int)ring) != cudaSuccess) return TC_ERR_CUDA;
    if (a.sums && launch_chained(true, group_totals_kernel, dim3((unsigned int)((a.n * a.groups + 7) / 8)), dim3(256), 0, s, a) != cudaSuccess) return TC_ERR_CUDA;
    return launch_chained(true, gradients, grid, block, last, s, a, (int)ring) == cudaSuccess ? TC_OK : TC_ERR_CUDA;
}

template <typename T, int V>
tc_status launch(int device, const GroupArgs &a, const GroupPlan &p, int act, cudaStream_t s)
{
    // (maps of other vectors never lie in shared memory: bulk copies begin at 16 bytes)
#define TC_GRADIENT(kAct) \
    do { \
        if constexpr (V * sizeof(T) == 16) { \
            if (p.shared) return launch_map<T, V, kAct>(device, a, p.threads, p.shared, s); \
            if (ring_takes(a.c, V, sizeof(T))) return launch_runs<T, V, kAct, true>(device, a, s); \
        } \
        return launch_runs<T, V, kAct, false>(device, a, s); \
    } while (0)
    if (act == kRelu) TC_GRADIENT(kRelu);
    if (act == kSilu) TC_GRADIENT(kSilu);
    TC_GRADIENT(kNoAct);
#undef TC_GRADIENT
}

}  // namespace

GroupPlan tc_plan_group_norm_backward(const GroupGradArgs &m, int sm_count)
{
    GroupPlan p;
    const int element = m.dtype == TC_BF16 ? 2 : 4;
    const bool vectors = m.dweight || m.dbias;
    p.vector = vector_of(m.c, element, m.aligned);
    p.threads = tc_group_threads(m.c / p.vector);
    GroupArgs a{};
    a.c = m.c;
    a.groups = m.groups;
    auto bytes = [&](int shares) { return shared_bytes(a, (m.hw + shares - 1) / shares, element, p.vector, p.threads); };
    if (p.vector * element == 16) {
        const int shares = shares_on_chip(m.n, m.hw, 1, sm_count, bytes);
        if (shares) {
            p.shares = shares;
            p.share = (m.hw + shares - 1) / shares;
            p.shared = bytes(shares);
            p.workspace = vectors ? (size_t)m.n * shares * m.c * sizeof(float2) : 0;
            return p;
        }
    }
    cut_runs(p, m.n, m.hw, m.c / p.vector, (long long)m.c * element, 2, ring_takes(m.c, p.vector, element) ? kGradientBlocks : 0, sm_count);
    p.workspace = ((vectors ? (size_t)m.n * p.shares * m.c : 0) + (size_t)m.n * m.groups * (p.shares + (p.join ? 1 : 0))) * sizeof(float2);
    return p;
}

tc_status tc_launch_group_norm_backward(int device, const GroupGradArgs &m, const GroupPlan &p, void *workspace, cudaStream_t s)
{
    GroupArgs a{};
    a.x = m.x;
    a.dy = m.dy;
    a.weight = m.weight;
    a.bias = m.bias;
    a.out = m.dx;
    a.stats = (float2 *)m.stats;
    a.n = m.n;
    a.c = m.c;
    a.hw = m.hw;
    a.groups = m.groups;
    a.share = p.share;
    a.shares = p.shares;
    a.status = m.status;
    a.dweight = m.dweight;
    a.dbias = m.dbias;
    tc_status st = TC_OK;
    if (m.n) {
        if (!p.shared) {
            a.runs = (float2 *)workspace;
            float2 *const rest = a.runs + (long long)a.n * a.shares * a.groups;
            if (p.join) a.sums = rest;
            if (a.dweight || a.dbias) a.part = rest + (p.join ? (long long)a.n * a.groups : 0);
        } else if (p.workspace)
            a.part = (float2 *)workspace;
        if (m.dtype == TC_BF16) st = p.vector == 8 ? launch<__nv_bfloat16, 8>(device, a, p, m.act, s) : p.vector == 2 ? launch<__nv_bfloat16, 2>(device, a, p, m.act, s) : launch<__nv_bfloat16, 1>(device, a, p, m.act, s);
        else st = p.vector == 4 ? launch<float, 4>(device, a, p, m.act, s) : p.vector == 2 ? launch<float, 2>(device, a, p, m.act, s) : launch<float, 1>(device, a, p, m.act, s);
    }
    if (st != TC_OK || (!a.dweight && !a.dbias)) return st;
    const dim3 grid((unsigned int)((a.c + kVectorChannels - 1) / kVectorChannels));
    return launch_chained(m.n > 0, group_vectors_kernel, grid, dim3(kVectorThreads), 0, s, a, a.n * a.shares) == cudaSuccess ? TC_OK : TC_ERR_CUDA;
}
