// tc_group_norm: of maps whose channels are neighbours in memory,
//
//   y = act((x - mean) rstd w + b),   mean and rstd = 1 / sqrt(var + eps) over a map's pixels and a group's channels
//
// Bound by the bytes moved, x once and y once.  Where a map fits the shared memory of a cluster's blocks (up to eight) it is read once: each block
// takes its pixels there by bulk copies, finds its mean and then its squares about that mean, the blocks' moments are put together through
// the cluster's shared memory, and the values leave from where they lie.  Larger maps, and rows that do not begin at 16 bytes, take
// three kernels: moments of runs of pixels, their joining, and the values (last runs first: they are the likeliest to be in L2 still).
//
// Moments are put together as (n, mean, M2): no sum of squares is taken about a mean far from its own.
#include "group_norm.cuh"
#include "integer_codes.cuh"
#include "sm100_ptx.cuh"

namespace {

using namespace groups;
using rowcodes::Coder;

// Mean and M2 (sum of squares about it) of each group over `pixels` pixels at `src`, to moments[group].
template <typename T, int V>
__device__ __forceinline__ void block_moments(const T *src, int pixels, const GroupArgs &a, const Lay &lay, float *red, float2 *moments)
{
    const int per_group = a.c / a.groups;
    const float count = (float)pixels * (float)per_group;
    for (int g = threadIdx.x; g < a.groups; g += blockDim.x) moments[g] = make_float2(0.f, 0.f);
    for (int b = 0; b < lay.blocks; ++b) {
        Pairs<V> sum = {};
        if (lay.at(b)) {
            const T *p = src + (long long)lay.row * a.c + (b * lay.lanes + lay.lane) * V;
#pragma unroll 4
            for (int i = lay.row; i < pixels; i += lay.rows, p += (long long)lay.rows * a.c) {
                Pairs<V> v;
                load_pairs<V>(p, v);
#pragma unroll
                for (int k = 0; k < kPairs<V>; ++k) sum[k] = add2(sum[k], v[k]);
            }
        }
        add_groups<V>(lay, b, per_group, a.groups, sum, red, [&](int g, float s) { moments[g].x += s; });
    }
    __syncthreads();
    for (int g = threadIdx.x; g < a.groups; g += blockDim.x) moments[g].x = pixels ? moments[g].x / count : 0.f;
    __syncthreads();
    for (int b = 0; b < lay.blocks; ++b) {
        Pairs<V> sum = {};
        if (lay.at(b)) {
            const int c = (b * lay.lanes + lay.lane) * V;
            const T *p = src + (long long)lay.row * a.c + c;
            Pairs<V> minus, unused;
            stats_pairs<V>(moments, c, per_group, minus, unused);
#pragma unroll 4
            for (int i = lay.row; i < pixels; i += lay.rows, p += (long long)lay.rows * a.c) {
                Pairs<V> v;
                load_pairs<V>(p, v);
#pragma unroll
                for (int k = 0; k < kPairs<V>; ++k) {
                    const uint64_t d = add2(v[k], minus[k]);
                    sum[k] = fma2(d, d, sum[k]);
                }
            }
        }
        add_groups<V>(lay, b, per_group, a.groups, sum, red, [&](int g, float s) { moments[g].y += s; });
    }
    __syncthreads();
}

// Joins the moments of `parts` runs of pixels: of(i) = (mean, M2), run i having pixels(i).
template <typename F, typename G>
__device__ __forceinline__ float2 joined(int parts, float count, int per_group, float eps, G pixels, F of)
{
    float mean = 0.f, m2 = 0.f;
    for (int i = 0; i < parts; ++i) mean += of(i).x * ((float)pixels(i) * (float)per_group / count);
    for (int i = 0; i < parts; ++i) {
        const float2 m = of(i);
        const float d = m.x - mean;
        m2 += m.y + (float)pixels(i) * (float)per_group * d * d;
    }
    return make_float2(mean, 1.0f / sqrtf(m2 / count + eps));
}

// The values of `pixels` pixels at `src`, the first of them pixel `first` of the tensor; stats[group] as they are found in shared memory.
template <typename T, int V, int kAct>
__device__ __forceinline__ void write_values(const T *src, int pixels, long long first, const GroupArgs &a, const Lay &lay, const float2 *stats)
{
    const int per_group = a.c / a.groups;
    for (int b = 0; b < lay.blocks; ++b) {
        if (!lay.at(b)) continue;
        const int c = (b * lay.lanes + lay.lane) * V;
        Pairs<V> minus, slope, w, bias;
        stats_pairs<V>(stats, c, per_group, minus, slope);
        vector_pairs<V>(a.weight, c, 1.f, w);
        vector_pairs<V>(a.bias, c, 0.f, bias);
#pragma unroll
        for (int k = 0; k < kPairs<V>; ++k) slope[k] = mul2(slope[k], w[k]);
        const long long at = (long long)lay.row * a.c + c, step = (long long)lay.rows * a.c;
        const T *p = src + at;
        T *q = (T *)a.out + first * a.c + at;
#pragma unroll 4
        for (int i = lay.row; i < pixels; i += lay.rows, p += step, q += step) {
            Pairs<V> v;
            load_pairs<V>(p, v);
#pragma unroll
            for (int k = 0; k < kPairs<V>; ++k) v[k] = activate2<kAct>(fma2(add2(v[k], minus[k]), slope[k], bias[k]));
            store_pairs<V>(q, v);
        }
    }
}

// The same as codes, and as values too where they are wanted: a team of lanes a pixel, its largest magnitude first.  `table`: [3][c] floats of shared memory.
template <typename T, int V, int kAct>
__device__ __forceinline__ void write_codes(const T *src, int pixels, long long first, const GroupArgs &a, const float2 *stats, float *table)
{
    const int per_group = a.c / a.groups;
    for (int c = threadIdx.x; c < a.c; c += blockDim.x) {
        const float2 s = stats[c / per_group];
        table[c] = -s.x;
        table[a.c + c] = s.y * (a.weight ? a.weight[c] : 1.f);
        table[2 * a.c + c] = a.bias ? a.bias[c] : 0.f;
    }
    __syncthreads();
    const int columns = a.c / V;
    int size = 1;
    while (size < 32 && size < columns) size *= 2;
    const int rank = threadIdx.x & (size - 1), step = blockDim.x / size;
    auto values = [&](int pixel, int c, Pairs<V> &v) {
        load_pairs<V>(src + (long long)pixel * a.c + c, v);
        Pairs<V> minus, slope, bias;
        vector_pairs<V>(table, c, 0.f, minus);
        vector_pairs<V>(table, a.c + c, 0.f, slope);
        vector_pairs<V>(table, 2 * a.c + c, 0.f, bias);
#pragma unroll
        for (int k = 0; k < kPairs<V>; ++k) v[k] = activate2<kAct>(fma2(add2(v[k], minus[k]), slope[k], bias[k]));
    };
    for (int base = 0; base < pixels; base += step) {         // (whole warps go round together)
        const int pixel = base + threadIdx.x / size;
        const bool here = pixel < pixels;
        uint32_t most = 0;
        if (here)
            for (int c = rank * V; c < a.c; c += size * V) {
                Pairs<V> v;
                values(pixel, c, v);
                if (a.out) store_pairs<V>((T *)a.out + (first + pixel) * a.c + c, v);
#pragma unroll
                for (int k = 0; k < kPairs<V>; ++k) {
                    float x, y;
                    halves(v[k], x, y);
                    most = max(most, max(abs_bits(x), V > 1 ? abs_bits(y) : 0u));
                }
            }
        for (int d = size / 2; d; d >>= 1) most = max(most, __shfl_xor_sync(0xffffffffu, most, d));
        const Coder coder(rowcodes::row_scale(most));
        if (!here) continue;
        if (rank == 0) a.codes.scales[first + pixel] = coder.scale;
        uint8_t *const to = a.codes.codes + (first + pixel) * a.codes.ld;
        for (int c = rank * V; c < a.c; c += size * V) {
            Pairs<V> v;
            values(pixel, c, v);
            float f[2 * kPairs<V>];
#pragma unroll
            for (int k = 0; k < kPairs<V>; ++k) halves(v[k], f[2 * k], f[2 * k + 1]);
            if constexpr (V == 8) *reinterpret_cast<uint2 *>(to + c) = make_uint2(rowcodes::codes_of4(f, coder), rowcodes::codes_of4(f + 4, coder));
            else if constexpr (V == 4) *reinterpret_cast<uint32_t *>(to + c) = rowcodes::codes_of4(f, coder);
            else to[c] = rowcodes::code_of(f[0], coder);
        }
    }
}

// ---- maps in a cluster's shared memory --------------------------------------------------------
// [data, to 16 bytes][red: threads x V floats][moments: groups float2][stats: groups float2][table of the codes: 3 c floats, room for which there
// always is: a map is cut the same way, and has the same statistics to the last bit, whatever is asked for]
size_t shared_bytes(const GroupArgs &a, int pixels, int element, int v, int threads)
{
    return ((size_t)pixels * a.c * element + 15) / 16 * 16 + (size_t)threads * v * 4 + 16 * (size_t)a.groups + 12 * (size_t)a.c;
}

template <typename T, int V, int kAct, bool kCodes>
__global__ void __launch_bounds__(512) group_norm_map_kernel(const __grid_constant__ GroupArgs a)
{
    using namespace sm100;
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ __align__(8) unsigned long long s_full;
    T *const data = reinterpret_cast<T *>(smem);
    float *const red = reinterpret_cast<float *>(smem + ((size_t)a.share * a.c * sizeof(T) + 15) / 16 * 16);
    float2 *const moments = reinterpret_cast<float2 *>(red + blockDim.x * V), *const stats = moments + a.groups;
    if (threadIdx.x == 0) { mbar_init(smem_u32(&s_full), 1); mbar_fence_init(); }
    __syncthreads();
    chain_next();
    chain_wait();
    const int rank = blockIdx.x % a.shares;
    const long long map = blockIdx.x / a.shares;
    const int p0 = rank * a.share, pixels = max(0, min(a.share, a.hw - p0)), per_group = a.c / a.groups;
    const long long first = map * a.hw + p0;
    if (pixels) {
        if (threadIdx.x == 0) {
            const uint32_t bytes = (uint32_t)pixels * a.c * sizeof(T);
            mbar_arrive_expect_tx(smem_u32(&s_full), bytes);
            const char *const src = (const char *)((const T *)a.x + first * a.c);
            for (uint32_t at = 0; at < bytes; at += 16384) bulk_load(smem_u32(smem) + at, src + at, min(16384u, bytes - at), smem_u32(&s_full));
        }
        // (a wait that runs out is reported; the values are wrong then, nothing else)
        if (!mbar_wait_soon(smem_u32(&s_full), 0) && !mbar_wait_soon(smem_u32(&s_full), 0)) tc_dev_set_status(a.status, TC_ERR_TIMEOUT);
    }
    const Lay lay(a.c / V);
    block_moments<T, V>(data, pixels, a, lay, red, moments);
    if (a.shares > 1) cluster_sync();
    const float count = (float)a.hw * (float)per_group;
    for (int g = threadIdx.x; g < a.groups; g += blockDim.x) {
        const float2 s = joined(a.shares, count, per_group, a.eps, [&](int i) { return max(0, min(a.share, a.hw - i * a.share)); }, [&](int i) {
            float2 m;
            asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(m.x), "=f"(m.y) : "r"(peer_address(&moments[g], (uint32_t)i)));
            return m;
        });
        stats[g] = s;
        if (rank == 0 && a.stats) a.stats[map * a.groups + g] = s;
    }
    __syncthreads();
    if (a.shares > 1) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    if constexpr (kCodes) write_codes<T, V, kAct>(data, pixels, first, a, stats, reinterpret_cast<float *>(stats + a.groups));
    else write_values<T, V, kAct>(data, pixels, first, a, lay, stats);
    if (a.shares > 1) {
        __syncwarp();
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");       // the others have read this block's moments
    }
}

// ---- any maps ----------------------------------------------------------------------------------
// part[map][share][group]: moments of a run of pixels.
template <typename T, int V>
__global__ void __launch_bounds__(512) group_moments_kernel(const __grid_constant__ GroupArgs a)
{
    extern __shared__ __align__(128) unsigned char smem[];
    float *const red = reinterpret_cast<float *>(smem);
    float2 *const moments = reinterpret_cast<float2 *>(red + blockDim.x * V);
    chain_next();
    chain_wait();
    const long long map = blockIdx.x / a.shares;
    const int p0 = (int)(blockIdx.x % a.shares) * a.share, pixels = max(0, min(a.share, a.hw - p0));
    const Lay lay(a.c / V);
    block_moments<T, V>((const T *)a.x + (map * a.hw + p0) * a.c, pixels, a, lay, red, moments);
    for (int g = threadIdx.x; g < a.groups; g += blockDim.x) a.part[(long long)blockIdx.x * a.groups + g] = moments[g];
}

// sums[map][group]: mean and 1 / deviation of a map's groups, a warp each.
__global__ void __launch_bounds__(256) group_join_kernel(const __grid_constant__ GroupArgs a)
{
    chain_next();
    chain_wait();
    const long long i = ((long long)blockIdx.x * 256 + threadIdx.x) / 32;
    const int lane = threadIdx.x & 31, per_group = a.c / a.groups;
    if (i >= a.n * a.groups) return;
    const long long map = i / a.groups;
    const int g = (int)(i - map * a.groups);
    const float count = (float)a.hw * (float)per_group;
    auto pixels = [&](int s) { return (float)max(0, min(a.share, a.hw - s * a.share)); };
    auto of = [&](int s) { return a.part[(map * a.shares + s) * a.groups + g]; };
    float mean = 0.f, m2 = 0.f;
    for (int s = lane; s < a.shares; s += 32) mean += of(s).x * (pixels(s) * (float)per_group / count);
    for (int d = 16; d; d >>= 1) mean += __shfl_xor_sync(0xffffffffu, mean, d);
    for (int s = lane; s < a.shares; s += 32) {
        const float2 m = of(s);
        m2 += m.y + pixels(s) * (float)per_group * (m.x - mean) * (m.x - mean);
    }
    for (int d = 16; d; d >>= 1) m2 += __shfl_xor_sync(0xffffffffu, m2, d);
    if (lane) return;
    const float2 s = make_float2(mean, 1.0f / sqrtf(m2 / count + a.eps));
    a.sums[i] = s;
    if (a.stats) a.stats[i] = s;
}

template <typename T, int V, int kAct, bool kCodes>
__global__ void __launch_bounds__(512) group_values_kernel(const __grid_constant__ GroupArgs a)
{
    extern __shared__ __align__(128) unsigned char smem[];
    float2 *const stats = reinterpret_cast<float2 *>(smem);
    chain_next();
    chain_wait();
    const long long block = (long long)gridDim.x - 1 - blockIdx.x, map = block / a.shares;
    const int p0 = (int)(block % a.shares) * a.share, pixels = max(0, min(a.share, a.hw - p0));
    for (int g = threadIdx.x; g < a.groups; g += blockDim.x) stats[g] = a.sums[map * a.groups + g];
    __syncthreads();
    const long long first = map * a.hw + p0;
    const T *const src = (const T *)a.x + first * a.c;
    const Lay lay(a.c / V);
    if constexpr (kCodes) write_codes<T, V, kAct>(src, pixels, first, a, stats, reinterpret_cast<float *>(stats + a.groups));
    else write_values<T, V, kAct>(src, pixels, first, a, lay, stats);
}

template <typename T, int V, int kAct, bool kCodes>
tc_status launch_map(int device, const GroupArgs &a, int threads, size_t smem, cudaStream_t s)
{
    constexpr auto kernel = group_norm_map_kernel<T, V, kAct, kCodes>;
    if (!allow_shared<kernel>(device, 225 * 1024)) return TC_ERR_CUDA;
    return launch_first_cluster(a.shares, kernel, dim3((unsigned int)(a.n * a.shares)), dim3(threads), smem, s, a) == cudaSuccess ? TC_OK : TC_ERR_CUDA;
}
template <typename T, int V, int kAct, bool kCodes>
tc_status launch_any(int device, const GroupArgs &a, int threads, cudaStream_t s)
{
    const size_t first = (size_t)threads * V * 4 + 8 * (size_t)a.groups, last = 8 * (size_t)a.groups + (kCodes ? 12 * (size_t)a.c : 0);
    if (!allow_shared<group_moments_kernel<T, V>>(device, 225 * 1024) || !allow_shared<group_values_kernel<T, V, kAct, kCodes>>(device, 225 * 1024)) return TC_ERR_CUDA;
    const dim3 grid((unsigned int)(a.n * a.shares)), block(threads);
    if (launch_first(true, group_moments_kernel<T, V>, grid, block, first, s, a) != cudaSuccess) return TC_ERR_CUDA;
    if (launch_chained(true, group_join_kernel, dim3((unsigned int)((a.n * a.groups + 7) / 8)), dim3(256), 0, s, a) != cudaSuccess) return TC_ERR_CUDA;
    return launch_chained(true, group_values_kernel<T, V, kAct, kCodes>, grid, block, last, s, a) == cudaSuccess ? TC_OK : TC_ERR_CUDA;
}

template <typename T, int V>
tc_status launch(int device, const GroupArgs &a, int act, int threads, size_t smem, cudaStream_t s)
{
#define TC_NORM(kAct) \
    (smem ? a.codes.codes ? launch_map<T, V, kAct, true>(device, a, threads, smem, s) : launch_map<T, V, kAct, false>(device, a, threads, smem, s) \
          : a.codes.codes ? launch_any<T, V, kAct, true>(device, a, threads, s) : launch_any<T, V, kAct, false>(device, a, threads, s))
    return act == kRelu ? TC_NORM(kRelu) : act == kSilu ? TC_NORM(kSilu) : TC_NORM(kNoAct);
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

GroupPlan tc_plan_group_norm(const GroupNormArgs &m, int sm_count)
{
    GroupPlan p;
    const int element = m.dtype == TC_BF16 ? 2 : 4;
    p.vector = m.c * element % 16 == 0 && m.aligned ? 16 / element : 1;
    p.threads = tc_group_threads(m.c / p.vector);
    GroupArgs a{};
    a.c = m.c;
    a.groups = m.groups;
    auto bytes = [&](int shares) { return shared_bytes(a, (m.hw + shares - 1) / shares, element, p.vector, p.threads); };
    if (p.vector > 1) {
        // as few blocks a map as let three share an SM (one loads while the others work), then as many as the SMs take
        int shares = 1;
        while (shares < 8 && bytes(shares) > 73 * 1024) shares *= 2;
        while (shares < 8 && (long long)m.n * shares * 2 <= sm_count && m.hw / shares >= 16) shares *= 2;
        if (bytes(shares) <= 225 * 1024 && (long long)m.n * shares < 1ll << 31) {
            p.shares = shares;
            p.share = (m.hw + shares - 1) / shares;
            p.shared = bytes(shares);
            return p;
        }
    }
    // runs of about 64 KB, as many as let every SM have several
    const long long row = (long long)m.c * element;
    long long share = std::max(1ll, 65536 / row);
    while (share > 1 && (long long)m.n * ((m.hw + share - 1) / share) < 4ll * sm_count) share = (share + 1) / 2;
    share = std::max(share, ((long long)m.hw * m.n + (1ll << 30) - 1) >> 30);
    p.share = (int)std::min<long long>(share, m.hw);
    p.shares = (m.hw + p.share - 1) / p.share;
    p.workspace = (size_t)m.n * m.groups * sizeof(float2) * (p.shares + 1);
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
        a.sums = (float2 *)workspace;
        a.part = a.sums + (long long)a.n * a.groups;
    }
    if (m.dtype == TC_BF16) return p.vector == 8 ? launch<__nv_bfloat16, 8>(device, a, m.act, p.threads, p.shared, s) : launch<__nv_bfloat16, 1>(device, a, m.act, p.threads, p.shared, s);
    return p.vector == 4 ? launch<float, 4>(device, a, m.act, p.threads, p.shared, s) : launch<float, 1>(device, a, m.act, p.threads, p.shared, s);
}
