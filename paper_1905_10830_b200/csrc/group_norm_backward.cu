// tc_group_norm_backward: gradients of y = act(z), z = n w + b, n = (x - mean) rstd.  With dz = dy act'(z), sums over a map's pixels
//
//   A_c = sum dz, B_c = sum dz n   ->   db = sum over the maps of A, dw = of B,   s1 = sum over a group's channels of w A, s2 = of w B,
//   dx = rstd (w dz - (s1 + n s2) / m),   m values a group
//
// Bound by the bytes moved, x and dy once and dx once.  As the forward pass: where a map's x and dy fit the shared memory of a cluster's
// blocks they are read once, else by two kernels; dz is computed for the sums and again for dx (it does not fit beside them).  Each block leaves its
// A and B, which the last kernel adds over maps in a fixed order.
#include "group_norm.cuh"
#include "sm100_ptx.cuh"

namespace {

using namespace groups;

// What a thread needs of its channels.
template <int V> struct Channel {
    Pairs<V> minus, rstd, w, b;
    __device__ __forceinline__ void load(const GroupArgs &a, const float2 *stats, int c)
    {
        stats_pairs<V>(stats, c, a.c / a.groups, minus, rstd);
        vector_pairs<V>(a.weight, c, 1.f, w);
        vector_pairs<V>(a.bias, c, 0.f, b);
    }
};

// sums[c] = (A, B) over `pixels` pixels; x and dy at `src` and `grad`.  red: blockDim x V float2.
template <typename T, int V, int kAct>
__device__ __forceinline__ void block_sums(const T *src, const T *grad, int pixels, const GroupArgs &a, const Lay &lay, const float2 *stats, float2 *red, float2 *sums)
{
    for (int b = 0; b < lay.blocks; ++b) {
        __syncthreads();                                      // the readers of the last block's sums
        if (lay.at(b)) {
            const int c = (b * lay.lanes + lay.lane) * V;
            Channel<V> ch;
            ch.load(a, stats, c);
            Pairs<V> sum_a = {}, sum_b = {};
            const long long at = (long long)lay.row * a.c + c, step = (long long)lay.rows * a.c;
            const T *p = src + at, *q = grad + at;
#pragma unroll 2
            for (int i = lay.row; i < pixels; i += lay.rows, p += step, q += step) {
                Pairs<V> v, d;
                load_pairs<V>(p, v);
                load_pairs<V>(q, d);
#pragma unroll
                for (int k = 0; k < kPairs<V>; ++k) {
                    const uint64_t n = mul2(add2(v[k], ch.minus[k]), ch.rstd[k]);
                    const uint64_t dz = slope2<kAct>(fma2(n, ch.w[k], ch.b[k]), d[k]);
                    sum_a[k] = add2(sum_a[k], dz);
                    sum_b[k] = fma2(dz, n, sum_b[k]);
                }
            }
            float fa[2 * kPairs<V>], fb[2 * kPairs<V>];
#pragma unroll
            for (int k = 0; k < kPairs<V>; ++k) {
                halves(sum_a[k], fa[2 * k], fa[2 * k + 1]);
                halves(sum_b[k], fb[2 * k], fb[2 * k + 1]);
            }
#pragma unroll
            for (int i = 0; i < V; ++i) red[(lay.row * V + i) * lay.lanes + lay.lane] = make_float2(fa[i], fb[i]);
        }
        __syncthreads();
        const int first = b * lay.lanes, lanes = min(lay.lanes, lay.columns - first);
        for (int j = threadIdx.x; j < lanes * V; j += blockDim.x) {
            const int i = j / lanes, lane = j - i * lanes;
            float2 s = red[i * lay.lanes + lane];
            for (int r = 1; r < lay.rows; ++r) {
                const float2 t = red[(r * V + i) * lay.lanes + lane];
                s.x += t.x;
                s.y += t.y;
            }
            sums[(first + lane) * V + i] = s;
        }
    }
    __syncthreads();
}

// totals[g] = (s1, s2) from sums of channels: of(c).
template <typename F>
__device__ __forceinline__ void group_totals(const GroupArgs &a, F of, float2 *totals)
{
    const int per_group = a.c / a.groups;
    const Team team(per_group);
    for (int base = 0; base < a.groups; base += team.step) {
        const int g = base + team.first;
        float s1 = 0.f, s2 = 0.f;
        if (g < a.groups)
            for (int i = team.rank; i < per_group; i += team.size) {
                const int c = g * per_group + i;
                const float w = a.weight ? a.weight[c] : 1.f;
                const float2 s = of(c);
                s1 += w * s.x;
                s2 += w * s.y;
            }
        s1 = team.sum(s1);
        s2 = team.sum(s2);
        if (g < a.groups && team.rank == 0) totals[g] = make_float2(s1, s2);
    }
    __syncthreads();
}

// dx of `pixels` pixels; totals[g] = (s1, s2) / m.
template <typename T, int V, int kAct>
__device__ __forceinline__ void write_gradients(const T *src, const T *grad, int pixels, long long first, const GroupArgs &a, const Lay &lay, const float2 *stats, const float2 *totals)
{
    for (int b = 0; b < lay.blocks; ++b) {
        if (!lay.at(b)) continue;
        const int c = (b * lay.lanes + lay.lane) * V;
        Channel<V> ch;
        ch.load(a, stats, c);
        Pairs<V> minus_s1, s2;
        stats_pairs<V>(totals, c, a.c / a.groups, minus_s1, s2);
        const long long at = (long long)lay.row * a.c + c, step = (long long)lay.rows * a.c;
        const T *p = src + at, *q = grad + at;
        T *to = (T *)a.out + first * a.c + at;
#pragma unroll 2
        for (int i = lay.row; i < pixels; i += lay.rows, p += step, q += step, to += step) {
            Pairs<V> v, d;
            load_pairs<V>(p, v);
            load_pairs<V>(q, d);
#pragma unroll
            for (int k = 0; k < kPairs<V>; ++k) {
                const uint64_t n = mul2(add2(v[k], ch.minus[k]), ch.rstd[k]);
                const uint64_t dz = slope2<kAct>(fma2(n, ch.w[k], ch.b[k]), d[k]);
                // w dz - s1 - n s2
                const uint64_t rest = fma2(n, s2[k] ^ 0x8000000080000000ull, fma2(dz, ch.w[k], minus_s1[k]));
                v[k] = mul2(rest, ch.rstd[k]);
            }
            store_pairs<V>(to, v);
        }
    }
}

// ---- maps in a cluster's shared memory --------------------------------------------------------
// [x][dy][red: threads x V float2][sums: c float2][stats: groups float2][own: groups float2][totals: groups float2]
size_t shared_bytes(const GroupArgs &a, int pixels, int element, int v, int threads)
{
    return 2 * (((size_t)pixels * a.c * element + 15) / 16 * 16) + (size_t)threads * v * 8 + 8 * (size_t)a.c + 24 * (size_t)a.groups;
}

template <typename T, int V, int kAct>
__global__ void __launch_bounds__(512) group_gradient_map_kernel(const __grid_constant__ GroupArgs a)
{
    using namespace sm100;
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ __align__(8) unsigned long long s_full;
    const size_t room = ((size_t)a.share * a.c * sizeof(T) + 15) / 16 * 16;
    const T *const data = reinterpret_cast<const T *>(smem), *const grad = reinterpret_cast<const T *>(smem + room);
    float2 *const red = reinterpret_cast<float2 *>(smem + 2 * room), *const sums = red + blockDim.x * V;
    float2 *const stats = sums + a.c, *const own = stats + a.groups, *const totals = own + a.groups;
    if (threadIdx.x == 0) { mbar_init(smem_u32(&s_full), 1); mbar_fence_init(); }
    __syncthreads();
    chain_next();
    chain_wait();
    const int rank = blockIdx.x % a.shares;
    const long long map = blockIdx.x / a.shares;
    const int p0 = rank * a.share, pixels = max(0, min(a.share, a.hw - p0)), per_group = a.c / a.groups;
    const long long first = map * a.hw + p0;
    if (pixels && threadIdx.x == 0) {
        const uint32_t bytes = (uint32_t)pixels * a.c * sizeof(T);
        mbar_arrive_expect_tx(smem_u32(&s_full), 2 * bytes);
        const char *const src = (const char *)((const T *)a.x + first * a.c), *const dy = (const char *)((const T *)a.dy + first * a.c);
        for (uint32_t at = 0; at < bytes; at += 16384) {
            bulk_load(smem_u32(smem) + at, src + at, min(16384u, bytes - at), smem_u32(&s_full));
            bulk_load(smem_u32(smem) + (uint32_t)room + at, dy + at, min(16384u, bytes - at), smem_u32(&s_full));
        }
    }
    for (int g = threadIdx.x; g < a.groups; g += blockDim.x) stats[g] = a.stats[map * a.groups + g];
    // (a wait that runs out is reported; the values are wrong then, nothing else)
    if (pixels && !mbar_wait_soon(smem_u32(&s_full), 0) && !mbar_wait_soon(smem_u32(&s_full), 0)) tc_dev_set_status(a.status, TC_ERR_TIMEOUT);
    const Lay lay(a.c / V);
    block_sums<T, V, kAct>(data, grad, pixels, a, lay, stats, red, sums);
    if (a.part)
        for (int c = threadIdx.x; c < a.c; c += blockDim.x) a.part[(long long)blockIdx.x * a.c + c] = sums[c];
    group_totals(a, [&](int c) { return sums[c]; }, own);
    if (a.shares > 1) cluster_sync();
    const float per_value = 1.0f / ((float)a.hw * (float)per_group);
    for (int g = threadIdx.x; g < a.groups; g += blockDim.x) {
        float2 t = make_float2(0.f, 0.f);
        for (int i = 0; i < a.shares; ++i) {
            float2 m;
            asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(m.x), "=f"(m.y) : "r"(peer_address(&own[g], (uint32_t)i)));
            t.x += m.x;
            t.y += m.y;
        }
        totals[g] = make_float2(t.x * per_value, t.y * per_value);
    }
    __syncthreads();
    if (a.shares > 1) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    write_gradients<T, V, kAct>(data, grad, pixels, first, a, lay, stats, totals);
    if (a.shares > 1) {
        __syncwarp();
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");       // the others have read this block's totals
    }
}

// ---- any maps ----------------------------------------------------------------------------------
// part[map][share][channel]: A and B of a run of pixels; runs[map][share][group]: its s1 and s2.
template <typename T, int V, int kAct>
__global__ void __launch_bounds__(512) group_sums_kernel(const __grid_constant__ GroupArgs a)
{
    extern __shared__ __align__(128) unsigned char smem[];
    float2 *const red = reinterpret_cast<float2 *>(smem), *const sums = red + blockDim.x * V, *const stats = sums + a.c;
    chain_next();
    chain_wait();
    const long long map = blockIdx.x / a.shares;
    const int p0 = (int)(blockIdx.x % a.shares) * a.share, pixels = max(0, min(a.share, a.hw - p0));
    for (int g = threadIdx.x; g < a.groups; g += blockDim.x) stats[g] = a.stats[map * a.groups + g];
    __syncthreads();
    const Lay lay(a.c / V);
    const long long at = (map * a.hw + p0) * a.c;
    block_sums<T, V, kAct>((const T *)a.x + at, (const T *)a.dy + at, pixels, a, lay, stats, red, sums);
    if (a.part)
        for (int c = threadIdx.x; c < a.c; c += blockDim.x) a.part[(long long)blockIdx.x * a.c + c] = sums[c];
    group_totals(a, [&](int c) { return sums[c]; }, a.runs + (long long)blockIdx.x * a.groups);
}

// sums[map][group] = (s1, s2) / m: a warp a group.
__global__ void __launch_bounds__(256) group_totals_kernel(const __grid_constant__ GroupArgs a)
{
    chain_next();
    chain_wait();
    const long long i = ((long long)blockIdx.x * 256 + threadIdx.x) / 32;
    const int lane = threadIdx.x & 31, per_group = a.c / a.groups;
    if (i >= a.n * a.groups) return;
    const long long map = i / a.groups;
    const int g = (int)(i - map * a.groups);
    float s1 = 0.f, s2 = 0.f;
    for (int k = lane; k < a.shares; k += 32) {
        const float2 s = a.runs[(map * a.shares + k) * a.groups + g];
        s1 += s.x;
        s2 += s.y;
    }
    for (int d = 16; d; d >>= 1) {
        s1 += __shfl_xor_sync(0xffffffffu, s1, d);
        s2 += __shfl_xor_sync(0xffffffffu, s2, d);
    }
    const float per_value = 1.0f / ((float)a.hw * (float)per_group);
    if (lane == 0) a.sums[i] = make_float2(s1 * per_value, s2 * per_value);
}

template <typename T, int V, int kAct>
__global__ void __launch_bounds__(512) group_gradients_kernel(const __grid_constant__ GroupArgs a)
{
    extern __shared__ __align__(128) unsigned char smem[];
    float2 *const stats = reinterpret_cast<float2 *>(smem), *const totals = stats + a.groups;
    chain_next();
    chain_wait();
    const long long block = (long long)gridDim.x - 1 - blockIdx.x, map = block / a.shares;
    const int p0 = (int)(block % a.shares) * a.share, pixels = max(0, min(a.share, a.hw - p0));
    for (int g = threadIdx.x; g < a.groups; g += blockDim.x) {
        stats[g] = a.stats[map * a.groups + g];
        totals[g] = a.sums[map * a.groups + g];
    }
    __syncthreads();
    const Lay lay(a.c / V);
    const long long first = map * a.hw + p0, at = first * a.c;
    write_gradients<T, V, kAct>((const T *)a.x + at, (const T *)a.dy + at, pixels, first, a, lay, stats, totals);
}

// db and dw: sums over the blocks' A and B, 8 channels a block, in 64 bits (there may be many).
constexpr int kVectorThreads = 512, kVectorChannels = 8;
__global__ void __launch_bounds__(kVectorThreads) group_vectors_kernel(const __grid_constant__ GroupArgs a, long long rows)
{
    chain_next();
    chain_wait();
    __shared__ double2 s_sum[kVectorThreads];
    const int c = blockIdx.x * kVectorChannels + (threadIdx.x & (kVectorChannels - 1));
    double2 s = make_double2(0.0, 0.0);
    if (c < a.c)
#pragma unroll 4
        for (long long r = threadIdx.x / kVectorChannels; r < rows; r += kVectorThreads / kVectorChannels) {
            const float2 t = a.part[r * a.c + c];
            s.x += t.x;
            s.y += t.y;
        }
    s_sum[threadIdx.x] = s;
    for (int d = kVectorThreads / 2; d >= kVectorChannels; d >>= 1) {
        __syncthreads();
        if (threadIdx.x < d) {
            s.x += s_sum[threadIdx.x + d].x;
            s.y += s_sum[threadIdx.x + d].y;
            s_sum[threadIdx.x] = s;
        }
    }
    if (threadIdx.x >= kVectorChannels || c >= a.c) return;
    if (a.dbias) a.dbias[c] = (float)s.x;
    if (a.dweight) a.dweight[c] = (float)s.y;
}

template <typename T, int V, int kAct>
tc_status launch_map(int device, const GroupArgs &a, int threads, size_t smem, cudaStream_t s)
{
    constexpr auto kernel = group_gradient_map_kernel<T, V, kAct>;
    if (!allow_shared<kernel>(device, 225 * 1024)) return TC_ERR_CUDA;
    return launch_first_cluster(a.shares, kernel, dim3((unsigned int)(a.n * a.shares)), dim3(threads), smem, s, a) == cudaSuccess ? TC_OK : TC_ERR_CUDA;
}
template <typename T, int V, int kAct>
tc_status launch_any(int device, const GroupArgs &a, int threads, cudaStream_t s)
{
    const size_t first = (size_t)threads * V * 8 + 8 * (size_t)a.c + 8 * (size_t)a.groups, last = 16 * (size_t)a.groups;
    if (!allow_shared<group_sums_kernel<T, V, kAct>>(device, 225 * 1024) || !allow_shared<group_gradients_kernel<T, V, kAct>>(device, 225 * 1024)) return TC_ERR_CUDA;
    const dim3 grid((unsigned int)(a.n * a.shares)), block(threads);
    if (launch_first(true, group_sums_kernel<T, V, kAct>, grid, block, first, s, a) != cudaSuccess) return TC_ERR_CUDA;
    if (launch_chained(true, group_totals_kernel, dim3((unsigned int)((a.n * a.groups + 7) / 8)), dim3(256), 0, s, a) != cudaSuccess) return TC_ERR_CUDA;
    return launch_chained(true, group_gradients_kernel<T, V, kAct>, grid, block, last, s, a) == cudaSuccess ? TC_OK : TC_ERR_CUDA;
}

template <typename T, int V>
tc_status launch(int device, const GroupArgs &a, int act, int threads, size_t smem, cudaStream_t s)
{
#define TC_GRADIENT(kAct) (smem ? launch_map<T, V, kAct>(device, a, threads, smem, s) : launch_any<T, V, kAct>(device, a, threads, s))
    return act == kRelu ? TC_GRADIENT(kRelu) : act == kSilu ? TC_GRADIENT(kSilu) : TC_GRADIENT(kNoAct);
#undef TC_GRADIENT
}

}  // namespace

GroupPlan tc_plan_group_norm_backward(const GroupGradArgs &m, int sm_count)
{
    GroupPlan p;
    const int element = m.dtype == TC_BF16 ? 2 : 4;
    const bool vectors = m.dweight || m.dbias;
    p.vector = m.c * element % 16 == 0 && m.aligned ? 16 / element : 1;
    p.threads = tc_group_threads(m.c / p.vector);
    GroupArgs a{};
    a.c = m.c;
    a.groups = m.groups;
    auto bytes = [&](int shares) { return shared_bytes(a, (m.hw + shares - 1) / shares, element, p.vector, p.threads); };
    if (p.vector > 1) {
        int shares = 1;
        while (shares < 8 && bytes(shares) > 110 * 1024) shares *= 2;
        while (shares < 8 && (long long)m.n * shares * 2 <= sm_count && m.hw / shares >= 16) shares *= 2;
        if (bytes(shares) <= 225 * 1024 && (long long)m.n * shares < 1ll << 31) {
            p.shares = shares;
            p.share = (m.hw + shares - 1) / shares;
            p.shared = bytes(shares);
            p.workspace = vectors ? (size_t)m.n * shares * m.c * sizeof(float2) : 0;
            return p;
        }
    }
    const long long row = (long long)m.c * element;
    long long share = std::max(1ll, 65536 / row);
    while (share > 1 && (long long)m.n * ((m.hw + share - 1) / share) < 4ll * sm_count) share = (share + 1) / 2;
    share = std::max(share, ((long long)m.hw * m.n + (1ll << 30) - 1) >> 30);
    p.share = (int)std::min<long long>(share, m.hw);
    p.shares = (m.hw + p.share - 1) / p.share;
    p.workspace = ((vectors ? (size_t)m.n * p.shares * m.c : 0) + (size_t)m.n * m.groups * (p.shares + 1)) * sizeof(float2);
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
            a.sums = (float2 *)workspace;
            a.runs = a.sums + (long long)a.n * a.groups;
            if (a.dweight || a.dbias) a.part = a.runs + (long long)a.n * a.shares * a.groups;
        } else if (p.workspace)
            a.part = (float2 *)workspace;
        if (m.dtype == TC_BF16) st = p.vector == 8 ? launch<__nv_bfloat16, 8>(device, a, m.act, p.threads, p.shared, s) : launch<__nv_bfloat16, 1>(device, a, m.act, p.threads, p.shared, s);
        else st = p.vector == 4 ? launch<float, 4>(device, a, m.act, p.threads, p.shared, s) : launch<float, 1>(device, a, m.act, p.threads, p.shared, s);
    }
    if (st != TC_OK || (!a.dweight && !a.dbias)) return st;
    const dim3 grid((unsigned int)((a.c + kVectorChannels - 1) / kVectorChannels));
    return launch_chained(m.n > 0, group_vectors_kernel, grid, dim3(kVectorThreads), 0, s, a, a.n * a.shares) == cudaSuccess ? TC_OK : TC_ERR_CUDA;
}
