// tc_gradient_norm, tc_clip_gradients: of a list of tensors, all together,
//
//   norm = sqrt(sum x^2),   out = x f,   f = min(1, max_norm / norm)
//
// Bound by the bytes moved: the list is read for the norm and, because f is known only then, read again and written; where it is not clipped in
// place it is read once.  The list's addresses are kernel parameters (no copy ahead of the kernel, and captured with it).  Tensors are cut
// into rows of 8 KB (16 bytes a thread), of which every block has its share, neighbours in the list: it looks a tensor up once and works on up to four rows at a time.  62 tensors
// of together 47 MB: 27.5 us, of which 14.5 are what a copy needs for the bytes and the rest two launches and the blocks' sums that lie between; 290 of 1.9 GB: 930 us
// (5.9 TB/s with the second read).
//
// A thread's squares of those rows, 16 or 32 of them, are summed in fp32 (four sums of four or eight, each addition rounded to 2^-24) where that neither overflows nor drops what is
// small, else in fp64; everything else is summed in fp64, in an order that the list's sizes, its alignments and the number of SMs decide.
#include "block_codes.cuh"
#include "tc_internal.h"

namespace {

using namespace tcdev;
using namespace blk;

constexpr int kThreads = 512, kInFlight = 4, kVector = 16, kRow = kThreads * kVector, kBlocksPerSm = 2;
constexpr float kLeast = 8.673617379884035e-19f;              // 2^-60: squares that fp32 loses are 2^-66 of this

template <int kMost>
struct List {
    const void *in[kMost];
    void *out[kMost];
    long long count[kMost];           // of values; bf16: -1 minus it
    int first[kMost + 1];             // row of a tensor's first byte, counted from 16-byte boundaries of the input; behind the last one all rows
    int tensors;
};

// A block's rows, tensor by tensor: work(tensor, first row in it, rows), up to kInFlight rows at a time.
template <int kMost, typename F>
__device__ __forceinline__ void for_rows(const List<kMost> &l, unsigned int block, F work)
{
    const long long rows = l.first[l.tensors];
    int row = (int)(rows * block / gridDim.x);
    const int end = (int)(rows * (block + 1) / gridDim.x);
    int t = 0, hi = l.tensors;
    while (hi - t > 1) {
        const int mid = (t + hi) >> 1;
        if (l.first[mid] <= row) t = mid;
        else hi = mid;
    }
    while (row < end) {
        while (row >= l.first[t + 1]) ++t;
        const int count = min(kInFlight, min(end, l.first[t + 1]) - row);
        work(t, row - l.first[t], count);
        row += count;
    }
}
struct Piece {
    long long at, count;              // first value of the thread's first vector (it may lie before the tensor), the tensor's values
    int rows;
    bool inside;                      // no vector of these rows reaches out of the tensor
};
template <typename T>
__device__ __forceinline__ Piece piece_of(const void *in, long long count, int row, int rows)
{
    constexpr int kPer = kVector / (int)sizeof(T);
    const int before = (int)(((uintptr_t)in & (kVector - 1)) / sizeof(T));
    const long long first = (long long)row * (kRow / (int)sizeof(T)) - before;
    return {first + threadIdx.x * kPer, count, rows, first >= 0 && first + (long long)kInFlight * (kRow / (int)sizeof(T)) <= count && rows == kInFlight};
}
// Vector i of the thread; zeros outside the tensor and behind the piece's rows.
template <typename T>
__device__ __forceinline__ uint4 load_vector(const T *in, const Piece &p, int i)
{
    constexpr int kPer = kVector / (int)sizeof(T);
    const long long at = p.at + (long long)i * kThreads * kPer;
    if (i < p.rows && at >= 0 && at + kPer <= p.count) return *reinterpret_cast<const uint4 *>(in + at);
    uint32_t w[4] = {};
    if (i < p.rows && at + kPer > 0 && at < p.count) {
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            if (at + j < 0 || at + j >= p.count) continue;
            if constexpr (sizeof(T) == 4) w[j] = __float_as_uint(in[at + j]);
            else w[j / 2] |= (uint32_t)reinterpret_cast<const unsigned short *>(in)[at + j] << (16 * (j & 1));
        }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
template <typename T>
__device__ __forceinline__ void load_vectors(const T *in, const Piece &p, uint4 (&r)[kInFlight])
{
    if (p.inside) {
        const uint4 *const at = reinterpret_cast<const uint4 *>(in + p.at);
#pragma unroll
        for (int i = 0; i < kInFlight; ++i) r[i] = at[i * kThreads];
    } else
#pragma unroll
        for (int i = 0; i < kInFlight; ++i) r[i] = load_vector(in, p, i);
}
template <typename T>
__device__ __forceinline__ void vector_values(const uint4 &r, float (&f)[kVector / sizeof(T)])
{
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if constexpr (sizeof(T) == 4) f[j] = __uint_as_float(w[j]);
        else {
            f[2 * j] = __uint_as_float(w[j] << 16);
            f[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
        }
    }
}

template <typename T>
__device__ __forceinline__ double squares_of(const void *in, long long count, int row, int rows)
{
    constexpr int kPer = kVector / (int)sizeof(T);
    const Piece p = piece_of<T>(in, count, row, rows);
    uint4 r[kInFlight];
    load_vectors((const T *)in, p, r);
    float s[4] = {};
#pragma unroll
    for (int i = 0; i < kInFlight; ++i) {
        float f[kPer];
        vector_values<T>(r[i], f);
#pragma unroll
        for (int j = 0; j < kPer; ++j) s[j & 3] = fmaf(f[j], f[j], s[j & 3]);
    }
    const float sum = (s[0] + s[1]) + (s[2] + s[3]);
    if (sum >= kLeast && sum < __int_as_float(0x7f800000)) return (double)sum;
    double d = 0.0;
#pragma unroll
    for (int i = 0; i < kInFlight; ++i) {
        float f[kPer];
        vector_values<T>(r[i], f);
#pragma unroll
        for (int j = 0; j < kPer; ++j)
            if (f[j] != 0.f) d = fma((double)f[j], (double)f[j], d);
    }
    return d;
}

// Sum over the block's threads, in all of them.
__device__ __forceinline__ double block_sum(double v, double *s_sum)
{
    for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    if ((threadIdx.x & 31) == 0) s_sum[threadIdx.x / 32] = v;
    __syncthreads();
    v = 0.0;
    for (int w = 0; w < kThreads / 32; ++w) v += s_sum[w];
    return v;
}

template <int kMost>
__global__ void __launch_bounds__(kThreads, kBlocksPerSm) squares_kernel(const __grid_constant__ List<kMost> l, double *partial)
{
    chain_next();
    chain_wait();
    __shared__ double s_sum[kThreads / 32];
    double sum = 0.0;
    for_rows(l, blockIdx.x, [&](int t, int row, int rows) {
        const long long n = l.count[t];
        sum += n < 0 ? squares_of<__nv_bfloat16>(l.in[t], -1 - n, row, rows) : squares_of<float>(l.in[t], n, row, rows);
    });
    sum = block_sum(sum, s_sum);
    if (threadIdx.x == 0) partial[blockIdx.x] = sum;
}

// The norm from the blocks' sums, the same in every block.
__device__ __forceinline__ float norm_of(const double *partial, int parts, double *s_sum)
{
    double sum = 0.0;
    for (int i = threadIdx.x; i < parts; i += kThreads) sum += partial[i];
    return (float)sqrt(block_sum(sum, s_sum));
}

__global__ void __launch_bounds__(kThreads) norm_kernel(const double *partial, int parts, float *norm)
{
    chain_next();
    chain_wait();
    __shared__ double s_sum[kThreads / 32];
    const float n = norm_of(partial, parts, s_sum);
    if (threadIdx.x == 0) *norm = n;
}

template <typename T>
__device__ __forceinline__ void scale_rows(const void *in, void *out, long long count, int row, int rows, float factor)
{
    constexpr int kPer = kVector / (int)sizeof(T);
    const Piece p = piece_of<T>(in, count, row, rows);
    const bool vectors = (((uintptr_t)in ^ (uintptr_t)out) & (kVector - 1)) == 0;
    uint4 r[kInFlight];
    load_vectors((const T *)in, p, r);
#pragma unroll
    for (int i = 0; i < kInFlight; ++i) {
        if (i >= rows) break;
        const long long at = p.at + (long long)i * kThreads * kPer;
        float f[kPer];
        vector_values<T>(r[i], f);
        if (factor != 1.f)                                    // (values that stay keep their bits, a NaN's too)
#pragma unroll
            for (int j = 0; j < kPer; ++j) f[j] *= factor;
        uint4 w = r[i];
        if (factor != 1.f) {
            if constexpr (sizeof(T) == 4) w = make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
            else w = make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
        }
        if (vectors && (p.inside || (at >= 0 && at + kPer <= p.count))) *reinterpret_cast<uint4 *>((T *)out + at) = w;
        else if (at + kPer > 0 && at < p.count) {
            const uint32_t words[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int j = 0; j < kPer; ++j) {
                if (at + j < 0 || at + j >= p.count) continue;
                if constexpr (sizeof(T) == 4) reinterpret_cast<uint32_t *>(out)[at + j] = words[j];
                else reinterpret_cast<unsigned short *>(out)[at + j] = (unsigned short)(words[j / 2] >> (16 * (j & 1)));
            }
        }
    }
}

template <int kMost>
__global__ void __launch_bounds__(kThreads, kBlocksPerSm) scale_kernel(const __grid_constant__ List<kMost> l, const double *partial, int parts, float max_norm, float *norm)
{
    chain_next();
    chain_wait();
    __shared__ double s_sum[kThreads / 32];
    const float n = norm_of(partial, parts, s_sum);
    if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = n;
    // (a norm that is not finite leaves the values as they are)
    const float factor = n > max_norm && n < __int_as_float(0x7f800000) ? __fdiv_rn(max_norm, n) : 1.f;
    // (the last ones first: they are the likeliest to be in L2 still)
    for_rows(l, gridDim.x - 1 - blockIdx.x, [&](int t, int row, int rows) {
        if (factor == 1.f && l.in[t] == l.out[t]) return;
        const long long count = l.count[t];
        if (count < 0) scale_rows<__nv_bfloat16>(l.in[t], l.out[t], -1 - count, row, rows, factor);
        else scale_rows<float>(l.in[t], l.out[t], count, row, rows, factor);
    });
}

// Tensors of one launch: as few addresses as a list needs, up to 28 KB of them.
constexpr int kListSizes[] = {32, 128, 512, 1024};
constexpr int kMostTensors = 1024;

long long rows_of(const tc_gradient &g)
{
    const size_t size = g.dtype == TC_BF16 ? 2 : 4;
    return ((long long)((uintptr_t)g.data & (kVector - 1)) + g.count * (long long)size + kRow - 1) / kRow;
}

template <int kMost>
void fill(List<kMost> &l, const tc_gradient *g, int n)
{
    int row = 0, used = 0;
    for (int i = 0; i < n; ++i) {
        if (g[i].count == 0) continue;
        l.in[used] = g[i].data;
        l.out[used] = g[i].out;
        l.count[used] = g[i].dtype == TC_BF16 ? -1 - g[i].count : g[i].count;
        l.first[used++] = row;
        row += (int)rows_of(g[i]);
    }
    l.first[used] = row;
    l.tensors = used;
}

template <int kMost>
tc_status launch_list(const tc_gradient *g, int n, bool scale, bool first, int blocks, double *partial, int parts, float max_norm, float *norm, cudaStream_t s)
{
    List<kMost> l;
    fill(l, g, n);
    const dim3 grid((unsigned int)std::max(1, std::min(blocks, l.first[l.tensors])));
    const cudaError_t err = scale ? launch_chained(true, scale_kernel<kMost>, grid, dim3(kThreads), 0, s, l, partial, parts, max_norm, norm)
                            : first ? launch_first(true, squares_kernel<kMost>, grid, dim3(kThreads), 0, s, l, partial)
                                    : launch_chained(true, squares_kernel<kMost>, grid, dim3(kThreads), 0, s, l, partial);
    return err == cudaSuccess ? TC_OK : TC_ERR_CUDA;
}
template <typename... A>
tc_status launch(const tc_gradient *g, int n, A... args)
{
    if (n <= kListSizes[0]) return launch_list<kListSizes[0]>(g, n, args...);
    if (n <= kListSizes[1]) return launch_list<kListSizes[1]>(g, n, args...);
    if (n <= kListSizes[2]) return launch_list<kListSizes[2]>(g, n, args...);
    return launch_list<kListSizes[3]>(g, n, args...);
}

// Blocks of a launch.
int blocks_of(const tc_gradient *g, int n, int sm_count)
{
    long long rows = 0;
    for (int i = 0; i < n; ++i)
        if (g[i].count) rows += rows_of(g[i]);
    return (int)std::max(1ll, std::min<long long>(rows, (long long)sm_count * kBlocksPerSm));
}

}  // namespace

size_t tc_gradient_norm_workspace(int tensors, int sm_count)
{
    return (size_t)std::max(1, (tensors + kMostTensors - 1) / kMostTensors) * sm_count * kBlocksPerSm * sizeof(double);
}

tc_status tc_launch_clip_gradients(const tc_gradient *list, int n, bool clip, float max_norm, float *norm, int sm_count, void *workspace, cudaStream_t s)
{
    double *const partial = (double *)workspace;
    int parts = 0;
    for (int first = 0; first == 0 || first < n; first += kMostTensors) {
        const int count = std::min(n - first, kMostTensors), blocks = blocks_of(list + first, count, sm_count);
        const tc_status st = launch(list + first, count, false, first == 0, blocks, partial + parts, 0, 0.f, (float *)nullptr, s);
        if (st != TC_OK) return st;
        parts += blocks;
    }
    if (!clip) return launch_chained(true, norm_kernel, dim3(1), dim3(kThreads), 0, s, partial, parts, norm) == cudaSuccess ? TC_OK : TC_ERR_CUDA;
    for (int first = 0; first == 0 || first < n; first += kMostTensors) {
        const int count = std::min(n - first, kMostTensors);
        const tc_status st = launch(list + first, count, true, false, blocks_of(list + first, count, sm_count), partial, parts, max_norm, first == 0 ? norm : nullptr, s);
        if (st != TC_OK) return st;
    }
    return TC_OK;
}
