// tc_quantize_blocks: e4m3 codes of a tensor with a scale for each block of 128 values (or tile of 128 x 128), by
// pixels (a row for each, along its channels) and by channels (a row for each, along the pixels).
//
//   a = max |x| over the block (2^-100 at least), scale = a / 448, code = nearest e4m3 value of x / scale
//
// Bound by the bytes moved: the tensor once, a byte per value and layout, 4 bytes per block.  Rows that lie one after
// the other in memory take a kernel that keeps a block in 16 lanes; everything else -- the layout that runs across
// memory, both layouts, tiles -- one that turns a tile of 128 x 128 values in shared memory, so that the tensor
// is read once for both.
#include "block_codes.cuh"
#include "tc_internal.h"

namespace {

using namespace tcdev;
using namespace blk;

// ---- rows as they lie in memory ----------------------------------------------------------
// 16 lanes a block, eight values each; a thread has kInFlight blocks' loads in flight.
constexpr int kInFlight = 4, kRowThreads = 256, kRowItems = kRowThreads / 16 * kInFlight;

template <typename T, bool kVec>
__global__ void __launch_bounds__(kRowThreads) quantize_rows_kernel(const T *x, uint32_t items, uint32_t k_blocks, int cols, BlockMatrix out)
{
    chain_next();
    chain_wait();
    const int lane16 = threadIdx.x & 15, k_lane = lane16 * 8;
    const uint32_t first = blockIdx.x * kRowItems + threadIdx.x / 16;
    Raw8<T> raw[kInFlight];
    uint32_t row[kInFlight], kb[kInFlight];
#pragma unroll
    for (int i = 0; i < kInFlight; ++i) {
        const uint32_t item = first + i * (kRowThreads / 16);
        row[i] = item / k_blocks;
        kb[i] = item - row[i] * k_blocks;
        const int k = (int)kb[i] * kBlock + k_lane;
        const T *src = x + (long long)row[i] * cols + k;
        zero8(raw[i]);
        if (item < items && k < cols) {
            if constexpr (kVec) load8(raw[i], src);
            else load8(raw[i], src, min(8, cols - k));
        }
    }
#pragma unroll
    for (int i = 0; i < kInFlight; ++i) {
        float v[8];
        values8(raw[i], v);
        uint32_t m = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) m = max(m, abs_bits(v[j]));
        const float scale = scale_of(max16(m));
        if (first + i * (kRowThreads / 16) >= items) continue;
        const int k = (int)kb[i] * kBlock + k_lane;
        if (k < cols) *reinterpret_cast<uint2 *>(out.codes + (long long)row[i] * out.ld + k) = codes8(v, __frcp_rn(scale));
        if (lane16 == 0) out.scales[(long long)kb[i] * out.scale_ld + row[i]] = scale;
    }
}

// ---- tiles of 128 x 128, turned in shared memory -----------------------------------------------
// `inner` is the index that is contiguous in memory (the channel of single pixels, else the pixel), `outer` the other.
struct TileArgs {
    long long pixels;
    int c, hw;
    BlockMatrix along, across;      // rows = outer (blocks along memory), rows = inner; codes null where not wanted
};

template <typename T, bool kMaps, bool kSquare>
__global__ void __launch_bounds__(256) quantize_tile_kernel(const T *x, TileArgs a, int vec)
{
    extern __shared__ __align__(16) unsigned char smem[];
    T(*tile)[kBlock] = reinterpret_cast<T(*)[kBlock]>(smem);                       // [outer][inner]
    __shared__ uint32_t s_max[4][kBlock];
    __shared__ uint32_t s_warp[8];
    chain_next();
    chain_wait();
    const long long outer_n = kMaps ? a.c : a.pixels, inner_n = kMaps ? a.pixels : a.c;
    const long long o0 = (long long)(kMaps ? blockIdx.y : blockIdx.x) * kBlock, i0 = (long long)(kMaps ? blockIdx.x : blockIdx.y) * kBlock;
    const int t = threadIdx.x, chunk = t & 15, row0 = t >> 4;
    // A thread's eight inner values are the same ones in each of its eight rows: where they lie is found once.
    long long off[8];
    int valid = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const long long i = i0 + chunk * 8 + j;
        if (i < inner_n) valid = j + 1;
        off[j] = i;
        if (kMaps) {
            if (j == 0 || vec < 8) {
                const long long img = i / a.hw;
                off[j] = img * a.c * (long long)a.hw + (i - img * a.hw);
            } else
                off[j] = off[0] + j;
        }
    }
    const long long pitch = kMaps ? a.hw : a.c;
    Raw8<T> raw[8];
#pragma unroll
    for (int r = 0; r < 8; ++r) {
        const long long o = o0 + row0 + 16 * r;
        zero8(raw[r]);
        if (o >= outer_n || valid == 0) continue;
        const T *src = x + o * pitch;
        if (vec == 8) load8(raw[r], src + off[0]);                                 // inner_n and the maps' sides are multiples of eight
        else if (vec == 4) {
            if constexpr (sizeof(T) == 2) {
                const uint2 p = *reinterpret_cast<const uint2 *>(src + off[0]);
                const uint2 q = valid > 4 ? *reinterpret_cast<const uint2 *>(src + off[4]) : make_uint2(0, 0);
                raw[r].v = make_uint4(p.x, p.y, q.x, q.y);
            } else {
                raw[r].v = *reinterpret_cast<const uint4 *>(src + off[0]);
                if (valid > 4) raw[r].w = *reinterpret_cast<const uint4 *>(src + off[4]);
            }
        } else {
            T *dst = reinterpret_cast<T *>(&raw[r]);
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (j < valid) dst[j] = src[off[j]];
        }
    }
    uint32_t m[8];
#pragma unroll
    for (int r = 0; r < 8; ++r) {
        *reinterpret_cast<Raw8<T> *>(&tile[row0 + 16 * r][chunk * 8]) = raw[r];
        float v[8];
        values8(raw[r], v);
        m[r] = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) m[r] = max(m[r], abs_bits(v[j]));
        m[r] = max16(m[r]);
    }
    float scale = 0.f;
    if constexpr (kSquare) {
        uint32_t all = 0;
#pragma unroll
        for (int r = 0; r < 8; ++r) all = max(all, m[r]);
        all = max(all, __shfl_xor_sync(0xffffffffu, all, 16));
        if ((t & 31) == 0) s_warp[t >> 5] = all;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < 8; ++w) all = max(all, s_warp[w]);
        scale = scale_of(all);
        if (t == 0) {
            if (a.along.codes) a.along.scales[i0 / kBlock * a.along.scale_ld + o0 / kBlock] = scale;
            if (a.across.codes) a.across.scales[o0 / kBlock * a.across.scale_ld + i0 / kBlock] = scale;
        }
    }
    if (a.along.codes && valid > 0) {
#pragma unroll
        for (int r = 0; r < 8; ++r) {
            const long long o = o0 + row0 + 16 * r;
            if (o >= outer_n) continue;
            const float s = kSquare ? scale : scale_of(m[r]);
            float v[8];
            values8(raw[r], v);
            *reinterpret_cast<uint2 *>(a.along.codes + o * a.along.ld + i0 + chunk * 8) = codes8(v, __frcp_rn(s));
            if (!kSquare && chunk == 0) a.along.scales[i0 / kBlock * a.along.scale_ld + o] = s;
        }
    }
    if (!a.across.codes) return;
    if (!kSquare) __syncthreads();                                                 // the tile (a square's maximum has waited for it)
    // two inner columns and 32 outer values a thread
    const int pair = t & 63, part = t >> 6;
    float v0[32], v1[32];
    uint32_t m0 = 0, m1 = 0;
#pragma unroll
    for (int r = 0; r < 32; ++r) {
        if constexpr (sizeof(T) == 2) {
            const uint32_t w = *reinterpret_cast<const uint32_t *>(&tile[part * 32 + r][pair * 2]);
            v0[r] = __uint_as_float(w << 16);
            v1[r] = __uint_as_float(w & 0xffff0000u);
        } else {
            const float2 w = *reinterpret_cast<const float2 *>(&tile[part * 32 + r][pair * 2]);
            v0[r] = w.x;
            v1[r] = w.y;
        }
        if (!kSquare) { m0 = max(m0, abs_bits(v0[r])); m1 = max(m1, abs_bits(v1[r])); }
    }
    float scale0 = scale, scale1 = scale;
    if constexpr (!kSquare) {
        s_max[part][2 * pair] = m0;
        s_max[part][2 * pair + 1] = m1;
        __syncthreads();
#pragma unroll
        for (int q = 0; q < 4; ++q) { m0 = max(m0, s_max[q][2 * pair]); m1 = max(m1, s_max[q][2 * pair + 1]); }
        scale0 = scale_of(m0);
        scale1 = scale_of(m1);
    }
    const long long o_first = o0 + part * 32;
    if (o_first >= outer_n) return;
    auto put = [&](long long i, const float (&v)[32], float s) {
        if (i >= inner_n) return;
        const float inv = __frcp_rn(s);
        uint8_t *dst = a.across.codes + i * a.across.ld + o_first;
#pragma unroll
        for (int q = 0; q < 2; ++q)
            if (o_first + 16 * q < outer_n)                                        // rows of codes end at a multiple of 16
                *reinterpret_cast<uint4 *>(dst + 16 * q) =
                    make_uint4(codes4(v[16 * q], v[16 * q + 1], v[16 * q + 2], v[16 * q + 3], inv), codes4(v[16 * q + 4], v[16 * q + 5], v[16 * q + 6], v[16 * q + 7], inv),
                               codes4(v[16 * q + 8], v[16 * q + 9], v[16 * q + 10], v[16 * q + 11], inv), codes4(v[16 * q + 12], v[16 * q + 13], v[16 * q + 14], v[16 * q + 15], inv));
        if (!kSquare && part == 0) a.across.scales[o0 / kBlock * a.across.scale_ld + i] = s;
    };
    put(i0 + 2 * pair, v0, scale0);
    put(i0 + 2 * pair + 1, v1, scale1);
}

template <typename T>
tc_status launch_rows(const T *x, long long rows, int cols, const BlockMatrix &out, cudaStream_t s)
{
    const uint32_t k_blocks = (uint32_t)((cols + kBlock - 1) / kBlock);
    const long long items = rows * k_blocks;
    const bool vec = cols % 8 == 0 && ((uintptr_t)x & 15u) == 0;
    const dim3 grid((unsigned int)((items + kRowItems - 1) / kRowItems));
    return launch_first(true, vec ? quantize_rows_kernel<T, true> : quantize_rows_kernel<T, false>, grid, dim3(kRowThreads), 0, s, x, (uint32_t)items, k_blocks,
                        cols, out) == cudaSuccess ? TC_OK : TC_ERR_CUDA;
}

template <typename T>
tc_status launch_tiles(const T *x, int n, int c, int hw, bool square, const BlockMatrix &pixels, const BlockMatrix &channels, cudaStream_t s)
{
    TileArgs a;
    a.pixels = (long long)n * hw;
    a.c = c;
    a.hw = hw;
    a.along = hw > 1 ? channels : pixels;
    a.across = hw > 1 ? pixels : channels;
    const long long inner = hw > 1 ? (n > 1 ? hw : a.pixels) : c;                  // consecutive values in memory
    const uintptr_t at = (uintptr_t)x;
    const int vec = inner % 8 == 0 && at % 16 == 0 ? 8 : inner % 4 == 0 && at % (4 * sizeof(T)) == 0 ? 4 : 1;
    const dim3 grid((unsigned int)((a.pixels + kBlock - 1) / kBlock), (unsigned int)((c + kBlock - 1) / kBlock));
    constexpr size_t smem = kBlock * kBlock * sizeof(T);
    auto launch = [&](auto kernel) {
        if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess) { cudaGetLastError(); return TC_ERR_CUDA; }
        return launch_first(true, kernel, grid, dim3(256), smem, s, x, a, vec) == cudaSuccess ? TC_OK : TC_ERR_CUDA;
    };
    if (hw > 1) return square ? launch(quantize_tile_kernel<T, true, true>) : launch(quantize_tile_kernel<T, true, false>);
    return square ? launch(quantize_tile_kernel<T, false, true>) : launch(quantize_tile_kernel<T, false, false>);
}

template <typename T>
tc_status quantize(const T *x, int n, int c, int hw, bool square, const BlockMatrix &pixels, const BlockMatrix &channels, cudaStream_t s)
{
    if (!square && !channels.codes && hw == 1) return launch_rows(x, n, c, pixels, s);
    if (!square && !pixels.codes && n == 1) return launch_rows(x, c, hw, channels, s);
    return launch_tiles(x, n, c, hw, square, pixels, channels, s);
}

}  // namespace

tc_status tc_launch_quantize_blocks(const void *x, int dtype, int n, int c, int hw, bool square, const BlockMatrix &pixels, const BlockMatrix &channels,
                                    cudaStream_t s)
{
    return dtype == TC_BF16 ? quantize((const __nv_bfloat16 *)x, n, c, hw, square, pixels, channels, s)
                            : quantize((const float *)x, n, c, hw, square, pixels, channels, s);
}
