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
#include "sm100_ptx.cuh"
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
        const float scale = scale_of(max_over<16>(max8(raw[i])));
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

// The tile comes by asynchronous copies and its values are read from shared memory where they are needed, twice for the layout across:
// with them in registers (96 a thread) two blocks fitted an SM, and a tile's memory time was hardly hidden (8192x4096, both layouts 38 us
// and 33; maps of 256x14x14 x 1024 56 and 41).
constexpr int kTileThreads = 256;
template <typename T, bool kMaps, bool kSquare>
__global__ void __launch_bounds__(kTileThreads, sizeof(T) == 2 ? 5 : 3) quantize_tile_kernel(const T *x, const __grid_constant__ TileArgs a, int vec)
{
    using namespace sm100;
    constexpr int kThreads = kTileThreads, kParts = kThreads / 64, kPart = kBlock / kParts;
    extern __shared__ __align__(16) unsigned char smem[];
    T(*tile)[kBlock] = reinterpret_cast<T(*)[kBlock]>(smem);                       // [outer][inner]
    __shared__ uint32_t s_max[kParts][kBlock];
    __shared__ uint32_t s_warp[kThreads / 32];
    chain_next();
    chain_wait();
    const long long outer_n = kMaps ? a.c : a.pixels, inner_n = kMaps ? a.pixels : a.c;
    const long long o0 = (long long)(kMaps ? blockIdx.y : blockIdx.x) * kBlock, i0 = (long long)(kMaps ? blockIdx.x : blockIdx.y) * kBlock;
    const int t = threadIdx.x;
    const int rows = (int)min((long long)kBlock, outer_n - o0), cols = (int)min((long long)kBlock, inner_n - i0);
    const long long pitch = kMaps ? a.hw : a.c;
    // Where inner value i lies in row 0 of the tile.
    auto inner_at = [&](long long i) {
        if (!kMaps) return o0 * pitch + i;
        const long long img = i / a.hw;
        return img * a.c * (long long)a.hw + (i - img * a.hw) + o0 * pitch;
    };
    // Values are moved `vec` at a time (inner_n and the maps' sides are multiples of it), zeros behind the tensor's end.
    if (vec >= 4) {
        constexpr int kCopy = 16 / (int)sizeof(T);                                 // eight values of fp32 go as two copies
        auto copy = [&](uint32_t dst, const T *src, bool ok) {
            if (vec * (int)sizeof(T) >= 16) cp_async_16(dst, src, ok ? 16u : 0u);
            else cp_async_8(dst, src, ok ? 8u : 0u);
        };
        const int step = vec < kCopy ? vec : kCopy, per_row = kBlock / step, k = t % per_row * step;
        const T *src = x + (k < cols ? inner_at(i0 + k) : 0);
        for (int r = t / per_row; r < kBlock; r += kThreads / per_row) {
            const bool ok = r < rows && k < cols;
            copy(smem_u32(&tile[r][k]), ok ? src + r * pitch : x, ok);
        }
    } else {
        const int k = t & (kBlock - 1);
        const T *src = x + (k < cols ? inner_at(i0 + k) : 0);
        constexpr int kRows = kThreads / kBlock;
        for (int r0 = t >> 7; r0 < kBlock; r0 += 16 * kRows) {
            T v[16];
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                v[j] = T(0.f);
                if (r0 + kRows * j < rows && k < cols) v[j] = src[(r0 + kRows * j) * pitch];
            }
#pragma unroll
            for (int j = 0; j < 16; ++j) tile[r0 + kRows * j][k] = v[j];
        }
    }
    cp_async_wait_all();
    __syncthreads();
    float scale = 0.f;
    if constexpr (kSquare) {
        uint32_t all = 0;
#pragma unroll
        for (int r = t >> 4; r < kBlock; r += kThreads / 16) all = max(all, max8(*reinterpret_cast<const Raw8<T> *>(&tile[r][(t & 15) * 8])));
        all = __reduce_max_sync(0xffffffffu, all);
        if ((t & 31) == 0) s_warp[t >> 5] = all;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kThreads / 32; ++w) all = max(all, s_warp[w]);
        scale = scale_of(all);
        if (t == 0) {
            if (a.along.codes) a.along.scales[i0 / kBlock * a.along.scale_ld + o0 / kBlock] = scale;
            if (a.across.codes) a.across.scales[o0 / kBlock * a.across.scale_ld + i0 / kBlock] = scale;
        }
    }
    if (a.along.codes) {
        const int k = (t & 15) * 8;
        uint8_t *to = a.along.codes + (o0 + (t >> 4)) * a.along.ld + i0 + k;
#pragma unroll 4
        for (int r = t >> 4; r < kBlock; r += kThreads / 16, to += kThreads / 16 * a.along.ld) {
            const Raw8<T> raw = *reinterpret_cast<const Raw8<T> *>(&tile[r][k]);
            float v[8];
            values8(raw, v);
            const float s = kSquare ? scale : scale_of(max_over<16>(max8(raw)));
            if (r < rows && k < cols) {
                *reinterpret_cast<uint2 *>(to) = codes8(v, __frcp_rn(s));
                if (!kSquare && k == 0) a.along.scales[i0 / kBlock * a.along.scale_ld + o0 + r] = s;
            }
        }
    }
    if (!a.across.codes) return;
    // two inner columns and kPart outer values a thread
    const int pair = t & 63, part = t >> 6;
    auto two = [&](int r, float &v0, float &v1) {
        if constexpr (sizeof(T) == 2) {
            const uint32_t w = *reinterpret_cast<const uint32_t *>(&tile[part * kPart + r][pair * 2]);
            v0 = __uint_as_float(w << 16);
            v1 = __uint_as_float(w & 0xffff0000u);
        } else {
            const float2 w = *reinterpret_cast<const float2 *>(&tile[part * kPart + r][pair * 2]);
            v0 = w.x;
            v1 = w.y;
        }
    };
    float scale0 = scale, scale1 = scale;
    if constexpr (!kSquare) {
        uint32_t m0 = 0, m1 = 0;
#pragma unroll 8
        for (int r = 0; r < kPart; ++r) {
            if constexpr (sizeof(T) == 2) m0 = max_pairs(m0, *reinterpret_cast<const uint32_t *>(&tile[part * kPart + r][pair * 2]));
            else {
                float v0, v1;
                two(r, v0, v1);
                m0 = max(m0, abs_bits(v0));
                m1 = max(m1, abs_bits(v1));
            }
        }
        if constexpr (sizeof(T) == 2) {                       // both columns' in one word
            m1 = m0 & 0xffff0000u;
            m0 <<= 16;
        }
        s_max[part][2 * pair] = m0;
        s_max[part][2 * pair + 1] = m1;
        __syncthreads();
#pragma unroll
        for (int q = 0; q < kParts; ++q) { m0 = max(m0, s_max[q][2 * pair]); m1 = max(m1, s_max[q][2 * pair + 1]); }
        scale0 = scale_of(m0);
        scale1 = scale_of(m1);
    }
    const float inv0 = __frcp_rn(scale0), inv1 = __frcp_rn(scale1);
    const int c = 2 * pair;
    uint8_t *const to = a.across.codes + (i0 + c) * a.across.ld + o0 + part * kPart;
#pragma unroll
    for (int q = 0; q < kPart / 16; ++q) {
        uint32_t w0[4], w1[4];
#pragma unroll
        for (int h = 0; h < 4; ++h) {
            float v0[4], v1[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) two(16 * q + 4 * h + j, v0[j], v1[j]);
            w0[h] = codes4(v0[0], v0[1], v0[2], v0[3], inv0);
            w1[h] = codes4(v1[0], v1[1], v1[2], v1[3], inv1);
        }
        if (part * kPart + 16 * q >= rows) break;                                     // rows of codes end at a multiple of 16
        if (c < cols) *reinterpret_cast<uint4 *>(to + 16 * q) = make_uint4(w0[0], w0[1], w0[2], w0[3]);
        if (c + 1 < cols) *reinterpret_cast<uint4 *>(to + a.across.ld + 16 * q) = make_uint4(w1[0], w1[1], w1[2], w1[3]);
    }
    if (!kSquare && part == 0) {
        if (c < cols) a.across.scales[o0 / kBlock * a.across.scale_ld + i0 + c] = scale0;
        if (c + 1 < cols) a.across.scales[o0 / kBlock * a.across.scale_ld + i0 + c + 1] = scale1;
    }
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
tc_status launch_tiles(int device, const T *x, int n, int c, int hw, bool square, const BlockMatrix &pixels, const BlockMatrix &channels, cudaStream_t s)
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
    auto launch = [&](bool allowed, auto kernel) {
        return allowed && launch_first(true, kernel, grid, dim3(kTileThreads), smem, s, x, a, vec) == cudaSuccess ? TC_OK : TC_ERR_CUDA;
    };
#define TC_TILES(maps, squares) launch(allow_shared<quantize_tile_kernel<T, maps, squares>>(device, smem), quantize_tile_kernel<T, maps, squares>)
    if (hw > 1) return square ? TC_TILES(true, true) : TC_TILES(true, false);
    return square ? TC_TILES(false, true) : TC_TILES(false, false);
#undef TC_TILES
}

template <typename T>
tc_status quantize(int device, const T *x, int n, int c, int hw, bool square, const BlockMatrix &pixels, const BlockMatrix &channels, cudaStream_t s)
{
    if (!square && !channels.codes && hw == 1) return launch_rows(x, n, c, pixels, s);
    if (!square && !pixels.codes && n == 1) return launch_rows(x, c, hw, channels, s);
    return launch_tiles(device, x, n, c, hw, square, pixels, channels, s);
}

}  // namespace

tc_status tc_launch_quantize_blocks(int device, const void *x, int dtype, int n, int c, int hw, bool square, const BlockMatrix &pixels, const BlockMatrix &channels,
                                    cudaStream_t s)
{
    return dtype == TC_BF16 ? quantize(device, (const __nv_bfloat16 *)x, n, c, hw, square, pixels, channels, s)
                            : quantize(device, (const float *)x, n, c, hw, square, pixels, channels, s);
}
