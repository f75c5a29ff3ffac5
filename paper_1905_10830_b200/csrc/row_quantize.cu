// tc_quantize_rows: 8-bit integer codes of a tensor with one scale for each row, a row being a pixel's channels or a channel's pixels.
//
//   a = max |x| over the row (2^-100 at least), scale = fl(a / 127), code = the integer nearest to x / scale, ties to even
//
// Bound by the bytes moved: the tensor once, a byte per value and layout.  Rows that lie one after the other in memory are held in registers
// between the maximum and the codes.  Otherwise the maxima come first, tile by tile of 128 x 128 with atomic maxima (whose order does not
// matter), and the codes from the tiles turned in shared memory.
#include "integer_codes.cuh"
#include "sm100_ptx.cuh"
#include "tc_internal.h"

namespace {

using namespace tcdev;
using namespace rowcodes;

constexpr int kTile = 128;

// ---- rows as they lie in memory ----------------------------------------------------------
// kThreads a row, eight values each, kPer times; kThreads = 32: eight rows a block.  Rows that do not fit are read twice.
constexpr int kRowThreads = 256;
template <int kThreads> constexpr int kRowsOfBlock = kThreads < kRowThreads ? kRowThreads / kThreads : 1;

template <int kThreads>
__device__ __forceinline__ uint32_t row_max(uint32_t m, uint32_t *s_max)
{
    m = __reduce_max_sync(0xffffffffu, m);
    if constexpr (kThreads > 32) {
        constexpr int kWarps = kThreads / 32;
        const int warp = threadIdx.x / 32, first = warp / kWarps * kWarps;
        if ((threadIdx.x & 31) == 0) s_max[warp] = m;
        __syncthreads();
        m = 0;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) m = max(m, s_max[first + w]);
    }
    return m;
}

template <typename T, int kThreads, int kPer, bool kVec>
__global__ void __launch_bounds__(kThreads < kRowThreads ? kRowThreads : kThreads) rows_in_registers_kernel(const T *x, long long rows, int cols, RowMatrix out)
{
    chain_next();
    chain_wait();
    __shared__ uint32_t s_max[32];
    const int lane = threadIdx.x % kThreads;
    const long long row = (long long)blockIdx.x * kRowsOfBlock<kThreads> + threadIdx.x / kThreads;
    const T *const src = x + row * cols;
    Raw8<T> raw[kPer];
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int k = (i * kThreads + lane) * 8;
        zero8(raw[i]);
        if (row < rows && k < cols) {
            if constexpr (kVec) load8(raw[i], src + k);
            else load8(raw[i], src + k, min(8, cols - k));
        }
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) m = max(m, max8(raw[i]));
    const Coder c(row_scale(row_max<kThreads>(m, s_max)));
    if (row >= rows) return;
    if (lane == 0) out.scales[row] = c.scale;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int k = (i * kThreads + lane) * 8;
        float v[8];
        values8(raw[i], v);
        if (k < cols) *reinterpret_cast<uint2 *>(out.codes + row * out.ld + k) = codes_of8(v, c);
    }
}

// Longer rows: a block each, read twice.
template <typename T, bool kVec>
__global__ void __launch_bounds__(1024) long_rows_kernel(const T *x, int cols, RowMatrix out)
{
    chain_next();
    chain_wait();
    __shared__ uint32_t s_max[32];
    const long long row = blockIdx.x;
    const T *const src = x + row * cols;
    auto load = [&](Raw8<T> &raw, long long k) {
        if constexpr (kVec) load8(raw, src + k);
        else load8(raw, src + k, (int)min(8ll, cols - k));
    };
    uint32_t m = 0;
    for (long long k = threadIdx.x * 8ll; k < cols; k += 8 * 1024) {
        Raw8<T> raw;
        load(raw, k);
        m = max(m, max8(raw));
    }
    const Coder c(row_scale(row_max<1024>(m, s_max)));
    if (threadIdx.x == 0) out.scales[row] = c.scale;
    for (long long k = threadIdx.x * 8ll; k < cols; k += 8 * 1024) {
        Raw8<T> raw;
        load(raw, k);
        float v[8];
        values8(raw, v);
        *reinterpret_cast<uint2 *>(out.codes + row * out.ld + k) = codes_of8(v, c);
    }
}

// ---- tiles of 128 x 128 in shared memory -----------------------------------------------
// `inner` is the index that is contiguous in memory (the channel of single pixels, else the pixel), `outer` the other.
struct TileArgs {
    long long pixels;
    int c, hw;
    RowMatrix along, across;          // rows = outer (values along memory), rows = inner; codes null where not wanted
    uint32_t *max_along, *max_across; // their maxima, [outer] and [inner]
};
constexpr int kTileThreads = 256;

template <typename T, bool kMaps, bool kMaxima>
__global__ void __launch_bounds__(kTileThreads, sizeof(T) == 2 ? 5 : 3) row_tile_kernel(const T *x, const __grid_constant__ TileArgs a, int vec)
{
    using namespace sm100;
    constexpr int kThreads = kTileThreads, kParts = kThreads / 64, kPart = kTile / kParts;
    extern __shared__ __align__(16) unsigned char smem[];
    T(*tile)[kTile] = reinterpret_cast<T(*)[kTile]>(smem);                         // [outer][inner]
    __shared__ uint32_t s_max[kParts][kTile];
    chain_next();
    chain_wait();
    const long long outer_n = kMaps ? a.c : a.pixels, inner_n = kMaps ? a.pixels : a.c;
    const long long o0 = (long long)(kMaps ? blockIdx.y : blockIdx.x) * kTile, i0 = (long long)(kMaps ? blockIdx.x : blockIdx.y) * kTile;
    const int t = threadIdx.x;
    const int rows = (int)min((long long)kTile, outer_n - o0), cols = (int)min((long long)kTile, inner_n - i0);
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
        const int step = vec < kCopy ? vec : kCopy, per_row = kTile / step, k = t % per_row * step;
        const T *src = x + (k < cols ? inner_at(i0 + k) : 0);
        for (int r = t / per_row; r < kTile; r += kThreads / per_row) {
            const bool ok = r < rows && k < cols;
            copy(smem_u32(&tile[r][k]), ok ? src + r * pitch : x, ok);
        }
    } else {
        const int k = t & (kTile - 1);
        const T *src = x + (k < cols ? inner_at(i0 + k) : 0);
        constexpr int kRows = kThreads / kTile;
        for (int r0 = t >> 7; r0 < kTile; r0 += 16 * kRows) {
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
    if (a.along.codes) {
        const int k = (t & 15) * 8;
        for (int r = t >> 4; r < kTile; r += kThreads / 16) {
            const Raw8<T> raw = *reinterpret_cast<const Raw8<T> *>(&tile[r][k]);
            if constexpr (kMaxima) {
                const uint32_t m = max_over<16>(max8(raw));
                if (r < rows && k == 0) atomicMax(&a.max_along[o0 + r], m);
            } else if (r < rows && k < cols) {
                float v[8];
                values8(raw, v);
                const Coder c(row_scale(a.max_along[o0 + r]));
                *reinterpret_cast<uint2 *>(a.along.codes + (o0 + r) * a.along.ld + i0 + k) = codes_of8(v, c);
                if (i0 == 0 && k == 0) a.along.scales[o0 + r] = c.scale;
            }
        }
    }
    if (!a.across.codes) return;
    // two inner columns and kPart outer values a thread
    const int pair = t & 63, part = t >> 6, c = 2 * pair;
    auto two = [&](int r, float &v0, float &v1) {
        if constexpr (sizeof(T) == 2) {
            const uint32_t w = *reinterpret_cast<const uint32_t *>(&tile[part * kPart + r][c]);
            v0 = __uint_as_float(w << 16);
            v1 = __uint_as_float(w & 0xffff0000u);
        } else {
            const float2 w = *reinterpret_cast<const float2 *>(&tile[part * kPart + r][c]);
            v0 = w.x;
            v1 = w.y;
        }
    };
    if constexpr (kMaxima) {
        uint32_t m0 = 0, m1 = 0;
#pragma unroll 8
        for (int r = 0; r < kPart; ++r) {
            if constexpr (sizeof(T) == 2) m0 = max_pairs(m0, *reinterpret_cast<const uint32_t *>(&tile[part * kPart + r][c]));
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
        s_max[part][c] = m0;
        s_max[part][c + 1] = m1;
        __syncthreads();
        if (t < cols) {
            uint32_t m = 0;
#pragma unroll
            for (int q = 0; q < kParts; ++q) m = max(m, s_max[q][t]);
            atomicMax(&a.max_across[i0 + t], m);
        }
    } else {
        const Coder c0(row_scale(c < cols ? a.max_across[i0 + c] : 0u)), c1(row_scale(c + 1 < cols ? a.max_across[i0 + c + 1] : 0u));
        uint8_t *const to = a.across.codes + (i0 + c) * a.across.ld + o0 + part * kPart;
#pragma unroll
        for (int q = 0; q < kPart / 16; ++q) {
            uint32_t w0[4], w1[4];
#pragma unroll
            for (int h = 0; h < 4; ++h) {
                float v0[4], v1[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) two(16 * q + 4 * h + j, v0[j], v1[j]);
                w0[h] = codes_of4(v0, c0);
                w1[h] = codes_of4(v1, c1);
            }
            if (part * kPart + 16 * q >= rows) break;                                 // rows of codes end at a multiple of 16
            if (c < cols) *reinterpret_cast<uint4 *>(to + 16 * q) = make_uint4(w0[0], w0[1], w0[2], w0[3]);
            if (c + 1 < cols) *reinterpret_cast<uint4 *>(to + a.across.ld + 16 * q) = make_uint4(w1[0], w1[1], w1[2], w1[3]);
        }
        if (o0 == 0 && part == 0) {
            if (c < cols) a.across.scales[i0 + c] = c0.scale;
            if (c + 1 < cols) a.across.scales[i0 + c + 1] = c1.scale;
        }
    }
}

template <typename T>
tc_status launch_rows(const T *x, long long rows, int cols, const RowMatrix &out, cudaStream_t s)
{
    const bool vec = cols % 8 == 0 && ((uintptr_t)x & 15u) == 0;
    auto go = [&](auto kernel, int threads, int rows_of_block) {
        return launch_first(true, kernel, dim3((unsigned int)((rows + rows_of_block - 1) / rows_of_block)), dim3(threads), 0, s, x, rows, cols, out) == cudaSuccess ? TC_OK : TC_ERR_CUDA;
    };
#define TC_ROWS(threads, per) \
    go(vec ? rows_in_registers_kernel<T, threads, per, true> : rows_in_registers_kernel<T, threads, per, false>, threads < kRowThreads ? kRowThreads : threads, kRowsOfBlock<threads>)
    if (cols <= 256) return TC_ROWS(32, 1);
    if (cols <= 512) return TC_ROWS(32, 2);
    if (cols <= 1024) return TC_ROWS(32, 4);
    if (cols <= 2048) return TC_ROWS(256, 1);
    if (cols <= 4096) return TC_ROWS(256, 2);
    if (cols <= 8192) return TC_ROWS(512, 2);
    if (cols <= 16384) return TC_ROWS(512, 4);
#undef TC_ROWS
    return launch_first(true, vec ? long_rows_kernel<T, true> : long_rows_kernel<T, false>, dim3((unsigned int)rows), dim3(1024), 0, s, x, cols, out) == cudaSuccess ? TC_OK : TC_ERR_CUDA;
}

template <typename T>
tc_status launch_tiles(int device, const T *x, const TileArgs &a, int n, size_t max_bytes, cudaStream_t s)
{
    const long long inner = a.hw > 1 ? (n > 1 ? a.hw : a.pixels) : a.c;            // consecutive values in memory
    const uintptr_t at = (uintptr_t)x;
    const int vec = inner % 8 == 0 && at % 16 == 0 ? 8 : inner % 4 == 0 && at % (4 * sizeof(T)) == 0 ? 4 : 1;
    const dim3 grid((unsigned int)((a.pixels + kTile - 1) / kTile), (unsigned int)((a.c + kTile - 1) / kTile));
    constexpr size_t smem = kTile * kTile * sizeof(T);
    if (cudaMemsetAsync(a.max_along ? a.max_along : a.max_across, 0, max_bytes, s) != cudaSuccess) { cudaGetLastError(); return TC_ERR_CUDA; }
    auto launch = [&](bool allowed, bool early, auto kernel) {
        return allowed && launch_chained(early, kernel, grid, dim3(kTileThreads), smem, s, x, a, vec) == cudaSuccess ? TC_OK : TC_ERR_CUDA;
    };
#define TC_TILES(maps, maxima) launch(allow_shared<row_tile_kernel<T, maps, maxima>>(device, smem), !(maxima), row_tile_kernel<T, maps, maxima>)
    tc_status st = a.hw > 1 ? TC_TILES(true, true) : TC_TILES(false, true);
    if (st == TC_OK) st = a.hw > 1 ? TC_TILES(true, false) : TC_TILES(false, false);
#undef TC_TILES
    return st;
}

bool in_memory(const RowQuantizeArgs &a, bool channels) { return channels ? a.hw > 1 && a.n == 1 : a.hw == 1; }

template <typename T>
tc_status quantize(int device, const RowQuantizeArgs &a, uint32_t *workspace, cudaStream_t s)
{
    const long long pixels = (long long)a.n * a.hw;
    RowMatrix left[2] = {a.pixels, a.channels};
    for (int i = 0; i < 2; ++i)
        if (left[i].codes && in_memory(a, i)) {
            const tc_status st = i ? launch_rows((const T *)a.x, a.c, (int)pixels, left[i], s) : launch_rows((const T *)a.x, pixels, a.c, left[i], s);
            if (st != TC_OK) return st;
            left[i] = RowMatrix{};
        }
    if (!left[0].codes && !left[1].codes) return TC_OK;
    TileArgs t{};
    t.pixels = pixels;
    t.c = a.c;
    t.hw = a.hw;
    t.along = a.hw > 1 ? left[1] : left[0];
    t.across = a.hw > 1 ? left[0] : left[1];
    const long long outer = a.hw > 1 ? a.c : pixels;
    if (t.along.codes) t.max_along = workspace;
    if (t.across.codes) t.max_across = workspace + (t.along.codes ? outer : 0);
    return launch_tiles(device, (const T *)a.x, t, a.n, tc_quantize_rows_workspace(a), s);
}

}  // namespace

size_t tc_quantize_rows_workspace(const RowQuantizeArgs &a)
{
    size_t words = 0;
    if (a.pixels.codes && !in_memory(a, false)) words += (size_t)a.n * a.hw;
    if (a.channels.codes && !in_memory(a, true)) words += (size_t)a.c;
    return words * sizeof(uint32_t);
}

tc_status tc_launch_quantize_rows(int device, const RowQuantizeArgs &a, void *workspace, cudaStream_t s)
{
    return a.dtype == TC_BF16 ? quantize<__nv_bfloat16>(device, a, (uint32_t *)workspace, s) : quantize<float>(device, a, (uint32_t *)workspace, s);
}
