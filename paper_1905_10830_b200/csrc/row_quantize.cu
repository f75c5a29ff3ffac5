// tc_quantize_rows: 8-bit integer codes of a tensor with one scale for each row, a row being a pixel's channels or a channel's pixels.
//
//   a = max |x| over the row (2^-100 at least), scale = fl(a / 127), code = the integer nearest to x / scale, ties to even
//
// Bound by the bytes moved: the tensor once, a byte per value and layout.  Rows that lie one after the other in memory are held in registers
// between the maximum and the codes; where both layouts of such a matrix are wanted, the same kernel keeps the maxima of its rows' columns.  Pixels of maps come with
// all their channels to shared memory.  Otherwise the maxima come first: of parts of the rows, which a small kernel joins to scales; and then the codes, from
// tiles of 128 x 128 that are turned in shared memory and found in L2.
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
        m = __reduce_max_sync(0xffffffffu, s_max[first + (threadIdx.x & (kWarps - 1))]);
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

// The same with the maxima of the columns over the block's rows, [block][cols]: where the codes by columns are wanted too.  The next row is on its way while one is
// worked on.
template <typename T, int kThreads, int kPer>
__global__ void __launch_bounds__(kThreads) rows_and_columns_kernel(const T *x, long long rows, int cols, RowMatrix out, uint32_t *partial)
{
    chain_next();
    chain_wait();
    __shared__ uint32_t s_max[2][32];
    const int lane = threadIdx.x;
    Raw8<T> raw[kPer], next[kPer];
    uint32_t most[kPer][8];
#pragma unroll
    for (int i = 0; i < kPer; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) most[i][j] = 0;
    auto load = [&](Raw8<T> (&r)[kPer], long long row) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int k = (i * kThreads + lane) * 8;
            zero8(r[i]);
            if (row < rows && k < cols) load8(r[i], x + row * cols + k);
        }
    };
    load(next, blockIdx.x);
    int turn = 0;
    for (long long row = blockIdx.x; row < rows; row += gridDim.x, turn ^= 1) {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < kPer; ++i) raw[i] = next[i];
        load(next, row + gridDim.x);
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            m = max(m, max8(raw[i]));
            if constexpr (sizeof(T) == 2) {                   // two columns' maxima in a word
                const uint32_t w[4] = {raw[i].v.x, raw[i].v.y, raw[i].v.z, raw[i].v.w};
#pragma unroll
                for (int j = 0; j < 4; ++j) most[i][j] = max_pairs(most[i][j], w[j]);
            } else {
                float v[8];
                values8(raw[i], v);
#pragma unroll
                for (int j = 0; j < 8; ++j) most[i][j] = max(most[i][j], abs_bits(v[j]));
            }
        }
        const Coder c(row_scale(row_max<kThreads>(m, s_max[turn])));
        if (lane == 0) out.scales[row] = c.scale;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int k = (i * kThreads + lane) * 8;
            float v[8];
            values8(raw[i], v);
            if (k < cols) *reinterpret_cast<uint2 *>(out.codes + row * out.ld + k) = codes_of8(v, c);
        }
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int k = (i * kThreads + lane) * 8;
        if (k >= cols) continue;
        uint4 *const to = reinterpret_cast<uint4 *>(partial + (long long)blockIdx.x * cols + k);
        if constexpr (sizeof(T) == 2) {
            to[0] = make_uint4(most[i][0] << 16, most[i][0] & 0xffff0000u, most[i][1] << 16, most[i][1] & 0xffff0000u);
            to[1] = make_uint4(most[i][2] << 16, most[i][2] & 0xffff0000u, most[i][3] << 16, most[i][3] & 0xffff0000u);
        } else {
            to[0] = make_uint4(most[i][0], most[i][1], most[i][2], most[i][3]);
            to[1] = make_uint4(most[i][4], most[i][5], most[i][6], most[i][7]);
        }
    }
}

// ---- maxima of rows that do not lie one after the other in memory ---------------------------------
// A matrix [outer][inner]: `inner` is the index that is contiguous in memory (the channel of single pixels, else the pixel), `outer` the other.
struct MatrixArgs {
    long long pixels;
    int c, hw;
    RowMatrix along, across;          // rows = outer (values along memory), rows = inner; codes null where not wanted
};
template <bool kMaps>
__device__ __forceinline__ long long place_of(const MatrixArgs &a, long long outer, long long inner)
{
    if (!kMaps) return outer * a.c + inner;
    const long long img = inner / a.hw;
    return (img * a.c + outer) * a.hw + (inner - img * a.hw);
}

// Of columns (across): partial[chunk][inner], kVec neighbouring columns a lane, 64 lanes, four rows of them a block.
template <typename T, bool kMaps, int kVec>
__global__ void __launch_bounds__(256) column_maxima_kernel(const T *x, const __grid_constant__ MatrixArgs a, long long outer_of_chunk, uint32_t *partial)
{
    chain_next();
    chain_wait();
    __shared__ uint32_t s_max[3][kVec][64];
    const long long outer_n = kMaps ? a.c : a.pixels, inner_n = kMaps ? a.pixels : a.c;
    const long long inner = ((long long)blockIdx.x * 64 + (threadIdx.x & 63)) * kVec, first = blockIdx.y * outer_of_chunk, end = min(first + outer_of_chunk, outer_n);
    const int group = threadIdx.x >> 6;
    uint32_t most[kVec] = {};
    if (inner < inner_n) {
        const T *p = x + place_of<kMaps>(a, first + group, inner);
        const long long pitch = 4ll * (kMaps ? a.hw : a.c);
#pragma unroll 8
        for (long long o = first + group; o < end; o += 4, p += pitch) {
            if constexpr (kVec == 8) {
                Raw8<T> r;
                load8(r, p);
                float v[8];
                values8(r, v);
#pragma unroll
                for (int j = 0; j < 8; ++j) most[j] = max(most[j], abs_bits(v[j]));
            } else
                most[0] = max(most[0], abs_bits(load1(p)));
        }
    }
    if (group)
#pragma unroll
        for (int j = 0; j < kVec; ++j) s_max[group - 1][j][threadIdx.x & 63] = most[j];
    __syncthreads();
    if (group || inner >= inner_n) return;
#pragma unroll
    for (int j = 0; j < kVec; ++j) {
#pragma unroll
        for (int g = 0; g < 3; ++g) most[j] = max(most[j], s_max[g][j][threadIdx.x]);
        partial[(long long)blockIdx.y * inner_n + inner + j] = most[j];
    }
}

// Of channels of maps (along): partial[chunk][channel], a block a channel and a chunk of images.
template <typename T, int kVec>
__global__ void __launch_bounds__(256) channel_maxima_kernel(const T *x, const __grid_constant__ MatrixArgs a, int images_of_chunk, uint32_t *partial)
{
    chain_next();
    chain_wait();
    __shared__ uint32_t s_max[32];
    const int c = blockIdx.x, per = a.hw / kVec, together = max(1, 256 / per);      // images at a time
    const long long images = a.pixels / a.hw, first = (long long)blockIdx.y * images_of_chunk, end = min(first + images_of_chunk, images);
    const int mine = per < 256 ? threadIdx.x / per : 0, k0 = per < 256 ? threadIdx.x - mine * per : threadIdx.x;
    uint32_t most = 0;
    if (mine < together)
        for (int k = k0; k < per; k += 256) {
            const T *p = x + ((first + mine) * a.c + c) * (long long)a.hw + k * kVec;
            const long long step = (long long)together * a.c * a.hw;
#pragma unroll 4
            for (long long img = first + mine; img < end; img += together, p += step) {
                if constexpr (kVec == 8) {
                    Raw8<T> r;
                    load8(r, p);
                    most = max(most, max8(r));
                } else if constexpr (kVec == 4) {
                    if constexpr (sizeof(T) == 2) {
                        const uint2 w = *reinterpret_cast<const uint2 *>(p);
                        most = max(most, max_of_pair(max_pairs(w.x & 0x7fff7fffu, w.y)));
                    } else {
                        const float4 w = *reinterpret_cast<const float4 *>(p);
                        most = max(most, max(max(abs_bits(w.x), abs_bits(w.y)), max(abs_bits(w.z), abs_bits(w.w))));
                    }
                } else
                    most = max(most, abs_bits(load1(p)));
            }
        }
    most = row_max<256>(most, s_max);
    if (threadIdx.x == 0) partial[(long long)blockIdx.y * a.c + c] = most;
}

// Scales from the parts' maxima: 32 rows a block, 32 lanes of parts each.
__global__ void __launch_bounds__(1024) join_maxima_kernel(const uint32_t *partial, int parts, long long rows, float *scales)
{
    chain_next();
    chain_wait();
    __shared__ uint32_t s_max[32][33];
    const long long row = blockIdx.x * 32ll + (threadIdx.x & 31);
    uint32_t most = 0;
    if (row < rows)
#pragma unroll 8
        for (int p = threadIdx.x >> 5; p < parts; p += 32) most = max(most, partial[p * rows + row]);
    s_max[threadIdx.x >> 5][threadIdx.x & 31] = most;
    __syncthreads();
    most = __reduce_max_sync(0xffffffffu, s_max[threadIdx.x & 31][threadIdx.x >> 5]);
    const long long mine = blockIdx.x * 32ll + (threadIdx.x >> 5);
    if ((threadIdx.x & 31) == 0 && mine < rows) scales[mine] = row_scale(most);
}

// ---- codes from tiles of 128 x 128 in shared memory ---------------------------------------------
constexpr int kTileThreads = 256;

template <typename T, bool kMaps>
__global__ void __launch_bounds__(kTileThreads, sizeof(T) == 2 ? 5 : 3) row_tile_kernel(const T *x, const __grid_constant__ MatrixArgs a, int vec)
{
    using namespace sm100;
    constexpr int kThreads = kTileThreads, kParts = kThreads / 64, kPart = kTile / kParts;
    extern __shared__ __align__(16) unsigned char smem[];
    T(*tile)[kTile] = reinterpret_cast<T(*)[kTile]>(smem);                         // [outer][inner]
    chain_next();
    chain_wait();
    const long long outer_n = kMaps ? a.c : a.pixels, inner_n = kMaps ? a.pixels : a.c;
    const long long o0 = (long long)(kMaps ? blockIdx.y : blockIdx.x) * kTile, i0 = (long long)(kMaps ? blockIdx.x : blockIdx.y) * kTile;
    const int t = threadIdx.x;
    const int rows = (int)min((long long)kTile, outer_n - o0), cols = (int)min((long long)kTile, inner_n - i0);
    const long long pitch = kMaps ? a.hw : a.c;
    // Values are moved `vec` at a time (inner_n and the maps' sides are multiples of it), zeros behind the tensor's end.
    if (vec >= 4) {
        constexpr int kCopy = 16 / (int)sizeof(T);                                 // eight values of fp32 go as two copies
        auto copy = [&](uint32_t dst, const T *src, bool ok) {
            if (vec * (int)sizeof(T) >= 16) cp_async_16(dst, src, ok ? 16u : 0u);
            else cp_async_8(dst, src, ok ? 8u : 0u);
        };
        const int step = vec < kCopy ? vec : kCopy, per_row = kTile / step, k = t % per_row * step;
        const T *src = x + (k < cols ? place_of<kMaps>(a, o0, i0 + k) : 0);
        for (int r = t / per_row; r < kTile; r += kThreads / per_row) {
            const bool ok = r < rows && k < cols;
            copy(smem_u32(&tile[r][k]), ok ? src + r * pitch : x, ok);
        }
    } else {
        const int k = t & (kTile - 1);
        const T *src = x + (k < cols ? place_of<kMaps>(a, o0, i0 + k) : 0);
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
        if (k < cols)
            for (int r = t >> 4; r < rows; r += kThreads / 16) {
                float v[8];
                values8(*reinterpret_cast<const Raw8<T> *>(&tile[r][k]), v);
                *reinterpret_cast<uint2 *>(a.along.codes + (o0 + r) * a.along.ld + i0 + k) = codes_of8(v, Coder(a.along.scales[o0 + r]));
            }
    }
    if (!a.across.codes) return;
    // two inner columns and kPart outer values a thread
    const int part = t >> 6, c = 2 * (t & 63);
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
    const Coder c0(c < cols ? a.across.scales[i0 + c] : 1.f), c1(c + 1 < cols ? a.across.scales[i0 + c + 1] : 1.f);
    uint8_t *const to = a.across.codes + (i0 + c) * a.across.ld + o0 + part * kPart;
#pragma unroll
    for (int q = 0; q < kPart / 16; ++q) {
        if (part * kPart + 16 * q >= rows) break;                                     // rows of codes end at a multiple of 16
        uint2 w0[2], w1[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            float v0[8], v1[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) two(16 * q + 8 * h + j, v0[j], v1[j]);
            w0[h] = codes_of8(v0, c0);
            w1[h] = codes_of8(v1, c1);
        }
        if (c < cols) *reinterpret_cast<uint4 *>(to + 16 * q) = make_uint4(w0[0].x, w0[0].y, w0[1].x, w0[1].y);
        if (c + 1 < cols) *reinterpret_cast<uint4 *>(to + a.across.ld + 16 * q) = make_uint4(w1[0].x, w1[0].y, w1[1].x, w1[1].y);
    }
}

// ---- pixels of maps with all their channels in shared memory -------------------------------------
// A block has one image, contiguous in memory (bulk copies), or `strip` neighbouring pixels of one (16-byte copies): [c][width] values.  A thread finds the maximum of a
// pixel, or two neighbours, over part of the channels, then codes 16 channels of it at a time.
struct StripArgs {
    int c, hw, width, strips;         // pixels of a block, blocks of an image (1: the whole)
    RowMatrix out;
    unsigned int *status;
};
constexpr int kStripThreads = 512;                            // of a block that has an image; of strips half (64 of 128x56x56 bf16: 36 us, 57 with all)
constexpr size_t kMostStrip = kMostShared - 4096;             // (static variables beside it)
template <typename T, int kTogether>
__global__ void __launch_bounds__(kStripThreads) pixel_strip_kernel(const T *x, const __grid_constant__ StripArgs a)
{
    using namespace sm100;
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ __align__(8) unsigned long long s_full;
    __shared__ uint32_t s_max[2][kStripThreads];
    const int threads = blockDim.x;
    T *const values = reinterpret_cast<T *>(smem);
    float *const scales = reinterpret_cast<float *>(smem + ((size_t)a.c * a.width * sizeof(T) + 15) / 16 * 16);
    if (threadIdx.x == 0) { mbar_init(smem_u32(&s_full), 1); mbar_fence_init(); }
    __syncthreads();
    chain_next();
    chain_wait();
    const long long img = blockIdx.x / (unsigned int)a.strips;
    const int p0 = (int)(blockIdx.x - (unsigned int)img * a.strips) * a.width, pixels = min(a.width, a.hw - p0);
    const T *const src = x + img * a.c * a.hw + p0;
    if (a.strips == 1) {
        if (threadIdx.x == 0) {
            const uint32_t bytes = (uint32_t)a.c * a.hw * sizeof(T);
            mbar_arrive_expect_tx(smem_u32(&s_full), bytes);
            for (uint32_t at = 0; at < bytes; at += 16384) bulk_load(smem_u32(smem) + at, (const char *)src + at, min(16384u, bytes - at), smem_u32(&s_full));
        }
        // (a wait that runs out is reported; the codes are wrong then, nothing else)
        if (!mbar_try_wait(smem_u32(&s_full), 0, 1000u) && !mbar_wait_soon(smem_u32(&s_full), 0) && !mbar_wait_soon(smem_u32(&s_full), 0)) tc_dev_set_status(a.status, TC_ERR_TIMEOUT);
    } else {
        constexpr int kPer = 16 / (int)sizeof(T);
        const int per_row = a.width / kPer, k = (int)(threadIdx.x % per_row) * kPer;
        if (threadIdx.x < threads / per_row * per_row)
            for (int c = threadIdx.x / per_row; c < a.c; c += threads / per_row)
                cp_async_16(smem_u32(values + c * a.width + k), k < pixels ? src + (long long)c * a.hw + k : x, k < pixels ? 16u : 0u);
        cp_async_wait_all();
        __syncthreads();
    }
    // maxima: `parts` threads kTogether neighbouring pixels
    auto two = [&](int c, int p, float &v0, float &v1) {
        if constexpr (kTogether == 1) v0 = load1(values + c * a.width + p);
        else if constexpr (sizeof(T) == 2) {
            const uint32_t w = *reinterpret_cast<const uint32_t *>(values + c * a.width + p);
            v0 = __uint_as_float(w << 16);
            v1 = __uint_as_float(w & 0xffff0000u);
        } else {
            const float2 w = *reinterpret_cast<const float2 *>(values + c * a.width + p);
            v0 = w.x;
            v1 = w.y;
        }
    };
    const int columns = a.width / kTogether, parts = max(1, threads / columns);
    for (int base = 0; base < columns; base += threads) {
        const int part = parts > 1 ? threadIdx.x / columns : 0, q = base + (parts > 1 ? threadIdx.x - part * columns : threadIdx.x), p = q * kTogether;
        uint32_t m0 = 0, m1 = 0;
        if (q < columns && part < parts) {
#pragma unroll 8
            for (int c = part; c < a.c; c += parts) {
                if constexpr (kTogether == 2 && sizeof(T) == 2) m0 = max_pairs(m0, *reinterpret_cast<const uint32_t *>(values + c * a.width + p));
                else {
                    float v0, v1 = 0.f;
                    two(c, p, v0, v1);
                    m0 = max(m0, abs_bits(v0));
                    m1 = max(m1, abs_bits(v1));
                }
            }
            if constexpr (kTogether == 2 && sizeof(T) == 2) {
                m1 = m0 & 0xffff0000u;
                m0 <<= 16;
            }
        }
        if (parts > 1) {
            s_max[0][threadIdx.x] = m0;
            s_max[1][threadIdx.x] = m1;
            __syncthreads();
            if (part == 0)
                for (int r = 1; r < parts; ++r) {
                    m0 = max(m0, s_max[0][r * columns + q]);
                    m1 = max(m1, s_max[1][r * columns + q]);
                }
        }
        if (part == 0 && q < columns)
#pragma unroll
            for (int k = 0; k < kTogether; ++k) {
                const float scale = row_scale(k ? m1 : m0);
                scales[p + k] = scale;
                if (p + k < pixels) a.out.scales[img * a.hw + p0 + p + k] = scale;
            }
    }
    __syncthreads();
    const int pieces = (a.c + 15) / 16;
    int piece = threadIdx.x / columns, q = threadIdx.x - piece * columns;
    const int more_pieces = threads / columns, more = threads - more_pieces * columns;
    for (; piece < pieces; piece += more_pieces, q += more) {
        if (q >= columns) {
            q -= columns;
            if (++piece >= pieces) break;
        }
        const int p = q * kTogether;
        if (p >= pixels) continue;
        const Coder c0(scales[p]), c1(scales[p + kTogether - 1]);
        uint2 w0[2], w1[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            float v0[8], v1[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int c = 16 * piece + 8 * h + j;
                v0[j] = v1[j] = 0.f;
                if (c < a.c) two(c, p, v0[j], v1[j]);
            }
            w0[h] = codes_of8(v0, c0);
            if constexpr (kTogether == 2) w1[h] = codes_of8(v1, c1);
        }
        uint8_t *const to = a.out.codes + (img * a.hw + p0 + p) * a.out.ld + 16 * piece;
        *reinterpret_cast<uint4 *>(to) = make_uint4(w0[0].x, w0[0].y, w0[1].x, w0[1].y);
        if constexpr (kTogether == 2)
            if (p + 1 < pixels) *reinterpret_cast<uint4 *>(to + a.out.ld) = make_uint4(w1[0].x, w1[0].y, w1[1].x, w1[1].y);
    }
}

// ---- launches --------------------------------------------------------------------------------------
template <typename T>
bool rows_aligned(const T *x, int cols) { return cols % 8 == 0 && ((uintptr_t)x & 15u) == 0; }

template <typename T>
tc_status launch_rows(const T *x, long long rows, int cols, const RowMatrix &out, cudaStream_t s)
{
    const bool vec = rows_aligned(x, cols);
    auto go = [&](auto kernel, int threads, int rows_of_block) {
        return launch_first(true, kernel, dim3((unsigned int)((rows + rows_of_block - 1) / rows_of_block)), dim3(threads), 0, s, x, rows, cols, out) == cudaSuccess ? TC_OK : TC_ERR_CUDA;
    };
#define TC_ROWS(threads, per) \
    go(vec ? rows_in_registers_kernel<T, threads, per, true> : rows_in_registers_kernel<T, threads, per, false>, threads < kRowThreads ? kRowThreads : threads, kRowsOfBlock<threads>)
    if (cols <= 256) return TC_ROWS(32, 1);
    if (cols <= 512) return TC_ROWS(32, 2);
    if (cols <= 1024) return TC_ROWS(32, 4);
    // (a row's maximum and scale are work of every warp: few warps, but for few rows, whose latency is their threads')
    const bool few = rows < 592;
    if (cols <= 2048) return few ? TC_ROWS(256, 1) : TC_ROWS(128, 2);
    if (cols <= 4096) return few ? TC_ROWS(512, 1) : TC_ROWS(128, 4);
    if (cols <= 8192) return few ? TC_ROWS(512, 2) : TC_ROWS(256, 4);
    if (cols <= 16384) return TC_ROWS(512, 4);
#undef TC_ROWS
    return launch_first(true, vec ? long_rows_kernel<T, true> : long_rows_kernel<T, false>, dim3((unsigned int)rows), dim3(1024), 0, s, x, cols, out) == cudaSuccess ? TC_OK : TC_ERR_CUDA;
}

bool in_memory(const RowQuantizeArgs &a, bool channels) { return channels ? a.hw > 1 && a.n == 1 : a.hw == 1; }

// Whether the rows that lie in memory and the columns go through one kernel, and its blocks.
// (Rows of 1024 and fewer leave most of its threads idle: 32768x512 bf16 66 us, in three passes 39; 32768x1024 82 and 65.  1280 to 4096: 30.3 to 31.6 at 8192x1280, 58 to 67 at 8192x4096,
// in fp32 26.4 to 31.4 and 70 to 82.  Longer ones would want 512 threads or four vectors each: 4096x5120 45 to 46.5, fp32 47.5 to 50, 4096x8192 61 to 65.5, less than a kernel more is worth.
// Three tensors in turn.)
bool rows_with_columns(const RowQuantizeArgs &a)
{
    return a.hw == 1 && a.pixels.codes && a.channels.codes && a.c % 8 == 0 && ((uintptr_t)a.x & 15u) == 0 && a.c > 1024 && a.c <= 4096;
}
int rows_blocks(const RowQuantizeArgs &a, int sm_count) { return (int)std::min<long long>(a.n, 4ll * sm_count); }

// Parts of the maxima of the columns (rows = the inner index), or of the channels of maps.
int parts_across(const RowQuantizeArgs &a, int vec, int sm_count)
{
    const long long outer = a.hw > 1 ? a.c : (long long)a.n, inner = a.hw > 1 ? (long long)a.n * a.hw : a.c, strips = (inner + 64 * vec - 1) / (64 * vec);
    return (int)std::max(1ll, std::min((outer + 31) / 32, std::max(1ll, 4ll * sm_count / strips)));
}
int parts_along(const RowQuantizeArgs &a, int sm_count) { return (int)std::max(1ll, std::min<long long>({a.n, 1024, 8ll * sm_count / a.c})); }
// Consecutive values in memory, and how many are moved at a time.
int vector_of(const RowQuantizeArgs &a)
{
    const long long inner = a.hw > 1 ? (a.n > 1 ? a.hw : (long long)a.n * a.hw) : a.c;
    const uintptr_t at = (uintptr_t)a.x;
    const size_t size = a.dtype == TC_BF16 ? 2 : 4;
    return inner % 8 == 0 && at % 16 == 0 ? 8 : inner % 4 == 0 && at % (4 * size) == 0 ? 4 : 1;
}

// Dynamic shared memory of pixel_strip_kernel: the values and a scale for each pixel.
size_t strip_bytes(int c, int width, size_t size) { return ((size_t)c * width * size + 15) / 16 * 16 + width * sizeof(float); }
// Pixels of a block of pixel_strip_kernel, 0: it does not take the maps.
int strip_of(const RowQuantizeArgs &a)
{
    const size_t size = a.dtype == TC_BF16 ? 2 : 4, at = (uintptr_t)a.x;
    if (a.hw <= 1 || at % 16) return 0;
    const size_t image = (size_t)a.c * a.hw * size;
    // (maps of few channels have as many bytes of scales as of values: they count too.  A block an SM is better than strips all the same: 16x56x56 x 128 bf16 13 us, in strips of 64 35)
    if (image <= kTwoBlocks - 4096 && image % 16 == 0 && strip_bytes(a.c, a.hw, size) <= kMostStrip) return a.hw;
    if (a.hw * size % 16) return image <= kMostStrip - 4096 && image % 16 == 0 && a.hw <= 1024 ? a.hw : 0;
    for (int width = 64; width >= (int)(16 / size); width /= 2)
        if ((size_t)a.c * width * size <= kTwoBlocks - 4096) return width < a.hw ? width : 0;
    return 0;
}

template <typename T>
tc_status quantize(int device, int sm_count, const RowQuantizeArgs &a, uint32_t *workspace, cudaStream_t s)
{
    const T *const x = (const T *)a.x;
    const long long pixels = (long long)a.n * a.hw;
    RowMatrix left[2] = {a.pixels, a.channels};
    bool first = true;
    auto launch = [&](auto kernel, dim3 grid, int threads, size_t smem, auto... args) {
        const cudaError_t err = first ? launch_first(true, kernel, grid, dim3(threads), smem, s, args...) : launch_chained(true, kernel, grid, dim3(threads), smem, s, args...);
        first = false;
        return err == cudaSuccess;
    };
    auto join = [&](int parts, long long rows, float *scales) {
        return launch(join_maxima_kernel, dim3((unsigned int)((rows + 31) / 32)), 1024, 0, (const uint32_t *)workspace, parts, rows, scales);
    };
    MatrixArgs t{};
    t.pixels = pixels;
    t.c = a.c;
    t.hw = a.hw;
    if (rows_with_columns(a)) {
        const int blocks = rows_blocks(a, sm_count);
        const long long rows = pixels;
        bool ok;
        if (a.c <= 2048) ok = launch(rows_and_columns_kernel<T, 256, 1>, dim3(blocks), 256, 0, x, rows, a.c, a.pixels, workspace);
        else ok = launch(rows_and_columns_kernel<T, 256, 2>, dim3(blocks), 256, 0, x, rows, a.c, a.pixels, workspace);
        if (!ok || !join(blocks, a.c, a.channels.scales)) return TC_ERR_CUDA;
        left[0] = RowMatrix{};
        t.across = left[1];
    } else {
        for (int i = 0; i < 2; ++i)
            if (left[i].codes && in_memory(a, i)) {
                const tc_status st = i ? launch_rows(x, a.c, (int)pixels, left[i], s) : launch_rows(x, pixels, a.c, left[i], s);
                if (st != TC_OK) return st;
                left[i] = RowMatrix{};
                first = false;
            }
        if (const int width = left[0].codes ? strip_of(a) : 0) {
            const StripArgs strip{a.c, a.hw, width, (a.hw + width - 1) / width, left[0], a.status};
            const size_t smem = strip_bytes(a.c, width, sizeof(T));
            const dim3 grid((unsigned int)(a.n * strip.strips));
            const int threads = strip.strips > 1 ? kStripThreads / 2 : kStripThreads;
            if (!allow_shared<pixel_strip_kernel<T, 1>>(device, kMostStrip) || !allow_shared<pixel_strip_kernel<T, 2>>(device, kMostStrip) ||
                !(width % 2 ? launch(pixel_strip_kernel<T, 1>, grid, threads, smem, x, strip) : launch(pixel_strip_kernel<T, 2>, grid, threads, smem, x, strip))) return TC_ERR_CUDA;
            left[0] = RowMatrix{};
        }
        if (!left[0].codes && !left[1].codes) return TC_OK;
        t.along = a.hw > 1 ? left[1] : left[0];
        t.across = a.hw > 1 ? left[0] : left[1];
        const int vec = vector_of(a);
        if (t.across.codes) {
            const int parts = parts_across(a, vec == 8 ? 8 : 1, sm_count);
            const long long outer = a.hw > 1 ? a.c : pixels, inner = a.hw > 1 ? pixels : a.c, of_chunk = (outer + parts - 1) / parts;
            const dim3 grid((unsigned int)((inner + 64 * (vec == 8 ? 8 : 1) - 1) / (64 * (vec == 8 ? 8 : 1))), (unsigned int)parts);
            const bool ok = a.hw > 1 ? vec == 8 ? launch(column_maxima_kernel<T, true, 8>, grid, 256, 0, x, t, of_chunk, workspace) : launch(column_maxima_kernel<T, true, 1>, grid, 256, 0, x, t, of_chunk, workspace)
                                     : vec == 8 ? launch(column_maxima_kernel<T, false, 8>, grid, 256, 0, x, t, of_chunk, workspace) : launch(column_maxima_kernel<T, false, 1>, grid, 256, 0, x, t, of_chunk, workspace);
            if (!ok || !join(parts, inner, t.across.scales)) return TC_ERR_CUDA;
        }
        if (t.along.codes) {
            const int parts = parts_along(a, sm_count), images = (a.n + parts - 1) / parts;
            const dim3 grid((unsigned int)a.c, (unsigned int)parts);
            if (!(vec == 8   ? launch(channel_maxima_kernel<T, 8>, grid, 256, 0, x, t, images, workspace)
                  : vec == 4 ? launch(channel_maxima_kernel<T, 4>, grid, 256, 0, x, t, images, workspace)
                             : launch(channel_maxima_kernel<T, 1>, grid, 256, 0, x, t, images, workspace)) ||
                !join(parts, a.c, t.along.scales)) return TC_ERR_CUDA;
        }
    }
    const dim3 grid((unsigned int)((pixels + kTile - 1) / kTile), (unsigned int)((a.c + kTile - 1) / kTile));
    constexpr size_t smem = kTile * kTile * sizeof(T);
    if (!allow_shared<row_tile_kernel<T, true>>(device, smem) || !allow_shared<row_tile_kernel<T, false>>(device, smem)) return TC_ERR_CUDA;
    return launch(a.hw > 1 ? row_tile_kernel<T, true> : row_tile_kernel<T, false>, grid, kTileThreads, smem, x, t, vector_of(a)) ? TC_OK : TC_ERR_CUDA;
}

}  // namespace

size_t tc_quantize_rows_workspace(const RowQuantizeArgs &a, int sm_count)
{
    if (rows_with_columns(a)) return (size_t)rows_blocks(a, sm_count) * a.c * sizeof(uint32_t);
    size_t words = 0;
    const size_t pixels = (size_t)a.n * a.hw;
    const bool by_pixel = a.pixels.codes && !in_memory(a, false) && !strip_of(a), by_channel = a.channels.codes && !in_memory(a, true);
    if (a.hw > 1 ? by_pixel : by_channel) words = parts_across(a, vector_of(a) == 8 ? 8 : 1, sm_count) * (a.hw > 1 ? pixels : (size_t)a.c);
    if (a.hw > 1 && by_channel) words = std::max(words, (size_t)parts_along(a, sm_count) * a.c);
    return words * sizeof(uint32_t);
}

tc_status tc_launch_quantize_rows(int device, int sm_count, const RowQuantizeArgs &a, void *workspace, cudaStream_t s)
{
    return a.dtype == TC_BF16 ? quantize<__nv_bfloat16>(device, sm_count, a, (uint32_t *)workspace, s) : quantize<float>(device, sm_count, a, (uint32_t *)workspace, s);
}
