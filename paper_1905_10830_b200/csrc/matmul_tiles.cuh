// What the products of 8-bit matrices share: the tiles' order, and the ways of a tile's values to the output (NCHW or rows; bias,
// activation, 16- and 8-byte stores through boxes in shared memory, single values).
#pragma once

#include "block_codes.cuh"
#include "tc_internal.h"

namespace tiles {

using namespace blk;

constexpr int kRowsM = 128;
constexpr int kBoxBytes = 4096;                               // what a warp turns on the way to the output: 32 rows of 128 bytes

struct TileArgs {
    int rows_a, rows_b;               // of the MMA's operands
    int k_blocks, splits;
    int tiles_m, tiles_n;
    const float *scale_a, *scale_b;
    long long scale_a_ld, scale_b_ld;
    int shift_a, shift_b;             // 0: a scale for each row, 7: for each 128
    int group;                        // tile rows that are worked on together
    int swapped, cluster;             // cluster: the parts of a tile's length are a cluster's CTAs
    int join_rows;                    // and a pixel's channels are neighbours in a row of the tile
    int out_channels, hw, relu;
    int vec;                          // bytes of a store by rows, 0: values one by one
    int by_rows;                      // a row's columns are neighbours in the output, else the rows of a column are
    int store_tma;                    // pairs: rows leave by TMA copies
    const float *bias;
    void *out;
    float *partial;                   // [unit][column][128 rows], where the length is split
    unsigned int *status;
};

struct Unit {
    int tile_m, tile_n, k_first, k_end;
};
// Units in the order they are worked on: the parts of a tile's length one after the other; tiles in columns of `group` tile rows,
// so that the SMs' operands at any time are few rows of both matrices.
__device__ __forceinline__ Unit unit_of(const TileArgs &a, int u)
{
    const int tile = u / a.splits, split = u - tile * a.splits;
    const int per_group = a.group * a.tiles_n, g = tile / per_group, rest = tile - g * per_group;
    const int high = min(a.group, a.tiles_m - g * a.group);
    Unit r;
    r.tile_n = rest / high;
    r.tile_m = g * a.group + rest - r.tile_n * high;
    r.k_first = (int)((long long)a.k_blocks * split / a.splits);
    r.k_end = (int)((long long)a.k_blocks * (split + 1) / a.splits);
    return r;
}

// Where element 0 of a pixel lies in an NCHW tensor.
__device__ __forceinline__ long long pixel_at(const TileArgs &a, int p)
{
    if (a.hw == 1) return (long long)p * a.out_channels;
    const int img = p / a.hw;
    return (long long)img * a.out_channels * a.hw + (p - img * a.hw);
}

__device__ __forceinline__ void put(float *out, long long at, float v) { out[at] = v; }
__device__ __forceinline__ void put(__nv_bfloat16 *out, long long at, float v) { out[at] = __float2bfloat16_rn(v); }

// One value, with bias and activation.
template <typename T>
__device__ __forceinline__ void store_value(const TileArgs &a, int row, int col, float v)
{
    if (row >= a.rows_a || col >= a.rows_b) return;
    const int p = a.swapped ? col : row, o = a.swapped ? row : col;
    if (a.bias) v += a.bias[o];
    if (a.relu && v < 0.f) v = 0.f;                           // (a NaN stays one: a comparison with it fails)
    put((T *)a.out, pixel_at(a, p) + (long long)o * a.hw, v);
}

// Four neighbouring channels of a pixel.
template <typename T>
__device__ __forceinline__ void store_four(const TileArgs &a, int row, int col, float (&v)[4])
{
    if (a.vec == 16 && !a.swapped && a.hw == 1 && col + 4 <= a.rows_b) {
        __align__(16) T w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (a.bias) v[j] += a.bias[col + j];
            if (a.relu && v[j] < 0.f) v[j] = 0.f;
            put(w, j, v[j]);
        }
        T *const to = (T *)a.out + (long long)row * a.out_channels + col;
        if constexpr (sizeof(T) == 2) *reinterpret_cast<uint2 *>(to) = *reinterpret_cast<const uint2 *>(w);
        else *reinterpret_cast<uint4 *>(to) = *reinterpret_cast<const uint4 *>(w);
    } else
#pragma unroll
        for (int j = 0; j < 4; ++j) store_value<T>(a, row, col + j, v[j]);
}

// Bias and activation, in a pass of their own: the stores, of which a warp's time between two tiles consists, stay short.  The j-th pair is of
// row and column place(j).
template <int kPairs, typename F>
__device__ __forceinline__ void finish(const TileArgs &a, uint64_t (&sum)[kPairs], F place)
{
    if (a.bias) {
#pragma unroll
        for (int j = 0; j < kPairs; ++j) {
            const int2 at = place(j);
            const int last = a.out_channels - 1, o = a.swapped ? at.x : at.y;
            sum[j] = add2(sum[j], pair_of(a.bias[min(o, last)], a.bias[min(a.swapped ? o : o + 1, last)]));
        }
    }
    if (a.relu)
#pragma unroll
        for (int j = 0; j < kPairs; ++j) {
            float x, y;
            halves(sum[j], x, y);
            sum[j] = pair_of(x < 0.f ? 0.f : x, y < 0.f ? 0.f : y);            // (a NaN stays one: a comparison with it fails)
        }
}

// The sums of a thread's row and kCols columns from `col0` on, a column at a time: where the lanes' rows are neighbours in the output.
template <typename T, int kCols>
__device__ __forceinline__ void store_lanes(const TileArgs &a, const uint64_t (&sum)[kCols / 2], int row, int col0)
{
    if (row >= a.rows_a) return;
    const int cols = min(kCols, a.rows_b - col0);
    const bool apart = a.swapped && a.hw > 1;                 // (few pixels: their places are looked up)
    T *const to = (T *)a.out + (a.swapped ? (long long)row * a.hw + (apart ? 0 : (long long)col0 * a.out_channels) : pixel_at(a, row) + (long long)col0 * a.hw);
    const int pitch = a.swapped ? a.out_channels : a.hw;
#pragma unroll
    for (int i = 0; i < kCols / 2; ++i) {
        float x, y;
        halves(sum[i], x, y);
        if (2 * i < cols) put(to, apart ? pixel_at(a, col0 + 2 * i) : (long long)(2 * i) * pitch, x);
        if (2 * i + 1 < cols) put(to, apart ? pixel_at(a, col0 + 2 * i + 1) : (long long)(2 * i + 1) * pitch, y);
    }
}

// Where a row's columns are neighbours in the output a warp turns them in shared memory: a box of 32 rows x 128 bytes, 16-byte pieces
// exchanged by XOR with the row.  (Stored by their threads, 16 bytes or a value at a time, each store meets 32 rows: 2000x1000 to 1000 took 14 us
// and 8.8.)
template <typename T> constexpr int kBoxCols = 128 / (int)sizeof(T);
// A thread's row of the box from the sums of its columns.
template <typename T>
__device__ __forceinline__ void fill_box(uint32_t box, const uint64_t *sum, int lane)
{
#pragma unroll
    for (int piece = 0; piece < 8; ++piece) {
        constexpr int kPer = 16 / (int)sizeof(T);
        __align__(16) T w[kPer];
#pragma unroll
        for (int j = 0; j < kPer; j += 2) {
            float x, y;
            halves(sum[(piece * kPer + j) / 2], x, y);
            put(w, j, x);
            put(w, j + 1, y);
        }
        const uint4 v = *reinterpret_cast<const uint4 *>(w);
        asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(box + lane * 128u + ((uint32_t)(piece ^ (lane & 7)) << 4)), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w)
                     : "memory");
    }
}
// The box to the output, its lanes along the columns.
template <typename T>
__device__ __forceinline__ void store_box(const TileArgs &a, uint32_t box, int first_row, int col, int lane)
{
    const int rows = min(32, a.rows_a - first_row), cols = min(kBoxCols<T>, a.rows_b - col);
    T *const out = (T *)a.out;
    constexpr int kPer = 16 / (int)sizeof(T);
    if (a.vec) {
        const int piece = lane & 7, c = piece * kPer;
        if (c >= cols) return;                                // (rows, or four or eight pixels of a map, end at a multiple of a store)
        const bool half = c + kPer / 2 >= cols;
        const long long pitch = a.swapped ? a.hw : a.out_channels;
        T *to = out + (a.swapped ? pixel_at(a, col + c) : (long long)(col + c)) + (long long)(first_row + (lane >> 3)) * pitch;
        const long long second = a.swapped && !half ? pixel_at(a, col + c + kPer / 2) - pixel_at(a, col + c) : kPer / 2;
#pragma unroll
        for (int r = lane >> 3; r < 32; r += 4, to += 4 * pitch)
            if (r < rows) {
                uint4 v;
                asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                             : "r"(box + (uint32_t)r * 128u + ((uint32_t)(piece ^ (r & 7)) << 4)));
                if (a.vec == 16) *reinterpret_cast<uint4 *>(to) = v;
                else {
                    *reinterpret_cast<uint2 *>(to) = make_uint2(v.x, v.y);
                    if (!half) *reinterpret_cast<uint2 *>(to + second) = make_uint2(v.z, v.w);
                }
            }
        return;
    }
#pragma unroll
    for (int h = 0; h < kBoxCols<T> / 32; ++h) {
        const int c = 32 * h + lane;
        if (c >= cols) continue;
        const uint32_t byte = (uint32_t)c * sizeof(T);
        T *to = out + (a.swapped ? pixel_at(a, col + c) + (long long)first_row * a.hw : (long long)first_row * a.out_channels + col + c);
        const long long pitch = a.swapped ? a.hw : a.out_channels;
#pragma unroll 8
        for (int r = 0; r < rows; ++r, to += pitch) {
            const uint32_t at = box + (uint32_t)r * 128u + (((byte >> 4) ^ (uint32_t)(r & 7)) << 4) + (byte & 15u);
            if constexpr (sizeof(T) == 2) {
                unsigned short v;
                asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(at));
                *reinterpret_cast<unsigned short *>(to) = v;
            } else {
                uint32_t v;
                asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(at));
                *reinterpret_cast<uint32_t *>(to) = v;
            }
        }
    }
}
template <typename T, int kCols>
__device__ __forceinline__ void store_by_rows(const TileArgs &a, uint32_t box, const uint64_t (&sum)[kCols / 2], int first_row, int col0, int lane)
{
    static_assert(kCols % kBoxCols<T> == 0, "whole boxes");
#pragma unroll
    for (int c = 0; c < kCols; c += kBoxCols<T>) {
        __syncwarp();                                         // the last box's readers
        fill_box<T>(box, sum + c / 2, lane);
        __syncwarp();
        if (first_row < a.rows_a && col0 + c < a.rows_b) store_box<T>(a, box, first_row, col0 + c, lane);
    }
}

}  // namespace tiles
