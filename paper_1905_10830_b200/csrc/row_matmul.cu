// tc_matmul_rows: product of two matrices of 8-bit integers with a scale for each row,
//
//   out[p][o] = act(fl(fl(fl(sum_k a[p][k] b[o][k]) sa[p]) sb[o]) + bias[o])
//
// The sum is exact: 32-bit integers in tensor memory hold up to kMostBlocks blocks of 128 codes, parts of a sum are added as
// 64-bit integers.  So a result does not depend on how the work was cut.
//
// Large products: pairs of CTAs (cta_group::2) on tiles of 256 x 256, two accumulators in tensor memory: the epilogue of a tile runs beside the
// next one's multiplications.  Small ones: one CTA on tiles of 128 rows x 16 to 128 columns, two to an SM up to 64; where tiles are
// fewer than SMs the sums' length is cut into parts, by the CTAs of a cluster that add through their shared memory, or
// through a workspace.
#include "block_codes.cuh"
#include "matmul_tiles.cuh"
#include "sm100_ptx.cuh"
#include "tc_internal.h"

namespace {

using namespace tcdev;
using namespace sm100;
using namespace blk;
using namespace tiles;

constexpr int kBlockK = 128;
constexpr int kStageA = kRowsM * kBlockK;
constexpr int kMostBlocks = 1023;                             // of a part: 2^14 x 128 x 1023 < 2^31 (codes of -128 too)

template <int kN> struct Shape {
    static constexpr int kSets = kN >= 128 ? 2 : 1;           // sets of four epilogue warps, each with its share of the columns
    static constexpr int kCols = kN / kSets;
    static constexpr int kEpiWarps = 4 * kSets, kProducer = kEpiWarps, kMma = kEpiWarps + 1;
    static constexpr int kThreads = (kEpiWarps + 2) * 32;
    static constexpr int kStageBytes = kStageA + kN * kBlockK;
    static constexpr int kStages = kN == 128 ? 5 : kN == 64 ? 3 : kN == 32 ? 4 : 5;
    static constexpr bool kBoxes = kN >= 64;
    static constexpr int kBuffers = 2;                        // of tensor memory
    static constexpr int kTmemCols = kN * kBuffers < 32 ? 32 : kN * kBuffers;
    static constexpr size_t kSmem = 1024 + (size_t)kStages * kStageBytes + (kBoxes ? kEpiWarps * kBoxBytes : 0);
};

// Tiles of a pair of CTAs: 256 x 256, 128 rows of each operand a CTA.
namespace pair {
constexpr int kN = 256, kRows = 256;
constexpr int kStageBytes = 2 * kStageA, kBuffers = 2, kTmemCols = 512;
constexpr int kSets = 2, kCols = kN / kSets;
constexpr int kEpiWarps = 8, kProducer = 8, kMma = 9;
constexpr int kThreads = 10 * 32;
// Long sums: a ring of five stages, a box a warp on the way out; short ones, whose stores are most of their time: four stages and two boxes (4096 to 8192 of 8192 rows 177 us
// with the first, 184 with the second; 256 to 256 of 200704 46 and 42).
template <bool kLong> constexpr int kStages = kLong ? 5 : 4;
template <bool kLong> constexpr int kBoxes = kLong ? 1 : 2;
template <bool kLong> constexpr size_t kSmem = 1024 + (size_t)kStages<kLong> * kStageBytes + kEpiWarps * kBoxes<kLong> * kBoxBytes;
constexpr int kLongBlocks = 8;
}

struct RowArgs : TileArgs {
    int *parts;                       // [unit - first_unit][column][128 rows], where the length is split through a workspace
    int first_unit, end_unit;
};

__device__ __forceinline__ float rounded(long long sum) { return __ll2float_rn(sum); }

// fl(fl(sum sa) sb), by the pixel's scale first.
__device__ __forceinline__ float scaled(const TileArgs &a, int row, int col, float v)
{
    if (row >= a.rows_a || col >= a.rows_b) return 0.f;       // (not stored)
    const float of_row = a.scale_a[row], of_col = a.scale_b[col];
    return a.swapped ? v * of_col * of_row : v * of_row * of_col;
}

// What an epilogue warp needs of a tile: its columns' scales and, where the columns are channels, their bias, in its slot of shared memory; its row's scale and
// bias.  Asked for while the tile before is stored (with sums of one or two blocks the wait for them was a quarter of a tile's time).
template <int kCols>
struct Scales {
    static constexpr int kMine = (kCols + 31) / 32;           // columns of a lane
    float *slot;                                              // [2][kCols]
    float of_column[kMine], bias[kMine], row_next, row_bias_next;
    float row, row_bias;
    __device__ __forceinline__ void ask(const TileArgs &a, int my_row, int col0, int lane)
    {
        const int at_row = min(my_row, a.rows_a - 1);
        row_next = a.scale_a[at_row];
        row_bias_next = a.bias && a.swapped ? a.bias[at_row] : 0.f;
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
            const int at = min(col0 + 32 * i + lane, a.rows_b - 1);                // (columns behind the last take its scale; nothing of theirs is stored)
            of_column[i] = a.scale_b[at];
            bias[i] = a.bias && !a.swapped ? a.bias[at] : 0.f;
        }
    }
    __device__ __forceinline__ void take(int lane)
    {
        __syncwarp();                                         // the last tile's readers
#pragma unroll
        for (int i = 0; i < kMine; ++i)
            if (32 * i + lane < kCols) {
                slot[32 * i + lane] = of_column[i];
                slot[kCols + 32 * i + lane] = bias[i];
            }
        row = row_next;
        row_bias = row_bias_next;
        __syncwarp();
    }
};
// kPairs pairs of neighbouring columns' sums to values, with bias and activation.
template <int kCols, int kPairs>
__device__ __forceinline__ void finish_rows(const TileArgs &a, const uint32_t *r, uint64_t *out, const Scales<kCols> &scales, int c)
{
    const uint64_t rs = pair_of(scales.row, scales.row), rb = pair_of(scales.row_bias, scales.row_bias);
    const uint64_t *const cs = reinterpret_cast<const uint64_t *>(scales.slot + c), *const cb = reinterpret_cast<const uint64_t *>(scales.slot + kCols + c);
#pragma unroll
    for (int j = 0; j < kPairs; ++j) {
        uint64_t v = pair_of((float)(int)r[2 * j], (float)(int)r[2 * j + 1]);
        v = a.swapped ? mul2(mul2(v, cs[j]), rs) : mul2(mul2(v, rs), cs[j]);
        if (a.bias) v = add2(v, a.swapped ? rb : cb[j]);
        if (a.relu) {
            float x, y;
            halves(v, x, y);
            v = pair_of(x < 0.f ? 0.f : x, y < 0.f ? 0.f : y);                     // (a NaN stays one: a comparison with it fails)
        }
        out[j] = v;
    }
}

template <typename T, int kN>
__global__ void __launch_bounds__(Shape<kN>::kThreads, kN <= 64 ? 2 : 1)
row_matmul_kernel(const __grid_constant__ RowArgs a, const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b)
{
    using S = Shape<kN>;
    extern __shared__ unsigned char smem_raw[];
    __shared__ __align__(8) unsigned long long s_full[S::kStages], s_empty[S::kStages], s_tfull[S::kBuffers], s_tempty[S::kBuffers];
    __shared__ uint32_t s_tmem_base;
    __shared__ __align__(16) float s_columns[S::kEpiWarps][2 * S::kCols];
    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
    const uint32_t ring = (smem_u32(smem_raw) + 1023u) & ~1023u;
    if (tid == S::kProducer * 32) { tensormap_prefetch(&map_a); tensormap_prefetch(&map_b); }
    if (tid == 0) {
        for (int s = 0; s < S::kStages; ++s) { mbar_init(smem_u32(&s_full[s]), 1); mbar_init(smem_u32(&s_empty[s]), 1); }
        for (int b = 0; b < S::kBuffers; ++b) { mbar_init(smem_u32(&s_tfull[b]), 1); mbar_init(smem_u32(&s_tempty[b]), S::kEpiWarps); }
        mbar_fence_init();
    }
    if (warp == S::kMma) { tmem_alloc(smem_u32(&s_tmem_base), S::kTmemCols); tmem_relinquish(); }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    chain_next();                                             // (behind the allocation of tensor memory)
    const uint32_t tmem_base = __shfl_sync(0xffffffffu, s_tmem_base, 0);
    chain_wait();

    if (warp == S::kProducer) {
        if (lane == 0) {
            int s = 0;
            long long issued = 0;
            uint32_t phase = 1;
            bool alive = true;
            for (int u = a.first_unit + blockIdx.x; u < a.end_unit && alive; u += gridDim.x) {
                const Unit t = unit_of(a, u);
                for (int kb = t.k_first; kb < t.k_end; ++kb) {
                    if (!mbar_wait_soon(smem_u32(&s_empty[s]), phase)) { alive = false; break; }
                    const uint32_t bar = smem_u32(&s_full[s]), dst = ring + (uint32_t)s * S::kStageBytes;
                    mbar_arrive_expect_tx(bar, (uint32_t)S::kStageBytes);
                    tma_load_2d(dst, &map_a, kb * kBlockK, t.tile_m * kRowsM, bar);
                    tma_load_2d(dst + kStageA, &map_b, kb * kBlockK, t.tile_n * kN, bar);
                    ++issued;
                    if (++s == S::kStages) { s = 0; phase ^= 1u; }
                }
            }
            if (!alive) tc_dev_set_status(a.status, TC_ERR_TIMEOUT);
            // The copies in flight land before the block's shared memory goes to another, whichever warp's wait ran out.
            for (long long i = issued > S::kStages ? issued - S::kStages : 0; i < issued; ++i) mbar_wait_soon(smem_u32(&s_full[i % S::kStages]), (uint32_t)(i / S::kStages & 1));
        }
    } else if (warp == S::kMma) {
        const uint32_t issuer = lane == 0 ? 1u : 0u;
        const uint32_t idesc = make_idesc_s8(kRowsM, kN);
        const uint64_t desc = make_smem_desc_sw128(ring, 1024);
        const uint32_t desc_lo = (uint32_t)desc, desc_hi = (uint32_t)(desc >> 32);
        int s = 0, b = 0;
        uint32_t phase = 0, tphase = 1;
        bool alive = true;
        for (int u = a.first_unit + blockIdx.x; u < a.end_unit && alive; u += gridDim.x) {
            const Unit t = unit_of(a, u);
            if (!mbar_wait_soon(smem_u32(&s_tempty[b]), tphase)) { alive = false; break; }
            for (int kb = t.k_first; kb < t.k_end; ++kb) {
                if (!mbar_wait_soon(smem_u32(&s_full[s]), phase)) { alive = false; break; }
                tc_fence_after_sync();
                const uint32_t a_lo = desc_lo + (uint32_t)s * (S::kStageBytes >> 4), b_lo = a_lo + (kStageA >> 4);
#pragma unroll
                for (int q = 0; q < kBlockK / 32; ++q)
                    mma_s8_ss_guarded(tmem_base + b * kN, a_lo + 2 * q, desc_hi, b_lo + 2 * q, desc_hi, idesc, q || kb > t.k_first ? 1u : 0u, issuer);
                mma_commit_guarded(smem_u32(&s_empty[s]), issuer);
                if (++s == S::kStages) { s = 0; phase ^= 1u; }
            }
            if (!alive) break;
            mma_commit_guarded(smem_u32(&s_tfull[b]), issuer);
            if (++b == S::kBuffers) { b = 0; tphase ^= 1u; }
        }
        if (!alive && issuer) tc_dev_set_status(a.status, TC_ERR_TIMEOUT);
    } else {
        const int set = warp >> 2, wq = warp & 3;
        const int row_in_tile = wq * 32 + lane;
        Scales<S::kCols> scales;
        scales.slot = s_columns[warp];
        int b = 0;
        uint32_t tphase = 0;
        bool alive = true;
        const bool whole = !a.cluster && !a.parts;
        Unit next = unit_of(a, a.first_unit + blockIdx.x);
        if (whole) scales.ask(a, next.tile_m * kRowsM + row_in_tile, next.tile_n * kN + set * S::kCols, lane);
        for (int u = a.first_unit + blockIdx.x; u < a.end_unit; u += gridDim.x) {
            const Unit t = next;
            const int row = t.tile_m * kRowsM + row_in_tile, col0 = t.tile_n * kN + set * S::kCols;
            if (whole) scales.take(lane);
            if (u + (int)gridDim.x < a.end_unit) {
                next = unit_of(a, u + gridDim.x);
                if (whole) scales.ask(a, next.tile_m * kRowsM + row_in_tile, next.tile_n * kN + set * S::kCols, lane);
            }
            // (asked of the whole warp: what follows is done by all its lanes together)
            if (!__all_sync(0xffffffffu, mbar_wait_soon(smem_u32(&s_tfull[b]), tphase))) { alive = false; break; }
            tc_fence_after_sync();
            const uint32_t at = tmem_base + b * kN + set * S::kCols + ((uint32_t)(wq * 32) << 16);
            auto hand_back = [&] {
                tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&s_tempty[b]));
            };
            if (!whole) {
                // this part's sums: in the ring, which the tensor cores are done with, [column][128 rows] or, where a pixel's channels are neighbours,
                // [row][kN + 4 columns]; or in the workspace
                int *const ring_at = reinterpret_cast<int *>(smem_raw + (ring - smem_u32(smem_raw)));
                int *const to = a.cluster ? ring_at : a.parts + (long long)(u - a.first_unit) * kN * kRowsM;
#pragma unroll
                for (int c = 0; c < S::kCols; c += 16) {
                    uint32_t r[16];
                    tmem_ld_32x32b_x16(at + c, r);
                    tmem_ld_wait(r);
                    if (c + 16 == S::kCols) hand_back();
                    if (a.cluster && a.join_rows) {
                        uint4 *const dst = reinterpret_cast<uint4 *>(to + row_in_tile * (kN + 4) + set * S::kCols + c);
#pragma unroll
                        for (int i = 0; i < 4; ++i) dst[i] = make_uint4(r[4 * i], r[4 * i + 1], r[4 * i + 2], r[4 * i + 3]);
                    } else {
#pragma unroll
                        for (int i = 0; i < 16; ++i) to[(set * S::kCols + c + i) * kRowsM + row_in_tile] = (int)r[i];
                    }
                }
                if (a.cluster) break;                         // a CTA has one part
            } else if (S::kBoxes && a.by_rows) {
                if constexpr (S::kBoxes) {
                    const uint32_t box = ring + S::kStages * S::kStageBytes + warp * kBoxBytes;
#pragma unroll
                    for (int c = 0; c < S::kCols; c += kBoxCols<T>) {
                        uint64_t v[kBoxCols<T> / 2];
#pragma unroll
                        for (int h = 0; h < kBoxCols<T>; h += 32) {
                            uint32_t r[32];
                            tmem_ld_32x32b_x32(at + c + h, r);
                            tmem_ld_wait(r);
                            if (c + h + 32 == S::kCols) hand_back();
                            finish_rows<S::kCols, 16>(a, r, v + h / 2, scales, c + h);
                        }
                        __syncwarp();                         // the last box's readers
                        fill_box<T>(box, v, lane);
                        __syncwarp();
                        if (row - lane < a.rows_a && col0 + c < a.rows_b) store_box<T>(a, box, row - lane, col0 + c, lane);
                    }
                }
            } else {
#pragma unroll
                for (int c = 0; c < S::kCols; c += 16) {
                    uint32_t r[16];
                    uint64_t v[8];
                    tmem_ld_32x32b_x16(at + c, r);
                    tmem_ld_wait(r);
                    if (c + 16 == S::kCols) hand_back();
                    finish_rows<S::kCols, 8>(a, r, v, scales, c);
                    store_lanes<T, 16>(a, v, row, col0 + c);
                }
            }
            __syncwarp();
            if (++b == S::kBuffers) { b = 0; tphase ^= 1u; }
        }
        if (!alive && lane == 0) tc_dev_set_status(a.status, TC_ERR_TIMEOUT);
    }
    tc_fence_before_sync();
    __syncthreads();
    if (warp == S::kMma) {
        tc_fence_after_sync();
        tmem_dealloc(tmem_base, S::kTmemCols);
    }
    if (a.cluster) {
        // The cluster's CTAs each add their share of the rows (columns) over all parts, four values at a time.
        const int u = blockIdx.x, rank = u % a.splits;
        const Unit t = unit_of(a, u);
        const int rows = min(kRowsM, a.rows_a - t.tile_m * kRowsM), cols = min(kN, a.rows_b - t.tile_n * kN);
        const int lines = a.join_rows ? rows : cols, fours = ((a.join_rows ? cols : rows) + 3) / 4, share = (lines + a.splits - 1) / a.splits;
        const int first = rank * share, count = (min(lines, first + share) - first) * fours;
        const uint32_t pitch = 4u * (a.join_rows ? kN + 4 : kRowsM);
        cluster_sync();
        for (int i = tid; i < count; i += S::kThreads) {
            const int line = first + i / fours, four = i - i / fours * fours;
            const uint32_t at = ring + (uint32_t)line * pitch + 16u * (uint32_t)four;
            int4 v[8];
#pragma unroll
            for (int part = 0; part < 8; ++part)
                if (part < a.splits)
                    asm volatile("ld.shared::cluster.v4.s32 {%0, %1, %2, %3}, [%4];" : "=r"(v[part].x), "=r"(v[part].y), "=r"(v[part].z), "=r"(v[part].w)
                                 : "r"(cluster_address(at, (uint32_t)part)));
            long long sum[4] = {v[0].x, v[0].y, v[0].z, v[0].w};
#pragma unroll
            for (int part = 1; part < 8; ++part)
                if (part < a.splits) { sum[0] += v[part].x; sum[1] += v[part].y; sum[2] += v[part].z; sum[3] += v[part].w; }
            const int row = t.tile_m * kRowsM + (a.join_rows ? line : 4 * four), col = t.tile_n * kN + (a.join_rows ? 4 * four : line);
            float r[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) r[j] = scaled(a, a.join_rows ? row : row + j, a.join_rows ? col + j : col, rounded(sum[j]));
            if (a.join_rows) store_four<T>(a, row, col, r);
            else
#pragma unroll
                for (int j = 0; j < 4; ++j) store_value<T>(a, row + j, col, r[j]);
        }
        cluster_sync();                                       // this block's shared memory is read no more
    }
}

// Adds the parts of the sums of tiles from `first_tile` on and writes the output.  Also the whole product where there is nothing to add.
template <typename T>
__global__ void __launch_bounds__(256) row_matmul_join_kernel(RowArgs a, int n, int first_tile, int end_tile)
{
    chain_next();
    chain_wait();
    const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
    const int row_in_tile = (int)(i & 127);
    const long long rest = i >> 7;
    const int tile = first_tile + (int)(rest / n), col_in_tile = (int)(rest % n);
    if (tile >= end_tile) return;
    const int splits = a.splits;
    a.splits = 1;
    const Unit t = unit_of(a, tile);
    const int row = t.tile_m * kRowsM + row_in_tile, col = t.tile_n * n + col_in_tile;
    if (splits == 0) { store_value<T>(a, row, col, 0.f); return; }
    long long sum = 0;
    const int *src = a.parts + ((long long)(tile - first_tile) * splits * n + col_in_tile) * kRowsM + row_in_tile;
    for (int s = 0; s < splits; ++s) sum += src[(long long)s * n * kRowsM];
    store_value<T>(a, row, col, scaled(a, row, col, rounded(sum)));
}

// ---- pairs of CTAs -------------------------------------------------------------------------
template <typename T, bool kLong>
__global__ void __launch_bounds__(pair::kThreads, 1)
row_matmul_pair_kernel(const __grid_constant__ RowArgs a, const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                       const __grid_constant__ CUtensorMap map_out)
{
    using namespace pair;
    constexpr int kStages = pair::kStages<kLong>, kBoxes = pair::kBoxes<kLong>;
    extern __shared__ unsigned char smem_raw[];
    // s_full and s_tempty are the even CTA's: both CTAs' copies and epilogues report there; s_empty and s_tfull are each CTA's own.
    __shared__ __align__(8) unsigned long long s_full[kStages], s_empty[kStages], s_tfull[kBuffers], s_tempty[kBuffers];
    __shared__ uint32_t s_tmem_base;
    __shared__ __align__(16) float s_columns[kEpiWarps][2 * kCols];
    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
    const uint32_t ring = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const int rank = blockIdx.x & 1;                          // the cluster is two neighbours
    if (tid == kProducer * 32) { tensormap_prefetch(&map_a); tensormap_prefetch(&map_b); }
    if (tid == 0) {
        for (int s = 0; s < kStages; ++s) { mbar_init(smem_u32(&s_full[s]), 1); mbar_init(smem_u32(&s_empty[s]), 1); }
        for (int b = 0; b < kBuffers; ++b) { mbar_init(smem_u32(&s_tfull[b]), 1); mbar_init(smem_u32(&s_tempty[b]), 2 * kEpiWarps); }
        mbar_fence_init();
    }
    if (warp == kMma) { tmem_alloc_pair(smem_u32(&s_tmem_base), kTmemCols); tmem_relinquish_pair(); }
    tc_fence_before_sync();
    __syncthreads();
    cluster_sync();                                           // the other CTA's barriers are there
    tc_fence_after_sync();
    chain_next();                                             // (behind the allocation of tensor memory)
    const uint32_t tmem_base = __shfl_sync(0xffffffffu, s_tmem_base, 0);
    chain_wait();
    const int units = a.tiles_m * a.tiles_n, step = gridDim.x >> 1;

    if (warp >= kEpiWarps) {
        if (warp == kProducer && lane == 0) {
            int s = 0;
            long long issued = 0;
            uint32_t phase = 1;
            bool alive = true;
            for (int u = blockIdx.x >> 1; u < units && alive; u += step) {
                const Unit t = unit_of(a, u);
                for (int kb = 0; kb < a.k_blocks; ++kb) {
                    if (!mbar_wait_soon(smem_u32(&s_empty[s]), phase)) { alive = false; break; }
                    const uint32_t dst = ring + (uint32_t)s * kStageBytes, bar = cluster_address(smem_u32(&s_full[s]), 0);
                    if (rank == 0) mbar_arrive_expect_tx(smem_u32(&s_full[s]), 2u * kStageBytes);
                    tma_load_2d_pair(dst, &map_a, kb * kBlockK, t.tile_m * kRows + rank * kRowsM, bar);
                    tma_load_2d_pair(dst + kStageA, &map_b, kb * kBlockK, t.tile_n * kN + rank * kRowsM, bar);
                    ++issued;
                    if (++s == kStages) { s = 0; phase ^= 1u; }
                }
            }
            if (!alive) tc_dev_set_status(a.status, TC_ERR_TIMEOUT);
            // The copies in flight land before the block ends: with every stage handed back there are none.
            for (long long i = issued > kStages ? issued - kStages : 0; i < issued; ++i) mbar_wait_soon(smem_u32(&s_empty[i % kStages]), (uint32_t)(i / kStages & 1));
        } else if (warp == kMma && rank == 0) {
            const uint32_t issuer = lane == 0 ? 1u : 0u;
            const uint32_t idesc = make_idesc_s8(kRows, kN);
            const uint64_t desc = make_smem_desc_sw128(ring, 1024);
            const uint32_t desc_lo = (uint32_t)desc, desc_hi = (uint32_t)(desc >> 32);
            int s = 0, b = 0;
            uint32_t phase = 0, tphase = 1;
            bool alive = true;
            for (int u = blockIdx.x >> 1; u < units && alive; u += step) {
                if (!mbar_wait_soon(smem_u32(&s_tempty[b]), tphase)) { alive = false; break; }
                for (int kb = 0; kb < a.k_blocks; ++kb) {
                    if (!mbar_wait_soon(smem_u32(&s_full[s]), phase)) { alive = false; break; }
                    tc_fence_after_sync();
                    const uint32_t a_lo = desc_lo + (uint32_t)s * (kStageBytes >> 4), b_lo = a_lo + (kStageA >> 4);
#pragma unroll
                    for (int q = 0; q < kBlockK / 32; ++q)
                        mma_s8_ss_pair_guarded(tmem_base + b * kN, a_lo + 2 * q, desc_hi, b_lo + 2 * q, desc_hi, idesc, q || kb ? 1u : 0u, issuer);
                    mma_commit_pair_guarded(smem_u32(&s_empty[s]), issuer);
                    if (++s == kStages) { s = 0; phase ^= 1u; }
                }
                if (!alive) break;
                mma_commit_pair_guarded(smem_u32(&s_tfull[b]), issuer);
                if (++b == kBuffers) { b = 0; tphase ^= 1u; }
            }
            if (!alive && issuer) tc_dev_set_status(a.status, TC_ERR_TIMEOUT);
        }
        __syncwarp();
    } else {
        const int set = warp >> 2, wq = warp & 3;
        Scales<kCols> scales;
        scales.slot = s_columns[warp];
        const uint32_t boxes = ring + kStages * kStageBytes + warp * kBoxes * kBoxBytes;
        int turn = 0;
        uint32_t tempty[kBuffers];
#pragma unroll
        for (int b = 0; b < kBuffers; ++b) tempty[b] = cluster_address(smem_u32(&s_tempty[b]), 0);
        int b = 0;
        uint32_t tphase = 0;
        bool alive = true;
        auto ask = [&](const Unit &t) { scales.ask(a, t.tile_m * kRows + rank * kRowsM + wq * 32 + lane, t.tile_n * kN + set * kCols, lane); };
        Unit next = unit_of(a, blockIdx.x >> 1);
        ask(next);
        for (int u = blockIdx.x >> 1; u < units; u += step) {
            const Unit t = next;
            const int first_row = t.tile_m * kRows + rank * kRowsM + wq * 32, col0 = t.tile_n * kN + set * kCols;
            scales.take(lane);
            if (u + step < units) ask(next = unit_of(a, u + step));
            // (asked of the whole warp: what follows is done by all its lanes together)
            if (!__all_sync(0xffffffffu, mbar_wait_soon(smem_u32(&s_tfull[b]), tphase))) { alive = false; break; }
            tc_fence_after_sync();
            const uint32_t at = tmem_base + b * kN + set * kCols + ((uint32_t)(wq * 32) << 16);
            auto hand_back = [&] {
                tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive_cluster(tempty[b]);
            };
            if (a.by_rows) {
#pragma unroll
                for (int c = 0; c < kCols; c += kBoxCols<T>) {
                    uint64_t v[kBoxCols<T> / 2];
#pragma unroll
                    for (int h = 0; h < kBoxCols<T>; h += 32) {
                        uint32_t r[32];
                        tmem_ld_32x32b_x32(at + c + h, r);
                        tmem_ld_wait(r);
                        if (c + h + 32 == kCols) hand_back();
                        finish_rows<kCols, 16>(a, r, v + h / 2, scales, c + h);
                    }
                    // boxes in turn: one may still be on its way out
                    const uint32_t box = boxes + turn * kBoxBytes;
                    turn = (turn + 1) % kBoxes;
                    if (a.store_tma && lane == 0) {
                        if constexpr (kBoxes == 2) tma_store_wait_read_but_one();
                        else tma_store_wait_read();
                    }
                    __syncwarp();                             // the last readers of this box
                    fill_box<T>(box, v, lane);
                    if (a.store_tma) fence_proxy_async_smem();
                    __syncwarp();
                    // (every turn has its group of copies, one outside the output an empty one, so that the group that may be pending is the other box's.  Boxes outside that took no turn
                    // instead made the turns' addresses unknown to the compiler: 256 to 256 of 1024 maps of 14x14 69 us for 65)
                    if (first_row < a.rows_a && col0 + c < a.rows_b) {
                        if (!a.store_tma) store_box<T>(a, box, first_row, col0 + c, lane);
                        else if (lane == 0) tma_store_2d(&map_out, col0 + c, first_row, box);
                    } else if (a.store_tma && lane == 0)
                        tma_store_none();
                }
            } else {
#pragma unroll
                for (int c = 0; c < kCols; c += 32) {
                    uint32_t r[32];
                    uint64_t v[16];
                    tmem_ld_32x32b_x32(at + c, r);
                    tmem_ld_wait(r);
                    if (c + 32 == kCols) hand_back();
                    finish_rows<kCols, 16>(a, r, v, scales, c);
                    store_lanes<T, 32>(a, v, first_row + lane, col0 + c);
                }
            }
            __syncwarp();
            if (++b == kBuffers) { b = 0; tphase ^= 1u; }
        }
        if (lane == 0) tma_store_wait();
        if (!alive && lane == 0) tc_dev_set_status(a.status, TC_ERR_TIMEOUT);
    }
    tc_fence_before_sync();
    __syncthreads();
    cluster_sync();                                           // nothing reports to this block any more
    if (warp == kMma) {
        tc_fence_after_sync();
        tmem_dealloc_pair(tmem_base, kTmemCols);
    }
}

template <typename T, int kN>
tc_status launch_tiles(const tc_ctx *ctx, const RowArgs &a, const CUtensorMap &map_a, const CUtensorMap &map_b, cudaStream_t s)
{
    constexpr auto kernel = row_matmul_kernel<T, kN>;
    if (!allow_shared<kernel>(ctx->device, Shape<kN>::kSmem)) return TC_ERR_CUDA;
    const int units = a.end_unit - a.first_unit, most = (kN <= 64 ? 2 : 1) * ctx->sm_count;
    const dim3 grid((unsigned int)(units < most || a.cluster ? units : most));
    return launch_first_cluster(a.cluster ? a.splits : 1, kernel, grid, dim3(Shape<kN>::kThreads), Shape<kN>::kSmem, s, a, map_a, map_b) == cudaSuccess ? TC_OK : TC_ERR_CUDA;
}

template <typename T, bool kLong>
tc_status launch_pairs(const tc_ctx *ctx, const RowArgs &a, const CUtensorMap &map_a, const CUtensorMap &map_b, const CUtensorMap &map_out, cudaStream_t s)
{
    constexpr auto kernel = row_matmul_pair_kernel<T, kLong>;
    if (!allow_shared<kernel>(ctx->device, pair::kSmem<kLong>)) return TC_ERR_CUDA;
    const int units = a.end_unit - a.first_unit, pairs = ctx->sm_count / 2;
    const dim3 grid((unsigned int)(2 * (units < pairs ? units : pairs)));
    return launch_first_cluster(2, kernel, grid, dim3(pair::kThreads), pair::kSmem<kLong>, s, a, map_a, map_b, map_out) == cudaSuccess ? TC_OK : TC_ERR_CUDA;
}

template <typename T>
tc_status launch(const tc_ctx *ctx, const RowArgs &a, bool pairs, int n, const CUtensorMap &map_a, const CUtensorMap &map_b, const CUtensorMap &map_out, cudaStream_t s)
{
    if (pairs) return a.k_blocks >= pair::kLongBlocks ? launch_pairs<T, true>(ctx, a, map_a, map_b, map_out, s) : launch_pairs<T, false>(ctx, a, map_a, map_b, map_out, s);
    switch (n) {
    case 16: return launch_tiles<T, 16>(ctx, a, map_a, map_b, s);
    case 32: return launch_tiles<T, 32>(ctx, a, map_a, map_b, s);
    case 64: return launch_tiles<T, 64>(ctx, a, map_a, map_b, s);
    case 128: return launch_tiles<T, 128>(ctx, a, map_a, map_b, s);
    default: return TC_ERR_UNSUPPORTED;                       // (no plan has it: a tile's size is a kernel's)
    }
}

constexpr size_t kPartsBytes = 64ull << 20;                   // parts of about so many bytes are added at a time

}  // namespace

MatmulPlan tc_plan_matmul_rows(const RowMatmulArgs &a, int sm_count)
{
    MatmulPlan best;
    const int k_blocks = (int)((a.cols + kBlockK - 1ll) / kBlockK);
    const int least = (k_blocks + kMostBlocks - 1) / kMostBlocks;                  // parts
    double best_cost = 0.0;
    auto consider = [&](bool swapped, bool pairs, int n, int splits) {
        const RowMatrix &m = swapped ? a.channels : a.pixels, &c = swapped ? a.pixels : a.channels;
        const int rows = pairs ? pair::kRows : kRowsM, workers = pairs ? sm_count / 2 : sm_count;
        const long long tiles = (((long long)m.rows + rows - 1) / rows) * (((long long)c.rows + n - 1) / n);
        const bool cluster = splits > 1 && splits <= 8;
        const long long units = tiles * splits;
        if (splits < least) return;
        if (splits > least && splits > 1 && (splits * 2 > k_blocks + 1 || (cluster ? units > (n <= 64 ? 2 : 1) * sm_count || (n > 64 && splits > 4) : units > sm_count))) return;
        const bool joined = cluster && units <= (n <= 64 ? 2 : 1) * sm_count && !(n > 64 && splits > 4);
        const double rounds = joined ? std::max(1.0, (double)units / sm_count) : (double)((units + workers - 1) / workers);
        const double block = pairs ? 560 : 330 + 2.5 * n;
        const bool by_rows = swapped ? a.hw > 1 : a.hw == 1;
        const double store = splits > 1 ? 8 * n : by_rows ? (pairs ? 4000 : n >= 64 ? 25 * n : 60 * n) : pairs ? 30000 : n == 128 ? 110 * n : 180 * n;
        const double cost = rounds * ((double)((k_blocks + splits - 1) / splits) * block + 600 + store) +
                            (joined ? 5000 + n * 22 : splits > 1 ? 9000 + (double)units * n * 0.5 : 0);
        if (best.n == 0 || cost < best_cost) {
            best_cost = cost;
            best.swapped = swapped;
            best.pairs = pairs;
            best.n = n;
            best.splits = splits;
            best.cluster = joined;
            best.tiles = tiles;
            const size_t tile_bytes = (size_t)splits * n * kRowsM * sizeof(int);
            best.workspace = splits > 1 && !joined ? std::min((size_t)tiles, std::max<size_t>(1, kPartsBytes / tile_bytes)) * tile_bytes : 0;
        }
    };
    for (int swapped = 0; swapped < 2; ++swapped) {
        for (int n = 16; n <= 128; n *= 2)
            if (n >= 64 || swapped) {
                for (const int splits : {1, 2, 3, 4, 6, 8, 16, 32, 64, 128}) consider(swapped, false, n, splits);
                if (least > 1) consider(swapped, false, n, least);
            }
        if (sm_count > 1 && least <= 1) consider(swapped, true, pair::kN, 1);
    }
    if (k_blocks == 0) { best.splits = 0; best.pairs = best.cluster = false; best.workspace = 0; }
    best.needs_workspace = best.workspace && least > 1;
    return best;
}

tc_status tc_launch_matmul_rows(const tc_ctx *ctx, const RowMatmulArgs &m, const MatmulPlan &plan, void *workspace, cudaStream_t s)
{
    const RowMatrix &ra = plan.swapped ? m.channels : m.pixels, &rb = plan.swapped ? m.pixels : m.channels;
    RowArgs a{};
    a.rows_a = ra.rows;
    a.rows_b = rb.rows;
    a.k_blocks = (int)((m.cols + kBlockK - 1ll) / kBlockK);
    a.splits = plan.splits;
    const int rows_tile = plan.pairs ? pair::kRows : kRowsM;
    a.tiles_m = (ra.rows + rows_tile - 1) / rows_tile;
    a.tiles_n = (rb.rows + plan.n - 1) / plan.n;
    a.group = plan.pairs ? 8 : 16;
    a.cluster = plan.cluster;
    a.by_rows = plan.swapped ? m.hw > 1 : m.hw == 1;
    a.join_rows = a.by_rows && !plan.swapped;
    a.scale_a = ra.scales;
    a.scale_b = rb.scales;
    a.swapped = plan.swapped;
    a.out_channels = m.channels.rows;
    a.hw = m.hw;
    a.relu = m.relu;
    // bytes that a store by rows moves: neighbouring channels of a pixel, or pixels of a map
    const long long line = m.hw == 1 ? m.channels.rows : m.hw, size = m.dtype == TC_BF16 ? 2 : 4;
    a.vec = !a.by_rows ? 0 : line * size % 16 == 0 && ((uintptr_t)m.out & 15u) == 0 ? 16 : line * size % 8 == 0 && ((uintptr_t)m.out & 7u) == 0 ? 8 : 0;
    a.bias = m.bias;
    a.out = m.out;
    a.status = m.status;
    const bool bf16 = m.dtype == TC_BF16;
    const int tiles = a.tiles_m * a.tiles_n;
    auto join = [&](bool early, int first, int end) {
        const long long values = (long long)(end - first) * plan.n * kRowsM;
        const dim3 grid((unsigned int)((values + 255) / 256));
        const cudaError_t err = bf16 ? launch_chained(early, row_matmul_join_kernel<__nv_bfloat16>, grid, dim3(256), 0, s, a, plan.n, first, end)
                                     : launch_chained(early, row_matmul_join_kernel<float>, grid, dim3(256), 0, s, a, plan.n, first, end);
        return err == cudaSuccess ? TC_OK : TC_ERR_CUDA;
    };
    if (plan.splits == 0) return join(false, 0, tiles);
    CUtensorMap map_a, map_b, map_out{};
    if (!tc_tensor_map_codes(&map_a, ra.codes, ra.rows, m.cols, ra.ld, kRowsM) ||
        !tc_tensor_map_codes(&map_b, rb.codes, rb.rows, m.cols, rb.ld, plan.pairs ? kRowsM : plan.n)) return TC_ERR_CUDA;
    a.store_tma = plan.pairs && a.vec == 16 && m.hw == 1 && tc_tensor_map_rows(&map_out, m.out, m.dtype, a.rows_a, a.rows_b, 32);
    auto multiply = [&] {
        return bf16 ? launch<__nv_bfloat16>(ctx, a, plan.pairs, plan.n, map_a, map_b, map_out, s) : launch<float>(ctx, a, plan.pairs, plan.n, map_a, map_b, map_out, s);
    };
    a.end_unit = tiles * plan.splits;
    if (!plan.workspace) return multiply();
    // some tiles at a time
    a.parts = (int *)workspace;
    const int most = (int)(plan.workspace / ((size_t)plan.splits * plan.n * kRowsM * sizeof(int)));
    for (int first = 0; first < tiles; first += most) {
        const int end = std::min(tiles, first + most);
        a.first_unit = first * plan.splits;
        a.end_unit = end * plan.splits;
        tc_status st = multiply();
        if (st == TC_OK) st = join(true, first, end);
        if (st != TC_OK) return st;
    }
    return TC_OK;
}
