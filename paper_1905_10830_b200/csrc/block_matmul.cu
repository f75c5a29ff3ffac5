// tc_matmul_blocks: product of two block-scaled e4m3 matrices,
//
//   out[p][o] = act(bias[o] + sum_kb sa[p][kb] sb[o][kb] sum_{k in block kb} a[p][k] b[o][k])
//
// A block of 128 codes is one row of a 128-byte swizzle atom, so a stage of the ring is a block: four MMAs of 32 codes
// leave its sum in tensor memory, the epilogue's warps read it back, multiply it by the block's scales and add it to sums in
// registers (fp32), while the MMAs of the next blocks fill the other buffers.
//
// Large products: pairs of CTAs (cta_group::2) walk tiles of 256 x 256, each CTA with half the rows of both operands in its
// shared memory.  With one CTA on a tile of 128 x 256 the operands' way from L2 bounds the kernel (48 KB a block and SM against 32).
// Small ones: one CTA walks tiles of 128 rows x 16 to 128 columns; where tiles are fewer than SMs the sums' length is cut into
// parts, by the CTAs of a cluster that add through their shared memory, or, for very long sums, through a workspace.
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

template <int kN> struct Shape {
    static constexpr int kSets = kN >= 128 ? 2 : 1;           // sets of four epilogue warps, each with its share of the columns
    static constexpr int kCols = kN / kSets;
    static constexpr int kEpiWarps = 4 * kSets, kProducer = kEpiWarps, kMma = kEpiWarps + 1;
    static constexpr int kThreads = (kEpiWarps + 2) * 32;
    static constexpr int kStageBytes = kStageA + kN * kBlockK;
    // up to 64 columns (few tokens): rings of which two fit an SM; of clusters of eight with one block an SM not all find a place at a time
    // (one row of 8192 by 2048: 15.0 us and 9.4)
    static constexpr int kStages = kN == 128 ? 5 : kN == 64 ? 3 : kN == 32 ? 4 : 5;
    static constexpr bool kBoxes = kN >= 64;
    static constexpr int kBuffers = 4;                        // of tensor memory
    static constexpr int kTmemCols = kN * kBuffers < 32 ? 32 : kN * kBuffers;
    static constexpr size_t kSmem = 1024 + (size_t)kStages * kStageBytes + (kBoxes ? kEpiWarps * kBoxBytes : 0);
};

// Tiles of a pair of CTAs: 256 x 256, 128 rows of each operand a CTA.
namespace pair {
constexpr int kN = 256, kRows = 256;
constexpr int kStageBytes = 2 * kStageA, kStages = 5, kBuffers = 2, kTmemCols = 512;
constexpr int kSets = 2, kCols = kN / kSets;
constexpr int kEpiWarps = 8, kProducer = 8, kMma = 9;         // warps 10 and 11 only give registers away
constexpr int kThreads = 12 * 32;
constexpr size_t kSmem = 1024 + (size_t)kStages * kStageBytes + kEpiWarps * kBoxBytes;
// Registers: 384 threads are launched with 168 each; 256 x 224 + 128 x 56 is the same sum, and so is 256 x 216 + 128 x 72
// (the kernel with scales for the columns: 4096x4096 over 16384 takes 477 us with the first and 441 with the second).
}

// Adds a piece of a row's block, kN columns, times the row's scale and the columns'.
template <int kN, bool kColumnScales>
__device__ __forceinline__ void add_scaled(uint64_t *sum, const uint32_t *r, uint64_t scale2, const float *cols)
{
#pragma unroll
    for (int j = 0; j < kN / 2; j += 2) {
        uint64_t f = scale2, g = scale2;
        if constexpr (kColumnScales) {
            const float4 c = *reinterpret_cast<const float4 *>(cols + 2 * j);
            f = mul2(f, pair_of(c.x, c.y));
            g = mul2(g, pair_of(c.z, c.w));
        }
        sum[j] = fma2(pair_of(r[2 * j], r[2 * j + 1]), f, sum[j]);
        sum[j + 1] = fma2(pair_of(r[2 * j + 2], r[2 * j + 3]), g, sum[j + 1]);
    }
}

// The scales of the next blocks on their way to shared memory, for one epilogue warp: of its rows (a lane's own), and either of its kCols
// columns or the one they share.  Asked for three blocks ahead: they come from L2, in 400 ns and more, and with the registers of one
// block ahead a block of few columns took as long as that (one row of 4096 by 4096: 11.2 us and 8.9).
constexpr int kAhead = 3, kScaleSlots = kAhead + 1;
template <int kCols, bool kColumnScales>
struct ScaleRing {
    static constexpr int kSlot = kColumnScales ? 32 + kCols : 64;                  // floats
    float *slots;
    const float *at_a, *at_b;
    long long ld_a, ld_b;
    bool has_b;
    int end;
    __device__ __forceinline__ void ask(int kb, int lane)
    {
        if (kb < end) {
            float *const slot = slots + (kb % kScaleSlots) * kSlot;
            cp_async_4(smem_u32(slot + lane), at_a + kb * ld_a);
            if constexpr (kColumnScales) {
                if (has_b) cp_async_16(smem_u32(slot + 32 + 4 * lane), at_b + kb * ld_b, 16u);
            } else
                cp_async_4(smem_u32(slot + 32 + lane), at_b + kb * ld_b);
        }
        cp_async_commit();
    }
    // Of a tile's row and columns, blocks [first, end_).
    __device__ __forceinline__ void start(const TileArgs &a, int row, int col0, int first, int end_, int lane)
    {
        // (rows behind the last 128 have no scales: they take another's, and nothing of theirs is stored)
        at_a = a.scale_a + (a.shift_a ? min(row, a.rows_a - 1) >> 7 : min(row, (int)a.scale_a_ld - 1));
        at_b = kColumnScales ? a.scale_b + col0 + 4 * lane : a.scale_b + min(col0 >> 7, (a.rows_b - 1) >> 7);
        has_b = 4 * lane < kCols && col0 + 4 * lane < a.scale_b_ld;
        ld_a = a.scale_a_ld;
        ld_b = a.scale_b_ld;
        end = end_;
        __syncwarp();                                         // the last tile's readers
        for (int i = 0; i < kAhead; ++i) ask(first + i, lane);
    }
    // The block's scales are there (and those of block kb + kAhead asked for).
    __device__ __forceinline__ const float *next(int kb, int lane)
    {
        __syncwarp();                                         // the slot's readers
        ask(kb + kAhead, lane);
        cp_async_wait<kAhead>();
        __syncwarp();
        return slots + (kb % kScaleSlots) * kSlot;
    }
};

// kColumnScales: B has a scale for each row (a column of the tile), else one for each 128.
template <typename T, int kN, bool kColumnScales>
__global__ void __launch_bounds__(Shape<kN>::kThreads, kN <= 64 ? 2 : 1)
block_matmul_kernel(const __grid_constant__ TileArgs a, const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b)
{
    using S = Shape<kN>;
    extern __shared__ unsigned char smem_raw[];
    __shared__ __align__(8) unsigned long long s_full[S::kStages], s_empty[S::kStages], s_tfull[S::kBuffers], s_tempty[S::kBuffers];
    __shared__ uint32_t s_tmem_base;
    __shared__ __align__(16) float s_scales[S::kEpiWarps][kScaleSlots * ScaleRing<S::kCols, kColumnScales>::kSlot];
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
    const int units = a.tiles_m * a.tiles_n * a.splits;

    if (warp == S::kProducer) {
        if (lane == 0) {
            int s = 0;
            long long issued = 0;
            uint32_t phase = 1;
            bool alive = true;
            for (int u = blockIdx.x; u < units && alive; u += gridDim.x) {
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
            if (!alive) {
                tc_dev_set_status(a.status, TC_ERR_TIMEOUT);
                // the copies in flight land before the block's shared memory goes to another
                const long long first = issued > S::kStages ? issued - S::kStages : 0;
                for (long long i = first; i < issued; ++i) mbar_wait_soon(smem_u32(&s_full[i % S::kStages]), (uint32_t)(i / S::kStages & 1));
            }
        }
    } else if (warp == S::kMma) {
        const uint32_t issuer = lane == 0 ? 1u : 0u;
        const uint32_t idesc = make_idesc_e4m3(kRowsM, kN);
        const uint64_t desc = make_smem_desc_sw128(ring, 1024);
        const uint32_t desc_lo = (uint32_t)desc, desc_hi = (uint32_t)(desc >> 32);
        int s = 0, b = 0;
        uint32_t phase = 0, tphase = 1;
        bool alive = true;
        for (int u = blockIdx.x; u < units && alive; u += gridDim.x) {
            const Unit t = unit_of(a, u);
            for (int kb = t.k_first; kb < t.k_end; ++kb) {
                if (!mbar_wait_soon(smem_u32(&s_tempty[b]), tphase) || !mbar_wait_soon(smem_u32(&s_full[s]), phase)) { alive = false; break; }
                tc_fence_after_sync();
                const uint32_t a_lo = desc_lo + (uint32_t)s * (S::kStageBytes >> 4), b_lo = a_lo + (kStageA >> 4);
#pragma unroll
                for (int q = 0; q < kBlockK / 32; ++q)
                    mma_e4m3_ss_guarded(tmem_base + b * kN, a_lo + 2 * q, desc_hi, b_lo + 2 * q, desc_hi, idesc, q ? 1u : 0u, issuer);
                mma_commit_guarded(smem_u32(&s_empty[s]), issuer);
                mma_commit_guarded(smem_u32(&s_tfull[b]), issuer);
                if (++s == S::kStages) { s = 0; phase ^= 1u; }
                if (++b == S::kBuffers) { b = 0; tphase ^= 1u; }
            }
        }
        if (!alive && issuer) tc_dev_set_status(a.status, TC_ERR_TIMEOUT);
    } else {
        constexpr int kPieces = S::kCols / 16;
        const int set = warp >> 2, wq = warp & 3;
        const int row_in_tile = wq * 32 + lane;
        ScaleRing<S::kCols, kColumnScales> scales;
        scales.slots = s_scales[warp];
        int b = 0;
        uint32_t tphase = 0;
        bool alive = true;
        for (int u = blockIdx.x; u < units && alive; u += gridDim.x) {
            const Unit t = unit_of(a, u);
            const int row = t.tile_m * kRowsM + row_in_tile, col0 = t.tile_n * kN + set * S::kCols;
            uint64_t sum[S::kCols / 2];
#pragma unroll
            for (int i = 0; i < S::kCols / 2; ++i) sum[i] = 0ull;
            if (u == (int)blockIdx.x) scales.start(a, row, col0, t.k_first, t.k_end, lane);
            for (int kb = t.k_first; kb < t.k_end; ++kb) {
                const float *const here = scales.next(kb, lane);
                const float scale = kColumnScales ? here[lane] : here[lane] * here[32 + lane];
                // (asked of the whole warp: what follows is done by all its lanes together)
                if (!__all_sync(0xffffffffu, mbar_wait_soon(smem_u32(&s_tfull[b]), tphase))) { alive = false; break; }
                tc_fence_after_sync();
                const uint32_t at = tmem_base + b * kN + set * S::kCols + ((uint32_t)(wq * 32) << 16);
                const uint64_t scale2 = pair_of(scale, scale);
                uint32_t r[2][16];
                tmem_ld_32x32b_x16(at, r[0]);
#pragma unroll
                for (int i = 0; i < kPieces; ++i) {
                    tmem_ld_wait(r[i & 1]);
                    if (i + 1 < kPieces) tmem_ld_32x32b_x16(at + 16 * (i + 1), r[(i + 1) & 1]);
                    else {
                        tc_fence_before_sync();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(smem_u32(&s_tempty[b]));
                    }
                    add_scaled<16, kColumnScales>(&sum[8 * i], r[i & 1], scale2, here + 32 + 16 * i);
                }
                if (++b == S::kBuffers) { b = 0; tphase ^= 1u; }
            }
            if (!alive) break;
            if (u + (int)gridDim.x < units) {                 // the next unit's scales are on their way while this one is stored
                const Unit next = unit_of(a, u + gridDim.x);
                scales.start(a, next.tile_m * kRowsM + row_in_tile, next.tile_n * kN + set * S::kCols, next.k_first, next.k_end, lane);
            }
            if (a.cluster) {
                // this part's sums in the ring, which the tensor cores are done with: [column][128 rows], or where a pixel's channels are neighbours
                // [row][kN + 4 columns]
                float *const parts = reinterpret_cast<float *>(smem_raw + (ring - smem_u32(smem_raw)));
                if (a.join_rows) {
                    float4 *dst = reinterpret_cast<float4 *>(parts + row_in_tile * (kN + 4) + set * S::kCols);
#pragma unroll
                    for (int i = 0; i < S::kCols / 4; ++i) {
                        float4 v;
                        halves(sum[2 * i], v.x, v.y);
                        halves(sum[2 * i + 1], v.z, v.w);
                        dst[i] = v;
                    }
                } else {
                    float *dst = parts + set * S::kCols * kRowsM + row_in_tile;
#pragma unroll
                    for (int i = 0; i < S::kCols / 2; ++i) {
                        float x, y;
                        halves(sum[i], x, y);
                        dst[(2 * i) * kRowsM] = x;
                        dst[(2 * i + 1) * kRowsM] = y;
                    }
                }
                break;                                        // a CTA has one part
            }
            if (a.partial) {
                float *dst = a.partial + ((long long)u * kN + set * S::kCols) * kRowsM + row_in_tile;
#pragma unroll
                for (int i = 0; i < S::kCols / 2; ++i) {
                    float x, y;
                    halves(sum[i], x, y);
                    dst[(2 * i) * kRowsM] = x;
                    dst[(2 * i + 1) * kRowsM] = y;
                }
                continue;
            }
            finish(a, sum, [&](int j) { return make_int2(row, col0 + 2 * j); });
            if constexpr (S::kBoxes) {
                if (a.by_rows) store_by_rows<T, S::kCols>(a, ring + S::kStages * S::kStageBytes + warp * kBoxBytes, sum, row - lane, col0, lane);
                else store_lanes<T, S::kCols>(a, sum, row, col0);
            } else
                store_lanes<T, S::kCols>(a, sum, row, col0);
            __syncwarp();
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
        // The cluster's CTAs each add their share of the rows (columns) over all parts, in the parts' order, four values at a time.
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
            float4 v[8];
#pragma unroll
            for (int part = 0; part < 8; ++part)
                if (part < a.splits)
                    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v[part].x), "=f"(v[part].y), "=f"(v[part].z), "=f"(v[part].w)
                                 : "r"(cluster_address(at, (uint32_t)part)));
            float r[4] = {v[0].x, v[0].y, v[0].z, v[0].w};
#pragma unroll
            for (int part = 1; part < 8; ++part)
                if (part < a.splits) { r[0] += v[part].x; r[1] += v[part].y; r[2] += v[part].z; r[3] += v[part].w; }
            const int row = t.tile_m * kRowsM + (a.join_rows ? line : 4 * four), col = t.tile_n * kN + (a.join_rows ? 4 * four : line);
            if (a.join_rows) store_four<T>(a, row, col, r);
            else
#pragma unroll
                for (int j = 0; j < 4; ++j) store_value<T>(a, row + j, col, r[j]);
        }
        cluster_sync();                                       // this block's shared memory is read no more
    }
}

// Adds the parts of a tile's sums in their order and writes the output.  Also the whole product where there is nothing to add.
template <typename T>
__global__ void __launch_bounds__(256) block_matmul_join_kernel(TileArgs a, int n)
{
    chain_next();
    chain_wait();
    const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
    const int row_in_tile = (int)(i & 127);
    const long long rest = i >> 7;
    const int tile = (int)(rest / n), col_in_tile = (int)(rest - (long long)tile * n);
    if (tile >= a.tiles_m * a.tiles_n) return;
    const int splits = a.splits;
    a.splits = 1;
    const Unit t = unit_of(a, tile);
    const int row = t.tile_m * kRowsM + row_in_tile, col = t.tile_n * n + col_in_tile;
    float v = 0.f;
    const float *src = a.partial + ((long long)tile * splits * n + col_in_tile) * kRowsM + row_in_tile;
    for (int s = 0; s < splits; ++s) v += src[(long long)s * n * kRowsM];
    store_value<T>(a, row, col, v);
}

// ---- pairs of CTAs -------------------------------------------------------------------------
template <typename T, bool kColumnScales>
__global__ void __launch_bounds__(pair::kThreads, 1)
block_matmul_pair_kernel(const __grid_constant__ TileArgs a, const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                         const __grid_constant__ CUtensorMap map_out)
{
    using namespace pair;
    extern __shared__ unsigned char smem_raw[];
    // s_full and s_tempty are the even CTA's: both CTAs' copies and epilogues report there; s_empty and s_tfull are each CTA's own.
    __shared__ __align__(8) unsigned long long s_full[kStages], s_empty[kStages], s_tfull[kBuffers], s_tempty[kBuffers];
    __shared__ uint32_t s_tmem_base;
    __shared__ __align__(16) float s_scales[kEpiWarps][kScaleSlots * ScaleRing<kCols, kColumnScales>::kSlot];
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
        if constexpr (kColumnScales) asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
        else asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
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
            const uint32_t idesc = make_idesc_e4m3(kRows, kN);
            const uint64_t desc = make_smem_desc_sw128(ring, 1024);
            const uint32_t desc_lo = (uint32_t)desc, desc_hi = (uint32_t)(desc >> 32);
            int s = 0, b = 0;
            uint32_t phase = 0, tphase = 1;
            bool alive = true;
            for (int u = blockIdx.x >> 1; u < units && alive; u += step) {
                for (int kb = 0; kb < a.k_blocks; ++kb) {
                    if (!mbar_wait_soon(smem_u32(&s_full[s]), phase) || !mbar_wait_soon(smem_u32(&s_tempty[b]), tphase)) { alive = false; break; }
                    tc_fence_after_sync();
                    const uint32_t a_lo = desc_lo + (uint32_t)s * (kStageBytes >> 4), b_lo = a_lo + (kStageA >> 4);
#pragma unroll
                    for (int q = 0; q < kBlockK / 32; ++q)
                        mma_e4m3_ss_pair_guarded(tmem_base + b * kN, a_lo + 2 * q, desc_hi, b_lo + 2 * q, desc_hi, idesc, q ? 1u : 0u, issuer);
                    mma_commit_pair_guarded(smem_u32(&s_tfull[b]), issuer);
                    mma_commit_pair_guarded(smem_u32(&s_empty[s]), issuer);
                    if (++s == kStages) { s = 0; phase ^= 1u; }
                    if (++b == kBuffers) { b = 0; tphase ^= 1u; }
                }
            }
            if (!alive && issuer) tc_dev_set_status(a.status, TC_ERR_TIMEOUT);
        }
        __syncwarp();
    } else {
        if constexpr (kColumnScales) asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");
        else asm volatile("setmaxnreg.inc.sync.aligned.u32 224;");
        const int set = warp >> 2, wq = warp & 3;
        ScaleRing<kCols, kColumnScales> scales;
        scales.slots = s_scales[warp];
        const uint32_t box = ring + kStages * kStageBytes + warp * kBoxBytes;
        uint32_t tempty[kBuffers];
#pragma unroll
        for (int b = 0; b < kBuffers; ++b) tempty[b] = cluster_address(smem_u32(&s_tempty[b]), 0);
        int b = 0;
        uint32_t tphase = 0;
        bool alive = true;
        // With scales for the columns a thread reads the fragments' layout, four rows and every fourth pair of columns: 32
        // columns' scales, where a row's thread has 128 to fetch, which shared memory's 128 bytes a cycle do not give in a block's time
        // (4096x4096 over 16384, not back to back: 442 us and 391 when it was made, 407 now).
        const int i = lane >> 2, q = lane & 3;                // row 8 k + i, columns 8 g + 2 q and the next
        for (int u = blockIdx.x >> 1; u < units && alive; u += step) {
            const Unit t = unit_of(a, u);
            const int first_row = t.tile_m * kRows + rank * kRowsM + wq * 32, col0 = t.tile_n * kN + set * kCols;
            uint64_t sum[kCols / 2];                          // of a row's columns, or [row k][32 columns' pairs]
#pragma unroll
            for (int j = 0; j < kCols / 2; ++j) sum[j] = 0ull;
            if (u == (int)(blockIdx.x >> 1)) scales.start(a, first_row + lane, col0, 0, a.k_blocks, lane);
            for (int kb = 0; kb < a.k_blocks; ++kb) {
                const float *const here = scales.next(kb, lane);
                uint64_t scale2[kColumnScales ? 4 : 1];
                if constexpr (kColumnScales) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) scale2[k] = pair_of(here[8 * k + i], here[8 * k + i]);
                } else {
                    const float scale = here[lane] * here[32 + lane];
                    scale2[0] = pair_of(scale, scale);
                }
                // (asked of the whole warp: what follows is done by all its lanes together)
                if (!__all_sync(0xffffffffu, mbar_wait_soon(smem_u32(&s_tfull[b]), tphase))) { alive = false; break; }
                tc_fence_after_sync();
                const uint32_t at = tmem_base + b * kN + set * kCols + ((uint32_t)(wq * 32) << 16);
                auto hand_back = [&] {
                    tc_fence_before_sync();
                    __syncwarp();
                    if (lane == 0) mbar_arrive_cluster(tempty[b]);
                };
                if constexpr (kColumnScales) {
                    uint32_t r[2][16];
                    uint64_t c[4];
                    tmem_ld_16x256b_x4(at, r[0]);
#pragma unroll
                    for (int n = 0; n < kCols / 16; ++n) {    // 32 columns, their first 16 rows, then their last
                        const int piece = n >> 1, half = n & 1;
                        if (half == 0)
#pragma unroll
                            for (int g = 0; g < 4; ++g) c[g] = *reinterpret_cast<const uint64_t *>(here + 32 + 32 * piece + 8 * g + 2 * q);
                        tmem_ld_wait(r[n & 1]);
                        if (n + 1 < kCols / 16) tmem_ld_16x256b_x4(at + 32 * ((n + 1) >> 1) + ((uint32_t)(16 * ((n + 1) & 1)) << 16), r[(n + 1) & 1]);
                        else hand_back();
#pragma unroll
                        for (int g = 0; g < 4; ++g)
#pragma unroll
                            for (int k = 0; k < 2; ++k) {
                                uint64_t &to = sum[(2 * half + k) * 16 + 4 * piece + g];
                                to = fma2(pair_of(r[n & 1][4 * g + 2 * k], r[n & 1][4 * g + 2 * k + 1]), mul2(c[g], scale2[2 * half + k]), to);
                            }
                    }
                } else {
                    uint32_t r[2][32];
                    tmem_ld_32x32b_x32(at, r[0]);
#pragma unroll
                    for (int n = 0; n < kCols / 32; ++n) {
                        tmem_ld_wait(r[n & 1]);
                        if (n + 1 < kCols / 32) tmem_ld_32x32b_x32(at + 32 * (n + 1), r[(n + 1) & 1]);
                        else hand_back();
                        add_scaled<32, false>(&sum[16 * n], r[n & 1], scale2[0], nullptr);
                    }
                }
                if (++b == kBuffers) { b = 0; tphase ^= 1u; }
            }
            if (!alive) break;
            if (u + step < units) {                           // the next tile's scales are on their way while this one is stored
                const Unit next = unit_of(a, u + step);
                scales.start(a, next.tile_m * kRows + rank * kRowsM + wq * 32 + lane, next.tile_n * kN + set * kCols, 0, a.k_blocks, lane);
            }
            finish(a, sum, [&](int j) {
                return kColumnScales ? make_int2(first_row + 8 * (j >> 4) + i, col0 + 8 * (j & 15) + 2 * q) : make_int2(first_row + lane, col0 + 2 * j);
            });
            if (a.by_rows) {
#pragma unroll
                for (int c = 0; c < kCols; c += kBoxCols<T>) {
                    if (a.store_tma && lane == 0) tma_store_wait_read();
                    __syncwarp();                             // the last box's readers
                    if constexpr (kColumnScales) {
#pragma unroll
                        for (int k = 0; k < 4; ++k)
#pragma unroll
                            for (int g = 0; g < kBoxCols<T> / 8; ++g) {
                                float x, y;
                                halves(sum[k * 16 + c / 8 + g], x, y);
                                const uint32_t byte = (uint32_t)(8 * g + 2 * q) * sizeof(T), to = box + (uint32_t)(8 * k + i) * 128u + (((byte >> 4) ^ i) << 4) + (byte & 15u);
                                if constexpr (sizeof(T) == 4) asm volatile("st.shared.v2.f32 [%0], {%1, %2};" ::"r"(to), "f"(x), "f"(y) : "memory");
                                else asm volatile("st.shared.u32 [%0], %1;" ::"r"(to), "r"(pack_bf16(x, y)) : "memory");
                            }
                    } else
                        fill_box<T>(box, sum + c / 2, lane);
                    if (a.store_tma) fence_proxy_async_smem();
                    __syncwarp();
                    if (first_row < a.rows_a && col0 + c < a.rows_b) {
                        if (!a.store_tma) store_box<T>(a, box, first_row, col0 + c, lane);
                        else if (lane == 0) tma_store_2d(&map_out, col0 + c, first_row, box);
                    }
                }
            } else if constexpr (kColumnScales) {
#pragma unroll
                for (int k = 0; k < 4; ++k)
#pragma unroll
                    for (int n = 0; n < 16; ++n) {
                        float v[2];
                        halves(sum[k * 16 + n], v[0], v[1]);
                        const int row = first_row + 8 * k + i, col = col0 + 8 * n + 2 * q;
#pragma unroll
                        for (int j = 0; j < 2; ++j)
                            if (row < a.rows_a && col + j < a.rows_b)
                                put((T *)a.out, pixel_at(a, a.swapped ? col + j : row) + (long long)(a.swapped ? row : col + j) * a.hw, v[j]);
                    }
            } else
                store_lanes<T, kCols>(a, sum, first_row + lane, col0);
            __syncwarp();
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

template <typename T, int kN, bool kColumnScales>
tc_status launch_tiles(const tc_ctx *ctx, const TileArgs &a, const CUtensorMap &map_a, const CUtensorMap &map_b, cudaStream_t s)
{
    constexpr auto kernel = block_matmul_kernel<T, kN, kColumnScales>;
    if (!allow_shared<kernel>(ctx->device, Shape<kN>::kSmem)) return TC_ERR_CUDA;
    const long long units = (long long)a.tiles_m * a.tiles_n * a.splits;
    const long long most = (kN <= 64 ? 2 : 1) * ctx->sm_count;
    const dim3 grid((unsigned int)(units < most || a.cluster ? units : most));
    return launch_first_cluster(a.cluster ? a.splits : 1, kernel, grid, dim3(Shape<kN>::kThreads), Shape<kN>::kSmem, s, a, map_a, map_b) == cudaSuccess ? TC_OK : TC_ERR_CUDA;
}

template <typename T, bool kColumnScales>
tc_status launch_pairs(const tc_ctx *ctx, const TileArgs &a, const CUtensorMap &map_a, const CUtensorMap &map_b, const CUtensorMap &map_out, cudaStream_t s)
{
    constexpr auto kernel = block_matmul_pair_kernel<T, kColumnScales>;
    if (!allow_shared<kernel>(ctx->device, pair::kSmem)) return TC_ERR_CUDA;
    const long long units = (long long)a.tiles_m * a.tiles_n, pairs = ctx->sm_count / 2;
    const dim3 grid((unsigned int)(2 * (units < pairs ? units : pairs)));
    return launch_first_cluster(2, kernel, grid, dim3(pair::kThreads), pair::kSmem, s, a, map_a, map_b, map_out) == cudaSuccess ? TC_OK : TC_ERR_CUDA;
}

template <typename T>
tc_status launch(const tc_ctx *ctx, const TileArgs &a, bool pairs, int n, const CUtensorMap &map_a, const CUtensorMap &map_b, const CUtensorMap &map_out, cudaStream_t s)
{
    const bool cols = a.shift_b == 0;
    if (pairs) return cols ? launch_pairs<T, true>(ctx, a, map_a, map_b, map_out, s) : launch_pairs<T, false>(ctx, a, map_a, map_b, map_out, s);
    switch (n) {
    case 16: return cols ? launch_tiles<T, 16, true>(ctx, a, map_a, map_b, s) : TC_ERR_UNSUPPORTED;
    case 32: return cols ? launch_tiles<T, 32, true>(ctx, a, map_a, map_b, s) : TC_ERR_UNSUPPORTED;
    case 64: return cols ? launch_tiles<T, 64, true>(ctx, a, map_a, map_b, s) : launch_tiles<T, 64, false>(ctx, a, map_a, map_b, s);
    case 128: return cols ? launch_tiles<T, 128, true>(ctx, a, map_a, map_b, s) : launch_tiles<T, 128, false>(ctx, a, map_a, map_b, s);
    default: return TC_ERR_UNSUPPORTED;                       // (no plan has it: a tile's size is a kernel's)
    }
}

}  // namespace

MatmulPlan tc_plan_matmul(const MatmulArgs &a, int sm_count)
{
    MatmulPlan best;
    const int k_blocks = (a.cols + kBlockK - 1) / kBlockK;
    double best_cost = 0.0;
    auto consider = [&](bool swapped, bool pairs, int n, int splits) {
        const MatmulOperand &m = swapped ? a.channels : a.pixels, &c = swapped ? a.pixels : a.channels;
        const int rows = pairs ? pair::kRows : kRowsM, workers = pairs ? sm_count / 2 : sm_count;
        const long long tiles = (long long)((m.rows + rows - 1) / rows) * ((c.rows + n - 1) / n);
        // Clusters run all at once: two blocks an SM with up to 64 columns, one with 128, of which clusters of more than four do not all
        // find a place (512x512 over 8192: 22.6 us in eight parts, 14.2 in six).
        const bool cluster = splits > 1 && splits <= 8;
        const long long units = tiles * splits;
        if (splits > 1 && (splits * 2 > k_blocks + 1 || (cluster ? units > (n <= 64 ? 2 : 1) * sm_count || (n > 64 && splits > 4) : units > sm_count))) return;
        const double rounds = cluster ? std::max(1.0, (double)units / sm_count) : (double)((units + workers - 1) / workers);
        // Cycles, fitted to the times of 130 forced plans: of a block (its operands from L2, or its sums), of a tile (its store, dearest where its
        // columns lie apart in memory), of joining parts.
        const double block = pairs ? (c.square ? 1100 : 1430) : std::max(600 + 3.4 * n, c.square ? 0.0 : 300 + 7.2 * n);
        const bool by_rows = swapped ? a.hw > 1 : a.hw == 1;
        const double store = splits > 1 ? 8 * n : by_rows ? (pairs ? 6000 : n >= 64 ? 25 * n : 60 * n) : pairs ? 30000 : n == 128 ? 110 * n : 180 * n;
        const double cost = rounds * ((double)((k_blocks + splits - 1) / splits) * block + 600 + store) +
                            (cluster ? 5000 + n * 22 : splits > 1 ? 9000 + (double)units * n * 0.5 : 0);
        if (best.n == 0 || cost < best_cost) {
            best_cost = cost;
            best.swapped = swapped;
            best.pairs = pairs;
            best.n = n;
            best.splits = splits;
            best.cluster = cluster;
            best.tiles = tiles;
            best.workspace = splits > 1 && !cluster ? (size_t)tiles * splits * n * kRowsM * sizeof(float) : 0;
        }
    };
    for (int swapped = 0; swapped < 2; ++swapped) {
        for (int n = 16; n <= 128; n *= 2)
            if (n >= 64 || (swapped && !a.pixels.square))
                for (const int splits : {1, 2, 3, 4, 6, 8, 16, 32, 64, 128}) consider(swapped, false, n, splits);
        if (sm_count > 1) consider(swapped, true, pair::kN, 1);
    }
    if (k_blocks == 0) { best.splits = 0; best.pairs = best.cluster = false; best.workspace = 0; }
    return best;
}

tc_status tc_launch_matmul_blocks(const tc_ctx *ctx, const MatmulArgs &m, const MatmulPlan &plan, void *workspace, cudaStream_t s)
{
    const MatmulOperand &ra = plan.swapped ? m.channels : m.pixels, &rb = plan.swapped ? m.pixels : m.channels;
    TileArgs a{};
    a.rows_a = ra.rows;
    a.rows_b = rb.rows;
    a.k_blocks = (m.cols + kBlockK - 1) / kBlockK;
    a.splits = plan.splits;
    const int rows_tile = plan.pairs ? pair::kRows : kRowsM;
    a.tiles_m = (ra.rows + rows_tile - 1) / rows_tile;
    a.group = plan.pairs ? 8 : 16;
    a.cluster = plan.cluster;
    a.by_rows = plan.swapped ? m.hw > 1 : m.hw == 1;
    a.join_rows = a.by_rows && !plan.swapped;
    a.tiles_n = (rb.rows + plan.n - 1) / plan.n;
    a.scale_a = ra.m.scales;
    a.scale_b = rb.m.scales;
    a.scale_a_ld = ra.m.scale_ld;
    a.scale_b_ld = rb.m.scale_ld;
    a.shift_a = ra.square ? 7 : 0;
    a.shift_b = rb.square ? 7 : 0;
    a.swapped = plan.swapped;
    a.out_channels = m.channels.rows;
    a.hw = m.hw;
    a.relu = m.relu;
    // bytes that a store by rows moves: neighbouring channels of a pixel, or pixels of a map
    const int line = m.hw == 1 ? m.channels.rows : m.hw, size = m.dtype == TC_BF16 ? 2 : 4;
    a.vec = !a.by_rows ? 0 : line * size % 16 == 0 && ((uintptr_t)m.out & 15u) == 0 ? 16 : line * size % 8 == 0 && ((uintptr_t)m.out & 7u) == 0 ? 8 : 0;
    a.bias = m.bias;
    a.out = m.out;
    a.partial = plan.workspace ? (float *)workspace : nullptr;
    a.status = m.status;
    if (plan.splits > 0) {
        CUtensorMap map_a, map_b, map_out{};
        if (!tc_tensor_map_codes(&map_a, ra.m.codes, ra.rows, m.cols, ra.m.ld, kRowsM) ||
            !tc_tensor_map_codes(&map_b, rb.m.codes, rb.rows, m.cols, rb.m.ld, plan.pairs ? kRowsM : plan.n)) return TC_ERR_CUDA;
        a.store_tma = plan.pairs && a.vec == 16 && m.hw == 1 && tc_tensor_map_rows(&map_out, m.out, m.dtype, a.rows_a, a.rows_b, 32);
        const tc_status st = m.dtype == TC_BF16 ? launch<__nv_bfloat16>(ctx, a, plan.pairs, plan.n, map_a, map_b, map_out, s) : launch<float>(ctx, a, plan.pairs, plan.n, map_a, map_b, map_out, s);
        if (st != TC_OK || !a.partial) return st;
    }
    const long long values = (long long)a.tiles_m * a.tiles_n * plan.n * kRowsM;
    const dim3 grid((unsigned int)((values + 255) / 256));
    const cudaError_t err = m.dtype == TC_BF16 ? launch_chained(plan.splits > 0, block_matmul_join_kernel<__nv_bfloat16>, grid, dim3(256), 0, s, a, plan.n)
                                               : launch_chained(plan.splits > 0, block_matmul_join_kernel<float>, grid, dim3(256), 0, s, a, plan.n);
    return err == cudaSuccess ? TC_OK : TC_ERR_CUDA;
}
