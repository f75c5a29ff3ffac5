// tc_matmul_blocks: product of two block-scaled e4m3 matrices,
//
//   out[p][o] = act(bias[o] + sum_kb sa[p][kb] sb[o][kb] sum_{k in block kb} a[p][k] b[o][k])
//
// A block of 128 codes is one row of a 128-byte swizzle atom, so a stage of the ring is a block: four MMAs of 32 codes
// leave its sum in tensor memory, the epilogue's warps read it back, multiply it by the block's scales and add it to sums in
// registers (fp32), while the MMAs of the next blocks fill the other buffers.  One CTA an SM walks tiles of 128 rows x
// up to 256 columns.
#include "device_utils.cuh"
#include "sm100_ptx.cuh"
#include "tc_internal.h"

namespace {

using namespace tcdev;
using namespace sm100;

constexpr int kBlockK = 128;
constexpr int kRowsM = 128;
constexpr int kStageA = kRowsM * kBlockK;
constexpr int kRing = 196608;                                 // bytes of the ring at most

template <int kN> struct Shape {
    static constexpr int kSets = kN >= 128 ? 2 : 1;           // sets of four epilogue warps, each with its share of the columns
    static constexpr int kCols = kN / kSets;
    static constexpr int kEpiWarps = 4 * kSets, kProducer = kEpiWarps, kMma = kEpiWarps + 1;
    static constexpr int kThreads = (kEpiWarps + 2) * 32;
    static constexpr int kStageBytes = kStageA + kN * kBlockK;
    static constexpr int kStages = kRing / kStageBytes > 10 ? 10 : kRing / kStageBytes;
    static constexpr int kBuffers = kN == 256 ? 2 : 4;        // of tensor memory
    static constexpr int kTmemCols = kN * kBuffers < 32 ? 32 : kN * kBuffers;
    static constexpr size_t kSmem = 1024 + (size_t)kStages * kStageBytes;
};

struct TileArgs {
    int rows_a, rows_b;               // of the MMA's operands
    int k_blocks, splits;
    int tiles_m, tiles_n;
    const float *scale_a, *scale_b;
    long long scale_a_ld, scale_b_ld;
    int shift_a, shift_b;             // 0: a scale for each row, 7: for each 128
    int swapped;
    int out_channels, hw, relu, vec;
    const float *bias;
    void *out;
    float *partial;                   // [unit][column][128 rows], where the length is split
    unsigned int *status;
};

__device__ __forceinline__ uint64_t pair_of(float a, float b)
{
    uint64_t v;
    asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(a), "f"(b));
    return v;
}
__device__ __forceinline__ uint64_t pair_of(uint32_t a, uint32_t b)
{
    uint64_t v;
    asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "r"(a), "r"(b));
    return v;
}
__device__ __forceinline__ void halves(uint64_t v, float &a, float &b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c)
{
    uint64_t d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b)
{
    uint64_t d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}

struct Unit {
    int tile_m, tile_n, k_first, k_end;
};
// Units in the order they are worked on: the parts of a tile's length one after the other; tiles in columns of 16 tile rows, so
// that the SMs' operands at any time are few rows of both matrices.
__device__ __forceinline__ Unit unit_of(const TileArgs &a, int u)
{
    const int tile = u / a.splits, split = u - tile * a.splits;
    constexpr int kGroup = 16;
    const int per_group = kGroup * a.tiles_n, g = tile / per_group, rest = tile - g * per_group;
    const int high = min(kGroup, a.tiles_m - g * kGroup);
    Unit r;
    r.tile_n = rest / high;
    r.tile_m = g * kGroup + rest - r.tile_n * high;
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

// kCols: B has a scale for each row (a column of the tile), else one for each 128.
template <typename T, int kN, bool kColumnScales>
__global__ void __launch_bounds__(Shape<kN>::kThreads, 1)
block_matmul_kernel(const __grid_constant__ TileArgs a, const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b)
{
    using S = Shape<kN>;
    extern __shared__ unsigned char smem_raw[];
    __shared__ __align__(8) unsigned long long s_full[S::kStages], s_empty[S::kStages], s_tfull[S::kBuffers], s_tempty[S::kBuffers];
    __shared__ uint32_t s_tmem_base;
    __shared__ __align__(16) float s_scale[kColumnScales ? S::kEpiWarps : 1][2][kColumnScales ? S::kCols : 4];
    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
    const uint32_t ring = (smem_u32(smem_raw) + 1023u) & ~1023u;
    chain_next();
    if (tid == 0) {
        for (int s = 0; s < S::kStages; ++s) { mbar_init(smem_u32(&s_full[s]), 1); mbar_init(smem_u32(&s_empty[s]), 1); }
        for (int b = 0; b < S::kBuffers; ++b) { mbar_init(smem_u32(&s_tfull[b]), 1); mbar_init(smem_u32(&s_tempty[b]), S::kEpiWarps); }
        mbar_fence_init();
    }
    if (warp == S::kMma) { tmem_alloc(smem_u32(&s_tmem_base), S::kTmemCols); tmem_relinquish(); }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
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
                    if (!mbar_wait(smem_u32(&s_empty[s]), phase)) { alive = false; break; }
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
                for (long long i = first; i < issued; ++i) mbar_wait(smem_u32(&s_full[i % S::kStages]), (uint32_t)(i / S::kStages & 1));
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
                if (!mbar_wait(smem_u32(&s_tempty[b]), tphase) || !mbar_wait(smem_u32(&s_full[s]), phase)) { alive = false; break; }
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
        float(*const scales)[kColumnScales ? S::kCols : 4] = s_scale[kColumnScales ? warp : 0];
        int b = 0;
        uint32_t tphase = 0;
        bool alive = true;
        for (int u = blockIdx.x; u < units && alive; u += gridDim.x) {
            const Unit t = unit_of(a, u);
            const int row = t.tile_m * kRowsM + row_in_tile, col0 = t.tile_n * kN + set * S::kCols;
            uint64_t sum[S::kCols / 2];
#pragma unroll
            for (int i = 0; i < S::kCols / 2; ++i) sum[i] = 0ull;
            // the scales of a block are asked for while the block before it is added
            const float *at_a = a.scale_a + (row >> a.shift_a);
            const float *at_b = kColumnScales ? a.scale_b + col0 + 4 * lane : a.scale_b + min(col0 >> 7, (a.rows_b - 1) >> 7);
            const bool has_b = kColumnScales && 4 * lane < S::kCols && col0 + 4 * lane < a.scale_b_ld;
            float next_a = 0.f, next_b = 0.f;
            float4 next_cols = make_float4(0.f, 0.f, 0.f, 0.f);
            auto ask = [&](int kb) {
                next_a = at_a[kb * a.scale_a_ld];
                if constexpr (kColumnScales) {
                    if (has_b) next_cols = *reinterpret_cast<const float4 *>(at_b + kb * a.scale_b_ld);
                } else
                    next_b = at_b[kb * a.scale_b_ld];
            };
            if (t.k_first < t.k_end) ask(t.k_first);
            for (int kb = t.k_first; kb < t.k_end; ++kb) {
                const float scale = kColumnScales ? next_a : next_a * next_b;
                float *const cols = scales[kColumnScales ? kb & 1 : 0];
                if constexpr (kColumnScales) {
                    if (4 * lane < S::kCols) *reinterpret_cast<float4 *>(cols + 4 * lane) = next_cols;
                    __syncwarp();
                }
                if (kb + 1 < t.k_end) ask(kb + 1);
                // (asked of the whole warp: what follows is done by all its lanes together)
                if (!__all_sync(0xffffffffu, mbar_wait(smem_u32(&s_tfull[b]), tphase, 20u))) { alive = false; break; }
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
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const uint64_t v = pair_of(r[i & 1][2 * j], r[i & 1][2 * j + 1]);
                        uint64_t f = scale2;
                        if constexpr (kColumnScales) f = mul2(f, *reinterpret_cast<const uint64_t *>(cols + 16 * i + 2 * j));
                        sum[8 * i + j] = fma2(v, f, sum[8 * i + j]);
                    }
                }
                if (++b == S::kBuffers) { b = 0; tphase ^= 1u; }
            }
            if (!alive) break;
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
            if (row < a.rows_a) {
                T *const out = (T *)a.out;
                const float floor_v = a.relu ? 0.f : __int_as_float((int)0xff800000u);
                const int cols_here = min(S::kCols, a.rows_b - col0);
                if (!a.swapped) {
                    long long dst = pixel_at(a, row) + (long long)col0 * a.hw;
                    if (a.vec && cols_here == S::kCols) {
                        constexpr int kPer = 16 / (int)sizeof(T);
    #pragma unroll
                        for (int i = 0; i < S::kCols; i += kPer) {
                            float v[kPer];
    #pragma unroll
                            for (int j = 0; j < kPer; j += 2) {
                                halves(sum[(i + j) / 2], v[j], v[j + 1]);
                                if (a.bias) { v[j] += a.bias[col0 + i + j]; v[j + 1] += a.bias[col0 + i + j + 1]; }
                                // (a NaN stays one: a comparison with it fails)
                                v[j] = v[j] < floor_v ? floor_v : v[j];
                                v[j + 1] = v[j + 1] < floor_v ? floor_v : v[j + 1];
                            }
                            __align__(16) T w[kPer];
    #pragma unroll
                            for (int j = 0; j < kPer; ++j) put(w, j, v[j]);
                            *reinterpret_cast<uint4 *>(out + dst + i) = *reinterpret_cast<const uint4 *>(w);
                        }
                    } else {
    #pragma unroll
                        for (int i = 0; i < S::kCols / 2; ++i) {
                            float x, y;
                            halves(sum[i], x, y);
                            if (2 * i < cols_here) {
                                if (a.bias) x += a.bias[col0 + 2 * i];
                                put(out, dst + (long long)(2 * i) * a.hw, x < floor_v ? floor_v : x);
                            }
                            if (2 * i + 1 < cols_here) {
                                if (a.bias) y += a.bias[col0 + 2 * i + 1];
                                put(out, dst + (long long)(2 * i + 1) * a.hw, y < floor_v ? floor_v : y);
                            }
                        }
                    }
                } else {
                    const float bias = a.bias ? a.bias[row] : 0.f;
                    const long long ch = (long long)row * a.hw;
    #pragma unroll
                    for (int i = 0; i < S::kCols / 2; ++i) {
                        float v[2];
                        halves(sum[i], v[0], v[1]);
    #pragma unroll
                        for (int j = 0; j < 2; ++j)
                            if (2 * i + j < cols_here) {
                                const float x = v[j] + bias;
                                put(out, ch + pixel_at(a, col0 + 2 * i + j), x < floor_v ? floor_v : x);
                            }
                    }
                }
            }
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
    if (row >= a.rows_a || col >= a.rows_b) return;
    float v = 0.f;
    const float *src = a.partial + ((long long)tile * splits * n + col_in_tile) * kRowsM + row_in_tile;
    for (int s = 0; s < splits; ++s) v += src[(long long)s * n * kRowsM];
    const int p = a.swapped ? col : row, o = a.swapped ? row : col;
    if (a.bias) v += a.bias[o];
    if (a.relu && v < 0.f) v = 0.f;
    put((T *)a.out, pixel_at(a, p) + (long long)o * a.hw, v);
}

template <typename T, int kN, bool kColumnScales>
tc_status launch_tiles(const tc_ctx *ctx, const TileArgs &a, const CUtensorMap &map_a, const CUtensorMap &map_b, cudaStream_t s)
{
    auto *kernel = block_matmul_kernel<T, kN, kColumnScales>;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Shape<kN>::kSmem) != cudaSuccess) { cudaGetLastError(); return TC_ERR_CUDA; }
    const long long units = (long long)a.tiles_m * a.tiles_n * a.splits;
    const dim3 grid((unsigned int)(units < ctx->sm_count ? units : ctx->sm_count));
    return launch_first(true, kernel, grid, dim3(Shape<kN>::kThreads), Shape<kN>::kSmem, s, a, map_a, map_b) == cudaSuccess ? TC_OK : TC_ERR_CUDA;
}

template <typename T>
tc_status launch(const tc_ctx *ctx, const TileArgs &a, int n, const CUtensorMap &map_a, const CUtensorMap &map_b, cudaStream_t s)
{
    const bool cols = a.shift_b == 0;
    switch (n) {
    case 16: return cols ? launch_tiles<T, 16, true>(ctx, a, map_a, map_b, s) : TC_ERR_UNSUPPORTED;
    case 32: return cols ? launch_tiles<T, 32, true>(ctx, a, map_a, map_b, s) : TC_ERR_UNSUPPORTED;
    case 64: return cols ? launch_tiles<T, 64, true>(ctx, a, map_a, map_b, s) : launch_tiles<T, 64, false>(ctx, a, map_a, map_b, s);
    case 128: return cols ? launch_tiles<T, 128, true>(ctx, a, map_a, map_b, s) : launch_tiles<T, 128, false>(ctx, a, map_a, map_b, s);
    default: return cols ? launch_tiles<T, 256, true>(ctx, a, map_a, map_b, s) : launch_tiles<T, 256, false>(ctx, a, map_a, map_b, s);
    }
}

}  // namespace

MatmulPlan tc_plan_matmul(const MatmulArgs &a, int sm_count)
{
    MatmulPlan best;
    const int k_blocks = (a.cols + kBlockK - 1) / kBlockK;
    double best_cost = 0.0;
    for (int swapped = 0; swapped < 2; ++swapped) {
        const MatmulOperand &m = swapped ? a.channels : a.pixels, &c = swapped ? a.pixels : a.channels;
        for (int n = 16; n <= 256; n *= 2) {
            if (n < 64 && (!swapped || c.square)) continue;
            const long long tiles = (long long)((m.rows + kRowsM - 1) / kRowsM) * ((c.rows + n - 1) / n);
            int splits = 1;
            if (tiles * 2 <= sm_count && k_blocks > 1) splits = (int)(sm_count / tiles < (k_blocks + 1) / 2 ? sm_count / tiles : (k_blocks + 1) / 2);
            const long long rounds = (tiles * splits + sm_count - 1) / sm_count;
            // a block's cycles: its operands from L2, or its sums; a tile's: its store
            const double load = (kRowsM + n) * 2.6, add = n * (c.square ? 2.2 : 4.2);
            const double cost = (double)rounds * ((double)((k_blocks + splits - 1) / splits) * (load > add ? load : add) + 600 + 8 * n) +
                                (splits > 1 ? 3000 + (double)tiles * splits * n * 0.5 : 0);
            if (best.n == 0 || cost < best_cost) {
                best_cost = cost;
                best.swapped = swapped;
                best.n = n;
                best.splits = splits;
                best.tiles = tiles;
                best.workspace = splits > 1 ? (size_t)tiles * splits * n * kRowsM * sizeof(float) : 0;
            }
        }
    }
    if (k_blocks == 0) { best.splits = 0; best.workspace = 0; }
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
    a.tiles_m = (ra.rows + kRowsM - 1) / kRowsM;
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
    a.vec = m.hw == 1 && !plan.swapped && ((uintptr_t)m.out & 15u) == 0 && m.channels.rows % (m.dtype == TC_BF16 ? 8 : 4) == 0;
    a.bias = m.bias;
    a.out = m.out;
    a.partial = plan.splits != 1 ? (float *)workspace : nullptr;
    a.status = m.status;
    if (plan.splits > 0) {
        CUtensorMap map_a, map_b;
        if (!tc_tensor_map_codes(&map_a, ra.m.codes, ra.rows, m.cols, ra.m.ld, kRowsM) ||
            !tc_tensor_map_codes(&map_b, rb.m.codes, rb.rows, m.cols, rb.m.ld, plan.n)) return TC_ERR_CUDA;
        const tc_status st = m.dtype == TC_BF16 ? launch<__nv_bfloat16>(ctx, a, plan.n, map_a, map_b, s) : launch<float>(ctx, a, plan.n, map_a, map_b, s);
        if (st != TC_OK || plan.splits == 1) return st;
    }
    const long long values = (long long)a.tiles_m * a.tiles_n * plan.n * kRowsM;
    const dim3 grid((unsigned int)((values + 255) / 256));
    const cudaError_t err = m.dtype == TC_BF16 ? launch_chained(plan.splits > 0, block_matmul_join_kernel<__nv_bfloat16>, grid, dim3(256), 0, s, a, plan.n)
                                               : launch_chained(plan.splits > 0, block_matmul_join_kernel<float>, grid, dim3(256), 0, s, a, plan.n);
    return err == cudaSuccess ? TC_OK : TC_ERR_CUDA;
}
