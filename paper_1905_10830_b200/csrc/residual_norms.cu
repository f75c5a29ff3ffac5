// tc_residual_norms and its gradient: the norm after a block, its gate and scale, the residual sum and the norm before the
// next block, in one pass over the maps.
//
//   q = 1 / sqrt(mean_c y^2 + eps), n = y q, u = n after;  s = h + scale gate u;  r = 1 / sqrt(mean_c s^2 + eps), x = s r before
//
// and, with t = dx before, m = mean_c t s, D = ds + r t - s r^3 m, g = gate, v = scale D g after:
//
//   dh = D;  dy = q (v - n mean_c v n);  dbefore = sum_p dx s r;  dafter = scale sum_p D g n;  dgate = scale D u;  dscale = sum D g u
//
// Bound by the bytes of the maps: each is read once and written once.  The gradient's mean_c v n is a sum of D's three parts, so
// that all sums over a pixel's channels -- s s, t s, y y, and ds, t and s times g after y -- are taken together and
// a pixel waits for one reduction.  Sums are fp32, in an order that does not depend on the launch's timing; sums over the pixels are first
// taken by block, and a second kernel adds the blocks' sums in their order.  scale's gradient, a sum over all values, carries what its additions round
// off within a block, and its blocks' parts are added in fp64.
#include "block_codes.cuh"
#include "sm100_ptx.cuh"
#include "tc_internal.h"

namespace {

using namespace tcdev;
using namespace blk;

__device__ __forceinline__ float inv_sqrt(float v) { return rsqrtf(v); }       // (off by 2^-22 at most)

// ---- single pixels (H W = 1): a pixel's channels are a row in memory ------------------------------
// kThreadsRow threads a row, kV chunks of eight channels a thread; rows of one warp share a block of eight, and aligned ones of up to 128 channels a
// warp (a warp each, 200000x64 in bf16: 72 us and 22, gradient 151 and 51).
// Rows that cannot be moved 16 bytes at a time (kVec false): a thread's eight values lie 32 apart, so that a warp's are neighbours.
template <int kThreadsRow>
__device__ __forceinline__ int chunk_at(int t, int i) { return (i * kThreadsRow + t) * 8; }
template <int kThreadsRow, bool kVec>
__device__ __forceinline__ int value_at(int t, int i, int j)
{
    return kVec ? chunk_at<kThreadsRow>(t, i) + j : i * kThreadsRow * 8 + (t >> 5) * 256 + j * 32 + (t & 31);
}
template <typename T, int kThreadsRow, bool kVec>
__device__ __forceinline__ void load_values(Raw8<T> &r, const T *row, int t, int i, int c)
{
    zero8(r);
    if constexpr (kVec) {
        const int k = chunk_at<kThreadsRow>(t, i);
        if (k < c) load8(r, row + k);
    } else {
        uint32_t h[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int k = value_at<kThreadsRow, false>(t, i, j);
            h[j] = 0u;
            if (k < c) {
                if constexpr (sizeof(T) == 2) h[j] = reinterpret_cast<const unsigned short *>(row)[k];
                else h[j] = reinterpret_cast<const uint32_t *>(row)[k];
            }
        }
        if constexpr (sizeof(T) == 2) r.v = make_uint4(h[0] | h[1] << 16, h[2] | h[3] << 16, h[4] | h[5] << 16, h[6] | h[7] << 16);
        else { r.v = make_uint4(h[0], h[1], h[2], h[3]); r.w = make_uint4(h[4], h[5], h[6], h[7]); }
    }
}
template <int kThreadsRow, bool kVec>
__device__ __forceinline__ void load_weights(float (&f)[8], const float *v, int t, int i, int c)
{
    if constexpr (kVec) {
        const int k = chunk_at<kThreadsRow>(t, i);
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = 0.f;
        if (k < c) {
            const float4 a = reinterpret_cast<const float4 *>(v + k)[0], b = reinterpret_cast<const float4 *>(v + k)[1];
            f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int k = value_at<kThreadsRow, false>(t, i, j);
            f[j] = k < c ? v[k] : 0.f;
        }
    }
}
template <typename T, int kThreadsRow, bool kVec>
__device__ __forceinline__ void store_values(T *row, const float (&f)[8], int t, int i, int c)
{
    if constexpr (kVec) {
        const int k = chunk_at<kThreadsRow>(t, i);
        if (k < c) store8(row + k, f);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int k = value_at<kThreadsRow, false>(t, i, j);
            if (k < c) store1(row + k, f[j]);
        }
    }
}

template <int kThreadsRow>
__device__ __forceinline__ float row_sum(float v, float *s_part)
{
    constexpr int kWarps = kThreadsRow / 32;
#pragma unroll
    for (int d = kThreadsRow < 32 ? kThreadsRow / 2 : 16; d; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    if constexpr (kWarps > 1) {
        const int lane = threadIdx.x & 31;
        if (lane == 0) s_part[threadIdx.x >> 5] = v;
        __syncthreads();
        v = s_part[lane % kWarps];
#pragma unroll
        for (int d = kWarps / 2; d; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    }
    return v;
}

// Codes of a thread's eight values of a row: 16 threads' are a block, or four of each of a warp's.
template <int kThreadsRow, bool kVec>
__device__ __forceinline__ void store_codes(const BlockMatrix &to, const float (&x)[8], long long row, int t, int i, int c)
{
    uint8_t *const codes = to.codes + row * to.ld;
    if constexpr (kVec) {
        const int k = chunk_at<kThreadsRow>(t, i);
        uint32_t m = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) m = max(m, abs_bits(x[j]));
        const float scale = scale_of(max_over<kThreadsRow < 16 ? kThreadsRow : 16>(m));
        if (k >= c) return;
        *reinterpret_cast<uint2 *>(codes + k) = codes8(x, __frcp_rn(scale));
        if ((t & 15) == 0) to.scales[(long long)(k / kBlock) * to.scale_ld + row] = scale;
    } else {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int k = value_at<kThreadsRow, false>(t, i, 4 * h);
            uint32_t m = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) m = max(m, abs_bits(x[4 * h + j]));
            const float scale = scale_of(__reduce_max_sync(0xffffffffu, m));
            const uint32_t four = codes4(x[4 * h], x[4 * h + 1], x[4 * h + 2], x[4 * h + 3], __frcp_rn(scale));
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (k + 32 * j < c) codes[k + 32 * j] = (uint8_t)(four >> 8 * j);
            if ((t & 31) == 0 && k < c) to.scales[(long long)(k / kBlock) * to.scale_ld + row] = scale;
        }
    }
}

template <typename T, int kThreadsRow, int kV, bool kVec>
__global__ void __launch_bounds__(kThreadsRow <= 32 ? 256 : kThreadsRow) norm_rows_kernel(NormArgs a)
{
    constexpr int kRows = kThreadsRow <= 32 ? 256 / kThreadsRow : 1;
    __shared__ float s_part[2][kThreadsRow <= 32 ? 1 : kThreadsRow / 32];
    chain_next();
    chain_wait();
    const int t = threadIdx.x % kThreadsRow;
    const long long row = (long long)blockIdx.x * kRows + (kRows > 1 ? threadIdx.x / kThreadsRow : 0);
    if (kThreadsRow >= 32 && row >= a.pixels) return;         // whole warps; with more than one a row, whole blocks
    const int c = kThreadsRow < 32 && row >= a.pixels ? 0 : a.c;                   // (of several rows of a warp each has its lanes' share of its sums to take)
    const long long base = row * a.c;
    Raw8<T> rh[kV], ry[kV], rg[kV];
#pragma unroll
    for (int i = 0; i < kV; ++i) {
        load_values<T, kThreadsRow, kVec>(rh[i], (const T *)a.h + base, t, i, c);
        if (a.y) load_values<T, kThreadsRow, kVec>(ry[i], (const T *)a.y + base, t, i, c);
        if (a.gate_map) load_values<T, kThreadsRow, kVec>(rg[i], (const T *)a.gate_map + base, t, i, c);
    }
    float s[kV][8];
#pragma unroll
    for (int i = 0; i < kV; ++i) values8(rh[i], s[i]);
    const float inv_c = 1.0f / (float)a.c;
    if (a.y) {
        float q = 1.f;
        if (a.after) {
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < kV; ++i) {
                float y[8];
                values8(ry[i], y);
#pragma unroll
                for (int j = 0; j < 8; ++j) sum = fmaf(y[j], y[j], sum);
            }
            q = inv_sqrt(fmaf(row_sum<kThreadsRow>(sum, s_part[0]), inv_c, a.eps));
        }
        const float scale = a.scale ? *a.scale : 1.f;
#pragma unroll
        for (int i = 0; i < kV; ++i) {
            float u[8];
            values8(ry[i], u);
            if (a.after) {
                float w[8];
                load_weights<kThreadsRow, kVec>(w, a.after, t, i, c);
#pragma unroll
                for (int j = 0; j < 8; ++j) u[j] = u[j] * q * w[j];
            }
            if (a.gate_map || a.gate) {
                float g[8];
                if (a.gate_map) values8(rg[i], g);
                else load_weights<kThreadsRow, kVec>(g, a.gate, t, i, c);
#pragma unroll
                for (int j = 0; j < 8; ++j) u[j] *= g[j];
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) s[i][j] = fmaf(scale, u[j], s[i][j]);
            store_values<T, kThreadsRow, kVec>((T *)a.sum + base, s[i], t, i, c);
        }
    }
    if (!a.before) return;
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < kV; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) sum = fmaf(s[i][j], s[i][j], sum);
    const float r = inv_sqrt(fmaf(row_sum<kThreadsRow>(sum, s_part[1]), inv_c, a.eps));
#pragma unroll
    for (int i = 0; i < kV; ++i) {
        float w[8];
        load_weights<kThreadsRow, kVec>(w, a.before, t, i, c);
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = s[i][j] * r * w[j];
        if (a.x) store_values<T, kThreadsRow, kVec>((T *)a.x + base, w, t, i, c);
        if (a.codes.codes) store_codes<kThreadsRow, kVec>(a.codes, w, row, t, i, c);
    }
}

// ---- rows on their way to shared memory ------------------------------------------------------
// Long rows: a block walks rows gridDim.x apart, whose parts of all inputs one thread brings to a ring in shared memory by bulk
// copies, several rows ahead, so that the memory is at work while the block waits for a row's sums (with a row's loads in
// registers, and the vectors read again for each row: gradient of 16384x4096 in bf16 278 us and 158, forward 113 and 107).
constexpr int kRingInputs = 5, kRingStages = 8;
constexpr size_t kRingSm = 200 * 1024;                        // of an SM's shared memory, for all its blocks' rings
struct RowRing {
    const char *in[kRingInputs];      // compact: input i is part i of a stage
    int inputs, stages;
    uint32_t part_bytes;              // of a stage for one input
    uint32_t row_bytes;
    long long rows;
};
// Rows that do not begin at a multiple of 16 bytes (kVec false; the inputs do) come with the bytes around them up to one, and are read
// value by value from where they begin: the gradient only (16000x4095 in bf16 419 us without the ring and 225; the forward, whose
// instructions bound it with such rows, 40000x1001 106 and 111).
template <bool kVec>
struct RowReader {
    uint32_t ring;
    unsigned long long *full;         // [kRingStages]
    int *brought;                     // rows asked for so far (the first thread's)
    bool alive;
    // The block's next row to a slot that its readers are done with, by the first thread, as long as that is alive: the slot's last copy has landed.
    __device__ __forceinline__ void bring(const RowRing &r, long long row, int slot)
    {
        using namespace sm100;
        ++*brought;
        const uint32_t bar = smem_u32(full + slot), to = ring + (uint32_t)(slot * r.inputs) * r.part_bytes;
        const long long first = row * r.row_bytes, from = first & ~15ll;
        uint32_t bytes = r.row_bytes;
        if constexpr (!kVec) {
            bytes = (uint32_t)(first - from) + r.row_bytes;
            if (row + 1 < r.rows) bytes = (bytes + 15u) & ~15u;
            else {                                            // nothing behind the last row is touched: its last values are copied by hand
                const uint32_t whole = bytes & ~15u;
                for (int i = 0; i < r.inputs; ++i)
                    for (uint32_t at = whole; at < bytes; at += 2)
                        asm volatile("st.shared.u16 [%0], %1;" ::"r"(to + (uint32_t)i * r.part_bytes + at), "h"(*reinterpret_cast<const unsigned short *>(r.in[i] + from + at)) : "memory");
                bytes = whole;
            }
        }
        mbar_arrive_expect_tx(bar, bytes * (uint32_t)r.inputs);
        for (int i = 0; i < r.inputs; ++i) bulk_load(to + (uint32_t)i * r.part_bytes, r.in[i] + from, bytes, bar);
    }
    // The block's first rows; ends with the block in step.
    __device__ __forceinline__ void start(const RowRing &r, long long rows)
    {
        using namespace sm100;
        if (threadIdx.x == 0) {
            *brought = 0;
            for (int i = 0; i < r.stages; ++i) mbar_init(smem_u32(full + i), 1);
            mbar_fence_init();
            for (int i = 0; i < r.stages && blockIdx.x + (long long)i * gridDim.x < rows; ++i) bring(r, blockIdx.x + (long long)i * gridDim.x, i);
        }
        alive = true;
        __syncthreads();
    }
    // Where the block's `turn`-th row, which is row `at` of all, lies, once it has come.
    __device__ __forceinline__ uint32_t row(const RowRing &r, long long at, int turn, int slot, unsigned int *status)
    {
        if (alive && !sm100::mbar_wait_soon(sm100::smem_u32(full + slot), (uint32_t)(turn / r.stages & 1))) {
            alive = false;                                    // (no wait is waited for twice)
            tc_dev_set_status(status, TC_ERR_TIMEOUT);
        }
        return ring + (uint32_t)(slot * r.inputs) * r.part_bytes + (kVec ? 0u : (uint32_t)(at * r.row_bytes & 15));
    }
    // Behind the last row: where a wait ran out, the copies in flight land before the block's shared memory goes to another.
    __device__ __forceinline__ void finish(const RowRing &r)
    {
        if (threadIdx.x != 0 || alive) return;
        for (int i = max(0, *brought - r.stages); i < *brought; ++i) sm100::mbar_wait_soon(sm100::smem_u32(full + i % r.stages), (uint32_t)(i / r.stages & 1));
    }
};
__device__ __forceinline__ uint4 lds16(uint32_t at)
{
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
    return v;
}
__device__ __forceinline__ void load8_shared(Raw8<__nv_bfloat16> &r, uint32_t at) { r.v = lds16(at); }
__device__ __forceinline__ void load8_shared(Raw8<float> &r, uint32_t at) { r.v = lds16(at); r.w = lds16(at + 16); }

// A thread's i-th eight values of the row at `at`.
template <typename T, int kThreadsRow, bool kVec>
__device__ __forceinline__ void load_shared(Raw8<T> &r, uint32_t at, int t, int i, int c)
{
    zero8(r);
    if constexpr (kVec) {
        const int k = chunk_at<kThreadsRow>(t, i);
        if (k < c) load8_shared(r, at + (uint32_t)k * sizeof(T));
    } else {
        uint32_t h[8];
        const int k = value_at<kThreadsRow, false>(t, i, 0);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            h[j] = 0u;
            if (k + 32 * j < c) {
                if constexpr (sizeof(T) == 2) {
                    unsigned short v;
                    asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(at + 2u * (uint32_t)(k + 32 * j)) : "memory");
                    h[j] = v;
                } else
                    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(h[j]) : "r"(at + 4u * (uint32_t)(k + 32 * j)) : "memory");
            }
        }
        if constexpr (sizeof(T) == 2) r.v = make_uint4(h[0] | h[1] << 16, h[2] | h[3] << 16, h[4] | h[5] << 16, h[6] | h[7] << 16);
        else { r.v = make_uint4(h[0], h[1], h[2], h[3]); r.w = make_uint4(h[4], h[5], h[6], h[7]); }
    }
}

template <typename T, int kWarps, int kV>
__global__ void __launch_bounds__(kWarps * 32, 16 / kWarps) norm_rows_ring_kernel(const __grid_constant__ NormArgs a, const __grid_constant__ RowRing r)
{
    constexpr int kThreadsRow = kWarps * 32;
    extern __shared__ __align__(16) unsigned char s_ring[];
    __shared__ __align__(8) unsigned long long s_full[kRingStages];
    __shared__ int s_brought;
    __shared__ float s_part[2][kWarps];
    chain_next();
    chain_wait();
    const int t = threadIdx.x;
    RowReader<true> reader;
    reader.ring = sm100::smem_u32(s_ring);
    reader.full = s_full;
    reader.brought = &s_brought;
    reader.start(r, a.pixels);
    const float inv_c = 1.0f / (float)a.c, scale = a.scale ? *a.scale : 1.f;
    float wy[kV][8], wx[kV][8];                               // after times the channels' gate; before
#pragma unroll
    for (int i = 0; i < kV; ++i) {
        float g[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) wy[i][j] = wx[i][j] = g[j] = 1.f;
        if (a.after) load_weights<kThreadsRow, true>(wy[i], a.after, t, i, a.c);
        if (a.gate) load_weights<kThreadsRow, true>(g, a.gate, t, i, a.c);
        if (a.before) load_weights<kThreadsRow, true>(wx[i], a.before, t, i, a.c);
#pragma unroll
        for (int j = 0; j < 8; ++j) wy[i][j] *= g[j];
    }
    int turn = 0, slot = 0;
    for (long long row = blockIdx.x; row < a.pixels; row += gridDim.x, ++turn) {
        const long long base = row * a.c;
        const uint32_t at = reader.row(r, row, turn, slot, a.status);
        Raw8<T> rh[kV], ry[kV], rg[kV];
        float sum = 0.f, s[kV][8];
#pragma unroll
        for (int i = 0; i < kV; ++i) {
            load_shared<T, kThreadsRow, true>(rh[i], at, t, i, a.c);
            load_shared<T, kThreadsRow, true>(ry[i], at + r.part_bytes, t, i, a.c);
            if (a.gate_map) load_shared<T, kThreadsRow, true>(rg[i], at + 2 * r.part_bytes, t, i, a.c);
            float y[8];
            values8(ry[i], y);
#pragma unroll
            for (int j = 0; j < 8; ++j) sum = fmaf(y[j], y[j], sum);
        }
        sum = row_sum<kThreadsRow>(sum, s_part[0]);                // (the block is in step here: all have read the slot)
        if (threadIdx.x == 0 && reader.alive && row + (long long)r.stages * gridDim.x < a.pixels) reader.bring(r, row + (long long)r.stages * gridDim.x, slot);
        const float f = (a.after ? inv_sqrt(fmaf(sum, inv_c, a.eps)) : 1.f) * scale;
        sum = 0.f;
#pragma unroll
        for (int i = 0; i < kV; ++i) {
            float y[8];
            values8(ry[i], y);
            values8(rh[i], s[i]);
            if (a.gate_map) {
                float g[8];
                values8(rg[i], g);
#pragma unroll
                for (int j = 0; j < 8; ++j) y[j] *= g[j];
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                s[i][j] = fmaf(f, y[j] * wy[i][j], s[i][j]);
                sum = fmaf(s[i][j], s[i][j], sum);
            }
            store_values<T, kThreadsRow, true>((T *)a.sum + base, s[i], t, i, a.c);
        }
        if (a.before) {
            const float rr = inv_sqrt(fmaf(row_sum<kThreadsRow>(sum, s_part[1]), inv_c, a.eps));
#pragma unroll
            for (int i = 0; i < kV; ++i) {
                float x[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] = s[i][j] * rr * wx[i][j];
                if (a.x) store_values<T, kThreadsRow, true>((T *)a.x + base, x, t, i, a.c);
                if (a.codes.codes) store_codes<kThreadsRow, true>(a.codes, x, row, t, i, a.c);
            }
        } else
            __syncthreads();                                  // the row's partial sums are read before the next row's are written
        if (++slot == r.stages) slot = 0;
    }
    reader.finish(r);
}

// ---- maps: a pixel's channels lie H W apart ------------------------------------------------------
// 32 pixels a block, a lane for each; of each block of 128 channels a warp takes 16.  The maps are read again for each of the
// passes (sums of y, of s, the output), from L1 and L2.
template <typename T>
__global__ void __launch_bounds__(256) norm_maps_kernel(NormArgs a)
{
    __shared__ float s_part[2][8][32];
    __shared__ uint32_t s_max[2][8][32];
    chain_next();
    chain_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const long long p = (long long)blockIdx.x * 32 + lane;
    const bool ok = p < a.pixels;
    const long long img = p / a.hw, base = img * a.c * (long long)a.hw + (p - img * a.hw);
    const T *h = (const T *)a.h + base, *y = a.y ? (const T *)a.y + base : nullptr, *gm = a.gate_map ? (const T *)a.gate_map + base : nullptr;
    const float scale = a.y && a.scale ? *a.scale : 1.f, inv_c = 1.0f / (float)a.c;
    auto over = [&](float (&part)[8][32], float v) {
        part[warp][lane] = v;
        __syncthreads();
        v = 0.f;
#pragma unroll
        for (int w = 0; w < 8; ++w) v += part[w][lane];
        return v;
    };
    float q = 1.f;
    auto sum_at = [&](int ch) {
        const long long at = (long long)ch * a.hw;
        float s = load1(h + at);
        if (y) {
            float u = load1(y + at) * q;
            if (a.after) u *= a.after[ch];
            if (gm) u *= load1(gm + at);
            else if (a.gate) u *= a.gate[ch];
            s = fmaf(scale, u, s);
        }
        return s;
    };
    if (y && a.after) {
        float sum = 0.f;
        for (int c0 = warp * 16; c0 < a.c; c0 += kBlock) {
            float v[16];
#pragma unroll
            for (int j = 0; j < 16; ++j) v[j] = ok && c0 + j < a.c ? load1(y + (long long)(c0 + j) * a.hw) : 0.f;
#pragma unroll
            for (int j = 0; j < 16; ++j) sum = fmaf(v[j], v[j], sum);
        }
        q = inv_sqrt(fmaf(over(s_part[0], sum), inv_c, a.eps));
    }
    float sum = 0.f;
    for (int c0 = warp * 16; c0 < a.c; c0 += kBlock) {
        float v[16];
#pragma unroll
        for (int j = 0; j < 16; ++j) v[j] = ok && c0 + j < a.c ? sum_at(c0 + j) : 0.f;
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            sum = fmaf(v[j], v[j], sum);
            if (y && ok && c0 + j < a.c) store1((T *)a.sum + base + (long long)(c0 + j) * a.hw, v[j]);
        }
    }
    if (!a.before) return;
    const float r = inv_sqrt(fmaf(over(s_part[1], sum), inv_c, a.eps));
    int turn = 0;
    for (int b0 = 0; b0 < a.c; b0 += kBlock, turn ^= 1) {
        const int c0 = b0 + warp * 16;
        float v[16];
        uint32_t m = 0;
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            v[j] = 0.f;
            if (ok && c0 + j < a.c) v[j] = sum_at(c0 + j) * r * a.before[c0 + j];
            m = max(m, abs_bits(v[j]));
        }
        if (a.x) {
#pragma unroll
            for (int j = 0; j < 16; ++j)
                if (ok && c0 + j < a.c) store1((T *)a.x + base + (long long)(c0 + j) * a.hw, v[j]);
        }
        if (a.codes.codes) {
            s_max[turn][warp][lane] = m;
            __syncthreads();                                  // (the other half's readers are past this barrier before it is written again)
#pragma unroll
            for (int w = 0; w < 8; ++w) m = max(m, s_max[turn][w][lane]);
            const float sc = scale_of(m), inv = __frcp_rn(sc);
            if (ok && c0 < a.c)
                *reinterpret_cast<uint4 *>(a.codes.codes + p * a.codes.ld + c0) = make_uint4(
                    codes4(v[0], v[1], v[2], v[3], inv), codes4(v[4], v[5], v[6], v[7], inv), codes4(v[8], v[9], v[10], v[11], inv), codes4(v[12], v[13], v[14], v[15], inv));
            if (ok && warp == 0) a.codes.scales[(long long)(b0 / kBlock) * a.codes.scale_ld + p] = sc;
        }
    }
}

// The same with all channels of a tile of kPx pixels in shared memory, where they fit: each value is fetched once, many at a time, and
// the vectors once a block (256x14x14 x 1024, bf16: 970 us and 138, the gradient 516 and 239).  A lane has two pixels, whose values one instruction works on, and
// eight channels in a row of every kStep.
constexpr size_t kTileSm = 220 * 1024, kTileStatic = 14 * 1024;       // of an SM's shared memory; what a block has beside its tile
template <typename T, int kPx, int kWarps>
struct MapTile {
    static constexpr int kThreads = 32 * kWarps, kPairs = kPx / 2, kSubs = 32 / kPairs, kStep = 8 * kSubs * kWarps;
    // Eight channels' rows lie together, a row apart from the next eight's where rows are shorter than 128 bytes: lanes that read rows eight
    // apart read them in different banks.
    static constexpr int kEight = 8 * kPx + (kPx * (int)sizeof(T) < 128 ? kPx : 0);
    static __host__ __device__ constexpr int values(int c8) { return c8 / 8 * kEight; }
    static __device__ __forceinline__ int row(int c) { return (c >> 3) * kEight + (c & 7) * kPx; }
    // Of a tile's eight rows (from a channel that is a multiple of eight on, at this lane's pixels) the j-th's two values.
    static __device__ __forceinline__ const T *eight(const T *tile, int c0, int pair) { return tile + (c0 >> 3) * kEight + 2 * pair; }
    static __device__ __forceinline__ uint64_t load(const T *rows, int j)
    {
        if constexpr (sizeof(T) == 2) {
            const uint32_t w = *reinterpret_cast<const uint32_t *>(rows + j * kPx);
            return pair_of(w << 16, w & 0xffff0000u);
        } else
            return *reinterpret_cast<const uint64_t *>(rows + j * kPx);
    }
    // A tensor's pixels p0 ..., four at a time; zeros behind the last.
    static __device__ __forceinline__ void fill_quads(T *dst, const T *src, uint32_t p0, uint32_t pixels, int c, int hw)
    {
        using namespace sm100;
        constexpr int kQuads = kPx / 4, kRows = kThreads / kQuads;            // (rows a multiple of eight: each step is as far)
        const int t = threadIdx.x, ch0 = t / kQuads;
        const uint32_t p = p0 + t % kQuads * 4, img = p / (uint32_t)hw, bytes = p < pixels ? 4u * sizeof(T) : 0u;
        const T *from = bytes ? src + (long long)img * c * hw + (p - img * (uint32_t)hw) + (long long)ch0 * hw : src;
        const long long step = bytes ? (long long)kRows * hw : 0;
        uint32_t to = smem_u32(dst + row(ch0) + t % kQuads * 4);
#pragma unroll 4
        for (int ch = ch0; ch < c; ch += kRows, from += step, to += kRows / 8 * kEight * (int)sizeof(T)) {
            if constexpr (sizeof(T) == 2) cp_async_8(to, from, bytes);
            else cp_async_16(to, from, bytes);
        }
    }
    // The same of all inputs a pixel at a time, to planes one after the other.  Values of two bytes have no asynchronous copy: they come through
    // registers, as many of all inputs at a time as there is room for.
    template <int kInputs>
    static __device__ __forceinline__ void fill(T *dst, int plane, const void *const (&src)[kInputs], uint32_t p0, uint32_t pixels, int c, int hw)
    {
        using namespace sm100;
        const int t = threadIdx.x;
        constexpr int kRows = kThreads / kPx, kBatch = 6;
        const int ch0 = t / kPx;
        const uint32_t p = p0 + t % kPx, img = p / (uint32_t)hw;
        const bool ok = p < pixels;
        long long at = (long long)img * c * hw + (p - img * (uint32_t)hw) + (long long)ch0 * hw;
        for (int ch = ch0; ch < c; ch += kBatch * kRows, at += (long long)kBatch * kRows * hw) {
            T v[kInputs][kBatch];
            T *to = dst + t % kPx;
#pragma unroll
            for (int n = 0; n < kInputs; ++n) {
                if (!src[n]) continue;
#pragma unroll
                for (int i = 0; i < kBatch; ++i) {
                    const T *const from = (const T *)src[n] + at + (long long)(kRows * i) * hw;
                    if constexpr (sizeof(T) == 2) {
                        v[n][i] = T(0.f);
                        if (ok && ch + kRows * i < c) v[n][i] = *from;
                    } else if (ch + kRows * i < c) {
                        if (ok) cp_async_4(smem_u32(to + row(ch + kRows * i)), reinterpret_cast<const float *>(from));
                        else to[row(ch + kRows * i)] = T(0.f);
                    }
                }
                if constexpr (sizeof(T) == 4) to += plane;
            }
            if constexpr (sizeof(T) == 2)
#pragma unroll
                for (int n = 0; n < kInputs; ++n) {
                    if (!src[n]) continue;
#pragma unroll
                    for (int i = 0; i < kBatch; ++i)
                        if (ch + kRows * i < c) to[row(ch + kRows * i)] = v[n][i];
                    to += plane;
                }
        }
    }
    // Sum over the block's lanes that share this lane's pixels.
    static __device__ __forceinline__ uint64_t over_block(float2 (*part)[kPairs], uint64_t v)
    {
        float x, y;
        halves(v, x, y);
#pragma unroll
        for (int d = kPairs; d < 32; d *= 2) {
            x += __shfl_xor_sync(0xffffffffu, x, d);
            y += __shfl_xor_sync(0xffffffffu, y, d);
        }
        const int lane = threadIdx.x & 31;
        if (lane < kPairs) part[threadIdx.x >> 5][lane] = make_float2(x, y);
        __syncthreads();
        x = y = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            const float2 q = part[w][lane % kPairs];
            x += q.x;
            y += q.y;
        }
        return pair_of(x, y);
    }
};
// Where a lane's two pixels lie in a map, and how they are written: one store for both where they are neighbours at an even place.
struct MapPixels {
    long long at0, at1;
    bool ok0, ok1, both;
    __device__ __forceinline__ MapPixels(uint32_t p, uint32_t pixels, int c, int hw, bool pairs)
    {
        ok0 = p < pixels;
        ok1 = p + 1 < pixels;
        const uint32_t img = p / (uint32_t)hw, in = p - img * (uint32_t)hw;
        at0 = (long long)img * c * hw + in;
        at1 = in + 1 == (uint32_t)hw ? (long long)(img + 1) * c * hw : at0 + 1;
        both = pairs && ok1;
    }
};
// Eight channels of them, from c0 on, those there are.
template <typename T>
struct MapRows {
    T *to0;
    long long apart;
    int hw, there;
    bool ok0, ok1, both;
    __device__ __forceinline__ MapRows(T *map, const MapPixels &px, int c0, int c, int hw_) : hw(hw_), ok0(px.ok0), ok1(px.ok1), both(px.both)
    {
        to0 = map + px.at0 + (long long)c0 * hw_;
        apart = px.at1 - px.at0;
        there = c - c0;
    }
    __device__ __forceinline__ void store1of(int j, float x, float y) const
    {
        T *const to = to0 + (long long)j * hw;
        if (both) {
            if constexpr (sizeof(T) == 2) *reinterpret_cast<uint32_t *>(to) = pack_bf16(x, y);
            else *reinterpret_cast<float2 *>(to) = make_float2(x, y);
        } else {
            if (ok0) store1(to, x);
            if (ok1) store1(to + apart, y);
        }
    }
    // Channels j0 ... j0 + 3: with one test for all of them where they are all there (a test for each took as many instructions as the values).
    __device__ __forceinline__ void store4(int j0, const uint64_t (&v)[4]) const
    {
        float x[4], y[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) halves(v[j], x[j], y[j]);
        if (both && there >= 8) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                T *const to = to0 + (long long)(j0 + j) * hw;
                if constexpr (sizeof(T) == 2) *reinterpret_cast<uint32_t *>(to) = pack_bf16(x[j], y[j]);
                else *reinterpret_cast<float2 *>(to) = make_float2(x[j], y[j]);
            }
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (j0 + j < there) store1of(j0 + j, x[j], y[j]);
        }
    }
};
// Each channel's vector value twice, as it multiplies two pixels.
__device__ __forceinline__ void weights8(uint64_t (&f)[8], const uint64_t *v)
{
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const ulonglong2 w = reinterpret_cast<const ulonglong2 *>(v)[j];
        f[2 * j] = w.x;
        f[2 * j + 1] = w.y;
    }
}
__device__ __forceinline__ void fill_weights(uint64_t *wy, uint64_t *wx, const float *after, const float *gate, const float *before, int c, int c8)
{
    for (int i = threadIdx.x; i < c8; i += blockDim.x) {
        const float y = i < c ? (after ? after[i] : 1.f) * (gate ? gate[i] : 1.f) : 0.f, x = i < c && before ? before[i] : 0.f;
        wy[i] = pair_of(y, y);
        wx[i] = pair_of(x, x);
    }
}

// Zeros in the rows of channels that there are not.
template <typename M, typename T>
__device__ __forceinline__ void zero_rows(T *tiles, int inputs, int plane, int c, int c8, int px)
{
    for (int n = 0; n < inputs; ++n)
        for (int i = threadIdx.x; i < (c8 - c) * px; i += blockDim.x) tiles[n * plane + M::row(c + i / px) + i % px] = T(0.f);
}

template <typename T, int kPx, int kWarps>
__global__ void __launch_bounds__(32 * kWarps, 24 / kWarps) norm_maps_tile_kernel(const __grid_constant__ NormArgs a, int vec, int pairs)
{
    using M = MapTile<T, kPx, kWarps>;
    extern __shared__ __align__(16) unsigned char s_tile[];   // with c8 channels, c rounded up to eight: after times the channels' gate, before; h, y, gate [c8][kPx]
    __shared__ float2 s_part[2][kWarps][M::kPairs];
    __shared__ uint2 s_max[2][kWarps][M::kPairs];
    const int c8 = (a.c + 7) & ~7;
    uint64_t *const wy = reinterpret_cast<uint64_t *>(s_tile), *const wx = wy + c8;
    const int plane = M::values(c8);
    T *const sh = reinterpret_cast<T *>(wx + c8), *const sy = sh + plane, *const sg = sy + (a.y ? plane : 0);
    chain_next();
    chain_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, pair = lane % M::kPairs, slice = warp * M::kSubs + lane / M::kPairs;
    fill_weights(wy, wx, a.after, a.gate, a.before, a.c, c8);
    zero_rows<M>(sh, 1 + (a.y != nullptr) + (a.gate_map != nullptr), plane, a.c, c8, kPx);
    const float scale = a.scale ? *a.scale : 1.f, inv_c = 1.0f / (float)a.c;
    const long long tiles = (a.pixels + kPx - 1) / kPx;
    for (long long tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const uint32_t p0 = (uint32_t)tile * kPx, pixels = (uint32_t)a.pixels;
        const long long p = (long long)p0 + 2 * pair;
        const MapPixels px((uint32_t)p, pixels, a.c, a.hw, pairs);
        __syncthreads();                                      // the last tile's readers
        if (vec) {
            M::fill_quads(sh, (const T *)a.h, p0, pixels, a.c, a.hw);
            if (a.y) M::fill_quads(sy, (const T *)a.y, p0, pixels, a.c, a.hw);
            if (a.gate_map) M::fill_quads(sg, (const T *)a.gate_map, p0, pixels, a.c, a.hw);
        } else {
            const void *const inputs[] = {a.h, a.y, a.gate_map};
            M::fill(sh, plane, inputs, p0, pixels, a.c, a.hw);
        }
        sm100::cp_async_wait_all();
        __syncthreads();
        uint64_t f = pair_of(scale, scale);
        if (a.y && a.after) {
            uint64_t sum = 0ull;
            for (int c0 = slice * 8; c0 < a.c; c0 += M::kStep) {
                const T *const y = M::eight(sy, c0, pair);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const uint64_t v = M::load(y, j);
                    sum = fma2(v, v, sum);
                }
            }
            float x, y;
            halves(M::over_block(s_part[0], sum), x, y);
            f = pair_of(scale * inv_sqrt(fmaf(x, inv_c, a.eps)), scale * inv_sqrt(fmaf(y, inv_c, a.eps)));
        }
        // s of eight channels from c0 on
        auto sums_at = [&](int c0, uint64_t (&v)[8]) {
            const T *const h = M::eight(sh, c0, pair), *const y = M::eight(sy, c0, pair), *const g = M::eight(sg, c0, pair);
            if (!a.y) {
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = M::load(h, j);
                return;
            }
            weights8(v, wy + c0);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = mul2(M::load(y, j), v[j]);
            if (a.gate_map)
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = mul2(v[j], M::load(g, j));
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = fma2(f, v[j], M::load(h, j));
        };
        uint64_t sum = 0ull;
        for (int c0 = slice * 8; c0 < a.c; c0 += M::kStep) {
            uint64_t v[8];
            sums_at(c0, v);
            const MapRows<T> to((T *)a.sum, px, c0, a.c, a.hw);
#pragma unroll
            for (int j = 0; j < 8; ++j) sum = fma2(v[j], v[j], sum);
            if (a.y) {
                to.store4(0, {v[0], v[1], v[2], v[3]});
                to.store4(4, {v[4], v[5], v[6], v[7]});
            }
        }
        if (!a.before) continue;
        float rx, ry;
        halves(M::over_block(s_part[1], sum), rx, ry);
        const uint64_t r = pair_of(inv_sqrt(fmaf(rx, inv_c, a.eps)), inv_sqrt(fmaf(ry, inv_c, a.eps)));
        int turn = 0;
        for (int b0 = 0; b0 < a.c; b0 += M::kStep, turn ^= 1) {                    // (the same for all lanes: the codes' barrier)
            const int c0 = b0 + slice * 8;
            uint64_t v[8];
            uint32_t m0 = 0, m1 = 0;
            if (c0 < a.c) {
                uint64_t w[8];
                sums_at(c0, v);
                weights8(w, wx + c0);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = mul2(mul2(v[j], r), w[j]);
                if (a.x) {
                    const MapRows<T> to((T *)a.x, px, c0, a.c, a.hw);
                    to.store4(0, {v[0], v[1], v[2], v[3]});
                    to.store4(4, {v[4], v[5], v[6], v[7]});
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    float x, y;
                    halves(v[j], x, y);
                    m0 = max(m0, abs_bits(x));
                    m1 = max(m1, abs_bits(y));
                }
            }
            if (a.codes.codes) {
                constexpr int kBlockWarps = kPx == 64 ? kWarps : kWarps * kBlock / M::kStep; // warps whose slices are a block of 128 (tiles of 64 pixels: up to 64 channels)
#pragma unroll
                for (int d = M::kPairs; d < 32; d *= 2) {
                    m0 = max(m0, __shfl_xor_sync(0xffffffffu, m0, d));
                    m1 = max(m1, __shfl_xor_sync(0xffffffffu, m1, d));
                }
                if (lane < M::kPairs) s_max[turn][warp][lane] = make_uint2(m0, m1);
                __syncthreads();                              // (the other half's readers are past this barrier before it is written again)
#pragma unroll
                for (int w = 0; w < kBlockWarps; ++w) {
                    const uint2 q = s_max[turn][warp / kBlockWarps * kBlockWarps + w][pair];
                    m0 = max(m0, q.x);
                    m1 = max(m1, q.y);
                }
                if (c0 < a.c) {
                    const float sc0 = scale_of(m0), sc1 = scale_of(m1);
                    float x[8], y[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) halves(v[j], x[j], y[j]);
                    uint8_t *const to = a.codes.codes + p * a.codes.ld + c0;
                    float *const scales = a.codes.scales + (long long)(c0 / kBlock) * a.codes.scale_ld + p;
                    if (px.ok0) {
                        *reinterpret_cast<uint2 *>(to) = codes8(x, __frcp_rn(sc0));
                        if (c0 % kBlock == 0) scales[0] = sc0;
                    }
                    if (px.ok1) {
                        *reinterpret_cast<uint2 *>(to + a.codes.ld) = codes8(y, __frcp_rn(sc1));
                        if (c0 % kBlock == 0) scales[1] = sc1;
                    }
                }
            }
        }
    }
}

// ---- gradient ----------------------------------------------------------------------------------
constexpr int kMostChannels = 16384;
constexpr int kSums = 6;        // s s, t s, y y, and ds, t, s times gate after y

// What a pixel's sums give.
struct PixelFactors {
    float r, m, q, mean;        // D = ds + r (t - s r m);  dy = q (v - y q mean)
    float e;                    // sum D gate n after: the pixel's part of scale's gradient
};
// Values are multiplied by r and by q first, one factor after the other: products of two or three factors leave fp32's range long before the values
// do (r^3 of values above 1e13 is subnormal, of those below 1e-13 infinite).
// A sum of one value a pixel that carries what its additions round off: scale's gradient is a sum over all values of the maps, whose terms cancel and long
// chains of fp32 additions showed in it.
struct CarriedSum {
    float sum = 0.f, off = 0.f;
    __device__ __forceinline__ void add(float v)
    {
        const float w = v - off, t = sum + w;
        off = fabsf(t) <= 3.4e38f ? (t - sum) - w : 0.f;      // (infinities stay ones)
        sum = t;
    }
    __device__ __forceinline__ float value() const { return sum - off; }
};
__device__ __forceinline__ PixelFactors pixel_factors(const float (&sums)[kSums], const NormGradArgs &a, float scale)
{
    const float inv_c = 1.0f / (float)a.c;
    PixelFactors f;
    f.r = a.before ? inv_sqrt(fmaf(sums[0], inv_c, a.eps)) : 0.f;
    f.m = f.r * (sums[1] * inv_c);
    f.q = a.after ? inv_sqrt(fmaf(sums[2], inv_c, a.eps)) : 1.f;
    const float dot = fmaf(f.r, fmaf(-f.m, f.r * sums[5], sums[4]), sums[3]);       // sum D gate after y
    f.e = f.q * dot;
    f.mean = a.after ? scale * f.e * inv_c : 0.f;
    return f;
}

// Sums of eight values over the warp at once: afterwards lane l holds that of value l / 4.
__device__ __forceinline__ float sum8_over_warp(const float (&v)[8], int lane)
{
    float a[4], b[2];
    const bool h16 = lane & 16, h8 = lane & 8, h4 = lane & 4;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float keep = h16 ? v[4 + j] : v[j], give = h16 ? v[j] : v[4 + j];
        a[j] = keep + __shfl_xor_sync(0xffffffffu, give, 16);
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const float keep = h8 ? a[2 + j] : a[j], give = h8 ? a[j] : a[2 + j];
        b[j] = keep + __shfl_xor_sync(0xffffffffu, give, 8);
    }
    float c = (h4 ? b[1] : b[0]) + __shfl_xor_sync(0xffffffffu, h4 ? b[0] : b[1], 4);
    c += __shfl_xor_sync(0xffffffffu, c, 2);
    c += __shfl_xor_sync(0xffffffffu, c, 1);
    return c;
}

// Sums of eight values over kLanes neighbouring lanes: a lane has those of values first .. first + 8 / kLanes (one at least; lanes of the same
// value have the same).
template <int kLanes>
__device__ __forceinline__ int sum8_over_lanes(float (&v)[8], int lane)
{
    int n = 8, first = 0;
#pragma unroll
    for (int d = kLanes / 2; d; d /= 2) {
        if (n > 1) {
            n /= 2;
            const bool high = lane & d;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (j < n) {
                    const float keep = high ? v[n + j] : v[j], give = high ? v[j] : v[n + j];
                    v[j] = keep + __shfl_xor_sync(0xffffffffu, give, d);
                }
            first += high ? n : 0;
        } else
            v[0] += __shfl_xor_sync(0xffffffffu, v[0], d);
    }
    return first;
}

// The row's six sums in every thread.
template <int kThreadsRow>
__device__ __forceinline__ void row_sums(float (&v)[8], float (*s_part)[8])
{
    constexpr int kWarps = kThreadsRow / 32;
    const int lane = threadIdx.x & 31;
    if constexpr (kThreadsRow < 32) {
        sum8_over_lanes<kThreadsRow>(v, lane);                // lane l of a row: value l / (kThreadsRow / 8)
        const float mine = v[0];
#pragma unroll
        for (int i = 0; i < kSums; ++i) v[i] = __shfl_sync(0xffffffffu, mine, i * (kThreadsRow / 8), kThreadsRow);
        return;
    }
    float mine = sum8_over_warp(v, lane);
    if constexpr (kWarps > 1) {
        if ((lane & 3) == 0) s_part[threadIdx.x >> 5][lane >> 2] = mine;
        __syncthreads();
        mine = 0.f;                                           // lane l: value l / 4, every fourth warp from l % 4 on
#pragma unroll
        for (int w = 0; w < (kWarps + 3) / 4; ++w)
            if (kWarps % 4 == 0 || 4 * w + (lane & 3) < kWarps) mine += s_part[4 * w + (lane & 3)][lane >> 2];
        mine += __shfl_xor_sync(0xffffffffu, mine, 1);
        mine += __shfl_xor_sync(0xffffffffu, mine, 2);
    }
#pragma unroll
    for (int i = 0; i < kSums; ++i) v[i] = __shfl_sync(0xffffffffu, mine, 4 * i);
}

template <typename T, int kThreadsRow, int kV, bool kVec>
__global__ void __launch_bounds__(kThreadsRow <= 32 ? 256 : kThreadsRow, kThreadsRow <= 32 ? 2 : (kThreadsRow >= 512 ? 1 : 512 / kThreadsRow))
norm_rows_grad_kernel(NormGradArgs a)
{
    constexpr int kRows = kThreadsRow <= 32 ? 256 / kThreadsRow : 1, kWarpRows = kThreadsRow < 32 ? 32 / kThreadsRow : 1;
    extern __shared__ float s_dyn[];                          // rows of a warp or less: [kRows][2][8 kThreadsRow kV] their threads' sums
    __shared__ float s_part[2][kThreadsRow <= 32 ? 1 : kThreadsRow / 32][8];
    __shared__ float s_scale[32];
    chain_next();
    chain_wait();
    const int t = threadIdx.x % kThreadsRow, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const float scale = a.y && a.scale ? *a.scale : 1.f;
    float sum_y[kV][8], sum_x[kV][8];                         // D n (times a map's gate);  dx s r
#pragma unroll
    for (int i = 0; i < kV; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) sum_y[i][j] = sum_x[i][j] = 0.f;
    CarriedSum total;
    int turn = 0;
    for (long long first = (long long)blockIdx.x * kRows + (kRows > 1 ? warp * kWarpRows : 0); first < a.pixels; first += (long long)gridDim.x * kRows, turn ^= 1) {
        const long long row = first + (kWarpRows > 1 ? lane / kThreadsRow : 0), base = row * a.c;
        const int c = kThreadsRow < 32 && row >= a.pixels ? 0 : a.c;               // (the rows of a warp keep in step)
        Raw8<T> rs[kV], ry[kV], rx[kV], rd[kV], rg[kV];
#pragma unroll
        for (int i = 0; i < kV; ++i) {
            zero8(rs[i]); zero8(ry[i]); zero8(rx[i]); zero8(rd[i]);
            if (a.before) {
                load_values<T, kThreadsRow, kVec>(rs[i], (const T *)a.s + base, t, i, c);
                load_values<T, kThreadsRow, kVec>(rx[i], (const T *)a.dx + base, t, i, c);
            }
            if (a.y) load_values<T, kThreadsRow, kVec>(ry[i], (const T *)a.y + base, t, i, c);
            if (a.ds) load_values<T, kThreadsRow, kVec>(rd[i], (const T *)a.ds + base, t, i, c);
            if (a.gate_map) load_values<T, kThreadsRow, kVec>(rg[i], (const T *)a.gate_map + base, t, i, c);
        }
        // gate times after of a chunk
        auto factors = [&](int i, float (&g)[8], float (&w)[8]) {
#pragma unroll
            for (int j = 0; j < 8; ++j) g[j] = w[j] = 1.f;
            if (a.gate_map) values8(rg[i], g);
            else if (a.gate) load_weights<kThreadsRow, kVec>(g, a.gate, t, i, c);
            if (a.after) load_weights<kThreadsRow, kVec>(w, a.after, t, i, c);
        };
        float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < kV; ++i) {
            float s[8], y[8], dx[8], ds[8], g[8], w[8], b[8];
            values8(rs[i], s); values8(ry[i], y); values8(rx[i], dx); values8(rd[i], ds);
            factors(i, g, w);
#pragma unroll
            for (int j = 0; j < 8; ++j) b[j] = 0.f;
            if (a.before) load_weights<kThreadsRow, kVec>(b, a.before, t, i, c);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float tt = dx[j] * b[j], gy = g[j] * w[j] * y[j];
                v[0] = fmaf(s[j], s[j], v[0]);
                v[1] = fmaf(tt, s[j], v[1]);
                v[2] = fmaf(y[j], y[j], v[2]);
                v[3] = fmaf(ds[j], gy, v[3]);
                v[4] = fmaf(tt, gy, v[4]);
                v[5] = fmaf(s[j], gy, v[5]);
            }
        }
        row_sums<kThreadsRow>(v, s_part[turn]);
        const float sums[kSums] = {v[0], v[1], v[2], v[3], v[4], v[5]};
        const PixelFactors f = pixel_factors(sums, a, scale);
        if (kWarpRows > 1 && c == 0) continue;
        total.add(f.e);
#pragma unroll
        for (int i = 0; i < kV; ++i) {
            float s[8], y[8], dx[8], d[8], g[8], w[8], b[8];
            values8(rs[i], s); values8(ry[i], y); values8(rx[i], dx); values8(rd[i], d);
            factors(i, g, w);
#pragma unroll
            for (int j = 0; j < 8; ++j) b[j] = 0.f;
            if (a.before) load_weights<kThreadsRow, kVec>(b, a.before, t, i, c);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float sr = s[j] * f.r;
                d[j] = fmaf(f.r, fmaf(-sr, f.m, dx[j] * b[j]), d[j]);
                sum_x[i][j] = fmaf(dx[j], sr, sum_x[i][j]);
            }
            store_values<T, kThreadsRow, kVec>((T *)a.dh + base, d, t, i, c);
            if (a.y) {
                float dy[8], dg[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float n = y[j] * f.q, dn = d[j] * n;
                    sum_y[i][j] += a.gate ? dn : dn * g[j];
                    dg[j] = scale * (dn * w[j]);
                    dy[j] = f.q * fmaf(-n, f.mean, scale * (d[j] * (g[j] * w[j])));
                }
                store_values<T, kThreadsRow, kVec>((T *)a.dy + base, dy, t, i, c);
                if (a.gate_map) store_values<T, kThreadsRow, kVec>((T *)a.dgate_map + base, dg, t, i, c);
            }
        }
    }
    // the block's sums
    float *const part = a.partial + (long long)blockIdx.x * 2 * a.c;
    if constexpr (kRows > 1) {
        constexpr int kRow = 8 * kThreadsRow * kV;
        float *const mine = s_dyn + threadIdx.x / kThreadsRow * 2 * kRow;
#pragma unroll
        for (int i = 0; i < kV; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                mine[value_at<kThreadsRow, kVec>(t, i, j)] = sum_y[i][j];
                mine[kRow + value_at<kThreadsRow, kVec>(t, i, j)] = sum_x[i][j];
            }
        __syncthreads();
        for (int i = threadIdx.x; i < 2 * kRow; i += 256) {
            const int k = i % kRow;
            float v = 0.f;
#pragma unroll
            for (int w = 0; w < kRows; ++w) v += s_dyn[w * 2 * kRow + i];
            if (k < a.c) part[(i / kRow) * (long long)a.c + k] = v;
        }
    } else {
#pragma unroll
        for (int i = 0; i < kV; ++i) {
            store_values<float, kThreadsRow, kVec>(part, sum_y[i], t, i, a.c);
            store_values<float, kThreadsRow, kVec>(part + a.c, sum_x[i], t, i, a.c);
        }
    }
    float sum_scale = t == 0 ? total.value() : 0.f;
#pragma unroll
    for (int d = 16; d; d >>= 1) sum_scale += __shfl_xor_sync(0xffffffffu, sum_scale, d);
    if (lane == 0) s_scale[warp] = sum_scale;
    __syncthreads();
    if (threadIdx.x == 0) {
        float v = 0.f;
        for (int w = 0; w < (int)(blockDim.x >> 5); ++w) v += s_scale[w];
        a.partial_scale[blockIdx.x] = v;
    }
}

// The same with the rows in a ring, the vectors and the sums over the rows in registers.
template <typename T, int kWarps, int kV, bool kVec>
__global__ void __launch_bounds__(kWarps * 32, 16 / kWarps) norm_rows_grad_ring_kernel(const __grid_constant__ NormGradArgs a, const __grid_constant__ RowRing r)
{
    constexpr int kThreadsRow = kWarps * 32;
    extern __shared__ __align__(16) unsigned char s_ring[];
    __shared__ __align__(8) unsigned long long s_full[kRingStages];
    __shared__ int s_brought;
    __shared__ float s_part[2][kWarps][8];
    chain_next();
    chain_wait();
    const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
    RowReader<kVec> reader;
    reader.ring = sm100::smem_u32(s_ring);
    reader.full = s_full;
    reader.brought = &s_brought;
    reader.start(r, a.pixels);
    // parts of a stage: s and dx (with before), y, ds, gate, those that there are
    const uint32_t part = r.part_bytes, at_y = a.before ? 2 * part : 0, at_d = at_y + (a.y ? part : 0), at_g = at_d + (a.ds ? part : 0);
    const float scale = a.y && a.scale ? *a.scale : 1.f;
    float wy[kV][8], wx[kV][8], sum_y[kV][8], sum_x[kV][8];
#pragma unroll
    for (int i = 0; i < kV; ++i) {
        float g[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) { wy[i][j] = g[j] = 1.f; wx[i][j] = sum_y[i][j] = sum_x[i][j] = 0.f; }
        if (a.after) load_weights<kThreadsRow, kVec>(wy[i], a.after, t, i, a.c);
        if (a.gate) load_weights<kThreadsRow, kVec>(g, a.gate, t, i, a.c);
        if (a.before) load_weights<kThreadsRow, kVec>(wx[i], a.before, t, i, a.c);
#pragma unroll
        for (int j = 0; j < 8; ++j) wy[i][j] *= g[j];
    }
    CarriedSum total;
    int turn = 0, slot = 0, last = 0;
    for (long long row = blockIdx.x; row < a.pixels; row += gridDim.x, ++turn) {
        const long long base = row * a.c;
        const uint32_t at = reader.row(r, row, turn, slot, a.status);
        auto get = [&](bool there, uint32_t where, int i, float (&f)[8]) {
            Raw8<T> raw;
            if (there) load_shared<T, kThreadsRow, kVec>(raw, at + where, t, i, a.c);
            else zero8(raw);
            values8(raw, f);
        };
        float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < kV; ++i) {
            float s[8], y[8], dx[8], d[8];
            get(a.before, 0, i, s);
            get(a.before, part, i, dx);
            get(a.y, at_y, i, y);
            get(a.ds, at_d, i, d);
            if (a.gate_map) {
                float g[8];
                get(true, at_g, i, g);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    v[2] = fmaf(y[j], y[j], v[2]);
                    y[j] *= g[j];
                }
            } else
#pragma unroll
                for (int j = 0; j < 8; ++j) v[2] = fmaf(y[j], y[j], v[2]);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float tt = dx[j] * wx[i][j], gy = wy[i][j] * y[j];
                v[0] = fmaf(s[j], s[j], v[0]);
                v[1] = fmaf(tt, s[j], v[1]);
                v[3] = fmaf(d[j], gy, v[3]);
                v[4] = fmaf(tt, gy, v[4]);
                v[5] = fmaf(s[j], gy, v[5]);
            }
        }
        row_sums<kThreadsRow>(v, s_part[turn & 1]);
        // (the block is in step: the last row's slot is free)
        if (t == 0 && reader.alive && turn > 0 && row + (long long)(r.stages - 1) * gridDim.x < a.pixels) reader.bring(r, row + (long long)(r.stages - 1) * gridDim.x, last);
        const float sums[kSums] = {v[0], v[1], v[2], v[3], v[4], v[5]};
        const PixelFactors f = pixel_factors(sums, a, scale);
        total.add(f.e);
        const float scale_q = scale * f.q, mean_q = f.mean * f.q;
#pragma unroll
        for (int i = 0; i < kV; ++i) {
            float s[8], y[8], d[8], g[8];
            get(a.ds, at_d, i, d);
            if (a.before) {
                float dx[8];
                get(true, 0, i, s);
                get(true, part, i, dx);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float sr = s[j] * f.r;
                    d[j] = fmaf(f.r, fmaf(-sr, f.m, dx[j] * wx[i][j]), d[j]);
                    sum_x[i][j] = fmaf(dx[j], sr, sum_x[i][j]);
                }
            }
            store_values<T, kThreadsRow, kVec>((T *)a.dh + base, d, t, i, a.c);
            if (a.y) {
                get(true, at_y, i, y);
#pragma unroll
                for (int j = 0; j < 8; ++j) g[j] = 1.f;
                if (a.gate_map) get(true, at_g, i, g);
                float dy[8], dg[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float n = y[j] * f.q, dw = d[j] * wy[i][j], dn = d[j] * n;
                    dg[j] = scale * (dw * n);
                    sum_y[i][j] = a.gate_map ? fmaf(dn, g[j], sum_y[i][j]) : sum_y[i][j] + dn;
                    dy[j] = fmaf(-n, mean_q, scale_q * (dw * g[j]));
                }
                store_values<T, kThreadsRow, kVec>((T *)a.dy + base, dy, t, i, a.c);
                if (a.gate_map) store_values<T, kThreadsRow, kVec>((T *)a.dgate_map + base, dg, t, i, a.c);
            }
        }
        last = slot;
        if (++slot == r.stages) slot = 0;
    }
    reader.finish(r);
    float *const to = a.partial + (long long)blockIdx.x * 2 * a.c;
#pragma unroll
    for (int i = 0; i < kV; ++i) {
        store_values<float, kThreadsRow, kVec>(to, sum_y[i], t, i, a.c);
        store_values<float, kThreadsRow, kVec>(to + a.c, sum_x[i], t, i, a.c);
    }
    if (t == 0) a.partial_scale[blockIdx.x] = total.value();
}

// Maps: 32 pixels at a time, a lane for each; warps take slices of eight channels in turn.  The sums over the pixels are
// kept in shared memory, each channel's by the one warp that has it.
template <typename T>
__global__ void __launch_bounds__(256) norm_maps_grad_kernel(NormGradArgs a)
{
    extern __shared__ float s_dyn[];                          // [2][c]
    __shared__ float s_part[8][kSums][32];
    chain_next();
    chain_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const float scale = a.y && a.scale ? *a.scale : 1.f;
    for (int i = threadIdx.x; i < 2 * a.c; i += 256) s_dyn[i] = 0.f;
    CarriedSum total;
    const long long groups = (a.pixels + 31) / 32;
    for (long long group = blockIdx.x; group < groups; group += gridDim.x) {
        const long long p = group * 32 + lane;
        const bool ok = p < a.pixels;
        const long long img = p / a.hw, base = img * a.c * (long long)a.hw + (p - img * a.hw);
        float sums[kSums] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        for (int c0 = warp * 8; c0 < a.c; c0 += 64) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int ch = c0 + j;
                if (!ok || ch >= a.c) continue;
                const long long at = base + (long long)ch * a.hw;
                const float s = a.before ? load1((const T *)a.s + at) : 0.f, t = a.before ? load1((const T *)a.dx + at) * a.before[ch] : 0.f;
                const float y = a.y ? load1((const T *)a.y + at) : 0.f, ds = a.ds ? load1((const T *)a.ds + at) : 0.f;
                float gy = y;
                if (a.after) gy *= a.after[ch];
                if (a.gate_map) gy *= load1((const T *)a.gate_map + at);
                else if (a.gate) gy *= a.gate[ch];
                sums[0] = fmaf(s, s, sums[0]);
                sums[1] = fmaf(t, s, sums[1]);
                sums[2] = fmaf(y, y, sums[2]);
                sums[3] = fmaf(ds, gy, sums[3]);
                sums[4] = fmaf(t, gy, sums[4]);
                sums[5] = fmaf(s, gy, sums[5]);
            }
        }
        __syncthreads();                                      // the last group's readers
#pragma unroll
        for (int i = 0; i < kSums; ++i) s_part[warp][i][lane] = sums[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kSums; ++i) {
            sums[i] = 0.f;
#pragma unroll
            for (int w = 0; w < 8; ++w) sums[i] += s_part[w][i][lane];
        }
        const PixelFactors f = pixel_factors(sums, a, scale);
        if (ok) total.add(f.e);
        for (int c0 = warp * 8; c0 < a.c; c0 += 64) {
            float sum_y[8], sum_x[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int ch = c0 + j;
                sum_y[j] = sum_x[j] = 0.f;
                if (!ok || ch >= a.c) continue;
                const long long at = base + (long long)ch * a.hw;
                float d = a.ds ? load1((const T *)a.ds + at) : 0.f;
                if (a.before) {
                    const float s = load1((const T *)a.s + at), dx = load1((const T *)a.dx + at);
                    const float sr = s * f.r;
                    d = fmaf(f.r, fmaf(-sr, f.m, dx * a.before[ch]), d);
                    sum_x[j] = dx * sr;
                }
                store1((T *)a.dh + at, d);
                if (a.y) {
                    const float n = load1((const T *)a.y + at) * f.q, w = a.after ? a.after[ch] : 1.f;
                    const float g = a.gate_map ? load1((const T *)a.gate_map + at) : a.gate ? a.gate[ch] : 1.f, dn = d * n;
                    sum_y[j] = a.gate ? dn : dn * g;
                    store1((T *)a.dy + at, f.q * fmaf(-n, f.mean, scale * (d * (g * w))));
                    if (a.gate_map) store1((T *)a.dgate_map + at, scale * (dn * w));
                }
            }
            const float vy = sum8_over_warp(sum_y, lane), vx = sum8_over_warp(sum_x, lane);
            if ((lane & 3) == 0 && c0 + (lane >> 2) < a.c) {
                s_dyn[c0 + (lane >> 2)] += vy;
                s_dyn[a.c + c0 + (lane >> 2)] += vx;
            }
        }
    }
    float sum_scale = total.value();                          // (every warp has the same pixels')
#pragma unroll
    for (int d = 16; d; d >>= 1) sum_scale += __shfl_xor_sync(0xffffffffu, sum_scale, d);
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * a.c; i += 256) a.partial[(long long)blockIdx.x * 2 * a.c + i] = s_dyn[i];
    if (threadIdx.x == 0) a.partial_scale[blockIdx.x] = sum_scale;
}

// The same with the inputs' tile in shared memory, as in the forward.
template <typename T, int kPx, int kWarps>
__global__ void __launch_bounds__(32 * kWarps, 16 / kWarps) norm_maps_grad_tile_kernel(const __grid_constant__ NormGradArgs a, int vec, int pairs)
{
    using M = MapTile<T, kPx, kWarps>;
    extern __shared__ __align__(16) unsigned char s_tile[];   // sums over the pixels [2][c8], after times the channels' gate, before; s, dx, y, ds, gate [c8][kPx]
    __shared__ float2 s_part[kSums][kWarps][M::kPairs];
    const int c8 = (a.c + 7) & ~7, plane = M::values(c8);
    uint64_t *const wy = reinterpret_cast<uint64_t *>(s_tile), *const wx = wy + c8;
    float *const sums_y = reinterpret_cast<float *>(wx + c8), *const sums_x = sums_y + c8;
    T *const ss = reinterpret_cast<T *>(sums_x + c8), *const sx = ss + (a.before ? plane : 0), *const sy = sx + (a.before ? plane : 0);
    T *const sd = sy + (a.y ? plane : 0), *const sg = sd + (a.ds ? plane : 0);
    chain_next();
    chain_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, pair = lane % M::kPairs, slice = warp * M::kSubs + lane / M::kPairs;
    fill_weights(wy, wx, a.after, a.gate, a.before, a.c, c8);
    for (int i = threadIdx.x; i < 2 * c8; i += M::kThreads) sums_y[i] = 0.f;
    zero_rows<M>(ss, (a.before ? 2 : 0) + (a.y != nullptr) + (a.ds != nullptr) + (a.gate_map != nullptr), plane, a.c, c8, kPx);
    const float scale = a.y && a.scale ? *a.scale : 1.f;
    CarriedSum total0, total1;
    const long long tiles = (a.pixels + kPx - 1) / kPx;
    for (long long tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const uint32_t p0 = (uint32_t)tile * kPx, pixels = (uint32_t)a.pixels;
        const MapPixels px(p0 + 2 * pair, pixels, a.c, a.hw, pairs);
        __syncthreads();                                      // the last tile's readers
        if (vec) {
            if (a.before) {
                M::fill_quads(ss, (const T *)a.s, p0, pixels, a.c, a.hw);
                M::fill_quads(sx, (const T *)a.dx, p0, pixels, a.c, a.hw);
            }
            if (a.y) M::fill_quads(sy, (const T *)a.y, p0, pixels, a.c, a.hw);
            if (a.ds) M::fill_quads(sd, (const T *)a.ds, p0, pixels, a.c, a.hw);
            if (a.gate_map) M::fill_quads(sg, (const T *)a.gate_map, p0, pixels, a.c, a.hw);
        } else {
            const void *const inputs[] = {a.before ? a.s : nullptr, a.before ? a.dx : nullptr, a.y, a.ds, a.gate_map};
            M::fill(ss, plane, inputs, p0, pixels, a.c, a.hw);
        }
        sm100::cp_async_wait_all();
        __syncthreads();
        uint64_t sums[kSums] = {0ull, 0ull, 0ull, 0ull, 0ull, 0ull};
        for (int c0 = slice * 8; c0 < a.c; c0 += M::kStep) {
            const T *const s = M::eight(ss, c0, pair), *const x = M::eight(sx, c0, pair), *const y = M::eight(sy, c0, pair), *const d = M::eight(sd, c0, pair),
                    *const g = M::eight(sg, c0, pair);
            uint64_t w[8], b[8];
            weights8(w, wy + c0);
            weights8(b, wx + c0);
#pragma unroll
            for (int h = 0; h < 8; h += 4) {
                uint64_t sv[4] = {0ull, 0ull, 0ull, 0ull}, tv[4] = {0ull, 0ull, 0ull, 0ull};
                if (a.before)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        sv[j] = M::load(s, h + j);
                        tv[j] = mul2(M::load(x, h + j), b[h + j]);
                        sums[0] = fma2(sv[j], sv[j], sums[0]);
                        sums[1] = fma2(tv[j], sv[j], sums[1]);
                    }
                if (a.y) {
                    uint64_t gy[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const uint64_t yv = M::load(y, h + j);
                        gy[j] = mul2(yv, w[h + j]);
                        sums[2] = fma2(yv, yv, sums[2]);
                    }
                    if (a.gate_map)
#pragma unroll
                        for (int j = 0; j < 4; ++j) gy[j] = mul2(gy[j], M::load(g, h + j));
                    if (a.ds)
#pragma unroll
                        for (int j = 0; j < 4; ++j) sums[3] = fma2(M::load(d, h + j), gy[j], sums[3]);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        sums[4] = fma2(tv[j], gy[j], sums[4]);
                        sums[5] = fma2(sv[j], gy[j], sums[5]);
                    }
                }
            }
        }
        float sum0[kSums], sum1[kSums];
#pragma unroll
        for (int i = 0; i < kSums; ++i) {
            halves(sums[i], sum0[i], sum1[i]);
#pragma unroll
            for (int d = M::kPairs; d < 32; d *= 2) {
                sum0[i] += __shfl_xor_sync(0xffffffffu, sum0[i], d);
                sum1[i] += __shfl_xor_sync(0xffffffffu, sum1[i], d);
            }
            if (lane < M::kPairs) s_part[i][warp][lane] = make_float2(sum0[i], sum1[i]);
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kSums; ++i) {
            sum0[i] = sum1[i] = 0.f;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
                const float2 q = s_part[i][w][pair];
                sum0[i] += q.x;
                sum1[i] += q.y;
            }
        }
        // (the zeros of a pixel behind the last one would have infinite factors without eps, and the vectors' sums be NaN)
        if (!px.ok0) sum0[0] = sum0[2] = 1.f;
        if (!px.ok1) sum1[0] = sum1[2] = 1.f;
        const PixelFactors f0 = pixel_factors(sum0, a, scale), f1 = pixel_factors(sum1, a, scale);
        if (px.ok0) total0.add(f0.e);
        if (px.ok1) total1.add(f1.e);
        const uint64_t r = pair_of(f0.r, f1.r), m = pair_of(-f0.m, -f1.m), q = pair_of(f0.q, f1.q), scale_q = pair_of(scale * f0.q, scale * f1.q);
        const uint64_t mean_q = pair_of(-f0.mean * f0.q, -f1.mean * f1.q), scales = pair_of(scale, scale);
        for (int c0 = slice * 8; c0 - slice * 8 < a.c; c0 += M::kStep) {           // (the same for all lanes: their sums go together)
            float sum_y[8], sum_x[8];
            const bool some = c0 < a.c;
#pragma unroll
            for (int j = 0; j < 8; ++j) sum_y[j] = sum_x[j] = 0.f;
            if (some) {
                const T *const s = M::eight(ss, c0, pair), *const x = M::eight(sx, c0, pair), *const y = M::eight(sy, c0, pair), *const dd = M::eight(sd, c0, pair),
                        *const g = M::eight(sg, c0, pair);
                const MapRows<T> to_h((T *)a.dh, px, c0, a.c, a.hw), to_y((T *)a.dy, px, c0, a.c, a.hw), to_g((T *)a.dgate_map, px, c0, a.c, a.hw);
                uint64_t w[8], b[8];
                weights8(w, wy + c0);
                weights8(b, wx + c0);
#pragma unroll
                for (int h = 0; h < 8; h += 4) {
                    uint64_t d[4] = {0ull, 0ull, 0ull, 0ull};
                    float u, v;
                    if (a.ds)
#pragma unroll
                        for (int j = 0; j < 4; ++j) d[j] = M::load(dd, h + j);
                    if (a.before)
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const uint64_t sr = mul2(r, M::load(s, h + j)), xv = M::load(x, h + j);
                            d[j] = fma2(r, fma2(sr, m, mul2(xv, b[h + j])), d[j]);
                            halves(mul2(xv, sr), u, v);
                            sum_x[h + j] = u + v;
                        }
                    to_h.store4(h, d);
                    if (a.y) {
                        uint64_t n[4], dw[4], dn[4], dwg[4];
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            n[j] = mul2(M::load(y, h + j), q);
                            dw[j] = dwg[j] = mul2(d[j], w[h + j]);
                            dn[j] = mul2(d[j], n[j]);
                        }
                        if (a.gate_map) {
                            uint64_t dg[4];
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                const uint64_t gv = M::load(g, h + j);
                                dn[j] = mul2(dn[j], gv);
                                dwg[j] = mul2(dw[j], gv);
                                dg[j] = mul2(scales, mul2(dw[j], n[j]));
                            }
                            to_g.store4(h, dg);
                        }
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            halves(dn[j], u, v);
                            sum_y[h + j] = u + v;
                            dwg[j] = fma2(n[j], mean_q, mul2(scale_q, dwg[j]));
                        }
                        to_y.store4(h, dwg);
                    }
                }
            }
            const int first = sum8_over_lanes<M::kPairs>(sum_y, lane);
            sum8_over_lanes<M::kPairs>(sum_x, lane);
            constexpr int kEach = 8 / M::kPairs > 1 ? 8 / M::kPairs : 1, kSame = M::kPairs > 8 ? M::kPairs / 8 : 1;
            if (some && lane % kSame == 0) {
#pragma unroll
                for (int j = 0; j < kEach; ++j) {
                    sums_y[c0 + first + j] += sum_y[j];
                    sums_x[c0 + first + j] += sum_x[j];
                }
            }
        }
    }
    float sum_scale = lane < M::kPairs ? total0.value() + total1.value() : 0.f;      // (every warp has the same pixels')
#pragma unroll
    for (int d = 16; d; d >>= 1) sum_scale += __shfl_xor_sync(0xffffffffu, sum_scale, d);
    __syncthreads();
    float *const to = a.partial + (long long)blockIdx.x * 2 * a.c;
    for (int i = threadIdx.x; i < a.c; i += M::kThreads) {
        to[i] = sums_y[i];
        to[a.c + i] = sums_x[i];
    }
    if (threadIdx.x == 0) a.partial_scale[blockIdx.x] = sum_scale;
}

// The blocks' sums, in their order: 32 channels a block, every kVectorWarps-th of the blocks' sums a warp (of up to eight an SM, 1184 on
// 148: what it waits for is memory, one sum after the other).
constexpr int kVectorWarps = 32;
__global__ void __launch_bounds__(kVectorWarps * 32) norm_vectors_kernel(NormGradArgs a, int blocks)
{
    __shared__ float s_sum[2][kVectorWarps][32];
    chain_next();
    chain_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, ch = blockIdx.x * 32 + lane;
    float vy = 0.f, vx = 0.f;
    if (ch < a.c)
        #pragma unroll 4
        for (int b = warp; b < blocks; b += kVectorWarps) {
            vy += a.partial[(long long)b * 2 * a.c + ch];
            vx += a.partial[(long long)b * 2 * a.c + a.c + ch];
        }
    s_sum[0][warp][lane] = vy;
    s_sum[1][warp][lane] = vx;
    __syncthreads();
    if (warp == 0 && ch < a.c) {
        vy = vx = 0.f;
        for (int w = 0; w < kVectorWarps; ++w) { vy += s_sum[0][w][lane]; vx += s_sum[1][w][lane]; }
        const float scale = a.y && a.scale ? *a.scale : 1.f;
        if (a.dafter) a.dafter[ch] = scale * vy * (a.gate ? a.gate[ch] : 1.f);
        if (a.dgate) a.dgate[ch] = scale * vy * (a.after ? a.after[ch] : 1.f);
        if (a.dbefore) a.dbefore[ch] = vx;
    }
    if (warp == 1 && blockIdx.x == 0 && a.dscale) {
        double v = 0.0;                                       // (one warp, and the blocks' sums cancel like their pixels')
        for (int b = lane; b < blocks; b += 32) v += a.partial_scale[b];
#pragma unroll
        for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
        if (lane == 0) *a.dscale = (float)v;
    }
}

template <typename T, int kThreadsRow, int kV>
tc_status launch_norm_rows(const NormArgs &a, cudaStream_t s)
{
    constexpr int kRows = kThreadsRow <= 32 ? 256 / kThreadsRow : 1;
    auto kernel = norm_rows_kernel<T, kThreadsRow, kV, true>;
    if constexpr (kThreadsRow >= 32)
        if (!a.vec) kernel = norm_rows_kernel<T, kThreadsRow, kV, false>;
    return launch_first(true, kernel, dim3((unsigned int)((a.pixels + kRows - 1) / kRows)), dim3(kThreadsRow <= 32 ? 256 : kThreadsRow), 0, s, a) == cudaSuccess ? TC_OK : TC_ERR_CUDA;
}

// A ring of rows of the given inputs, for `blocks` blocks an SM; none (no stages) where two rows do not fit, and where a block has no more than two rows, which
// registers hold as soon.
RowRing make_ring(std::initializer_list<const void *> inputs, int c, size_t size, long long rows, long long grid, int blocks, bool vec)
{
    RowRing r{};
    for (const void *p : inputs)
        if (p) {
            if ((uintptr_t)p & 15u) return RowRing{};
            r.in[r.inputs++] = (const char *)p;
        }
    r.rows = rows;
    r.row_bytes = (uint32_t)(c * size);
    r.part_bytes = vec ? r.row_bytes : (r.row_bytes + 30u) & ~15u;
    const size_t stage = (size_t)r.inputs * r.part_bytes, fit = kRingSm / blocks / stage;
    r.stages = fit < 2 || rows <= 2 * grid ? 0 : (int)(fit < kRingStages ? fit : kRingStages);
    return r;
}

template <auto kKernel, typename A>
cudaError_t launch_ring(int device, const A &a, const RowRing &r, long long grid, int threads, cudaStream_t s)
{
    if (!allow_shared<kKernel>(device, kRingSm)) return cudaErrorInvalidValue;
    return launch_first(true, kKernel, dim3((unsigned int)grid), dim3(threads), (size_t)r.stages * r.inputs * r.part_bytes, s, a, r);
}

// Forward with the ring, kBlocks blocks an SM; false where there is none.
template <typename T, int kWarps, int kV>
bool launch_norm_ring(const NormArgs &a, cudaStream_t s, tc_status &st)
{
    constexpr int kBlocks = 16 / kWarps;
    if (!a.vec || !a.y) return false;
    const long long grid = (long long)a.sms * kBlocks;
    const RowRing r = make_ring({a.h, a.y, a.gate_map}, a.c, sizeof(T), a.pixels, grid, kBlocks, true);
    if (r.stages == 0) return false;
    st = launch_ring<norm_rows_ring_kernel<T, kWarps, kV>>(a.device, a, r, grid, kWarps * 32, s) == cudaSuccess ? TC_OK : TC_ERR_CUDA;
    return true;
}

// Whether maps are moved four pixels at a time.
template <typename T, typename... P>
bool four_pixels(int hw, P... p)
{
    return hw % 4 == 0 && ((((uintptr_t)p) | ...) & (4 * sizeof(T) - 1)) == 0;
}
// Whether two neighbouring pixels are written at once.
template <typename T, typename... P>
bool pixel_pairs(int hw, P... p)
{
    return hw % 2 == 0 && ((((uintptr_t)p) | ...) & (2 * sizeof(T) - 1)) == 0;
}

// Tile of a maps' kernel: as many pixels as fit, but no more than 16 while the tiles are fewer than two an SM, and 64 only of up to 64 channels,
// which leave half of the warps idle with 32.  0 where not even eight fit, of about 1250 channels on for the gradient in fp32 (1030 with a gate for
// each value), 2200 (1850) in bf16, 2390 (1700) and 4060 (3010) for the forward: those maps take the kernels that read them again for each pass, 1.5 to five
// times as long (gradient of 1248x7x7 x 128 in fp32 163 us, of 1256 310; forward of 4056x1x8192 in bf16 225, of 4064 1166).
// `two`: rather tiles of which two fit an SM, the forward's (944x7x7 x 431 in bf16 185 us and 127, 512x28x28 x 60 in fp32 105 and 78; the
// gradient of the first takes 204 with one and 223 with two, though even sides in fp32 would gain: 256x14x14 x 1024 345 and 302).  Up to 32 channels
// keep four warps busy: more blocks of those (25x20x20 x 437 in bf16, forward 26 us and 17, gradient 57 and 37).  Where one tile of the
// gradient's fits an SM and its pixels come one at a time, sixteen warps work on it (944x7x7 x 431 in bf16 260 us and 204; by
// fours it costs time in fp32, 512x28x28 x 60 172 and 195, and gains a little in bf16, 944x8x8 x 200 83 and 79).
struct MapPlan {
    int px = 0, warps = 8;
    size_t smem = 0;
    long long blocks = 0;
};
MapPlan plan_maps(int inputs, int vectors, int c, int hw, size_t size, long long pixels, int sms, int warps_sm, bool two)
{
    MapPlan m;
    const size_t c8 = (size_t)((c + 7) & ~7);
    for (int px = c <= 64 ? 64 : 32; px >= 8; px /= 2) {
        const size_t rows = px * size < 128 ? 9 : 8, smem = c8 * vectors * sizeof(float) + inputs * (c8 / 8) * rows * px * size;
        if (smem + kTileStatic > kTileSm || (px > 16 && pixels <= 2ll * sms * px) || (two && px > 8 && 2 * (smem + kTileStatic) > kTileSm)) continue;
        m.warps = px == 64 && c <= 32 ? 4 : !two && hw % 4 && c > 256 && 2 * (smem + kTileStatic) > kTileSm ? 16 : 8;
        const long long fit = (long long)(kTileSm / (smem + kTileStatic / (m.warps < 8 ? 2 : 1))), held = warps_sm / m.warps, tiles = (pixels + px - 1) / px, most = (fit < held ? fit : held) * sms;
        m.px = px;
        m.smem = smem;
        m.blocks = tiles < most ? tiles : most;
        break;
    }
    return m;
}
MapPlan plan_grad_maps(const NormGradArgs &a, size_t size, int sms)
{
    return plan_maps((a.before ? 2 : 0) + (a.y != nullptr) + (a.ds != nullptr) + (a.gate_map != nullptr), 6, a.c, a.hw, size, a.pixels, sms, 16, false);
}

template <auto kKernel, typename A>
cudaError_t launch_maps(const A &a, const MapPlan &m, long long blocks, bool vec, bool pairs, cudaStream_t s)
{
    if (!allow_shared<kKernel>(a.device, kTileSm - kTileStatic)) return cudaErrorInvalidValue;
    return launch_first(true, kKernel, dim3((unsigned int)blocks), dim3(32 * m.warps), m.smem, s, a, (int)vec, (int)pairs);
}

template <typename T>
tc_status norms(const NormArgs &a, cudaStream_t s)
{
    if (a.hw > 1) {
        const MapPlan m = plan_maps(1 + (a.y != nullptr) + (a.gate_map != nullptr), 4, a.c, a.hw, sizeof(T), a.pixels, a.sms, 24, true);
        const bool vec = four_pixels<T>(a.hw, a.h, a.y, a.gate_map), pairs = pixel_pairs<T>(a.hw, a.sum, a.x);
        if (m.px == 64 && m.warps == 4) return launch_maps<norm_maps_tile_kernel<T, 64, 4>>(a, m, m.blocks, vec, pairs, s) == cudaSuccess ? TC_OK : TC_ERR_CUDA;
        if (m.px == 64) return launch_maps<norm_maps_tile_kernel<T, 64, 8>>(a, m, m.blocks, vec, pairs, s) == cudaSuccess ? TC_OK : TC_ERR_CUDA;
        if (m.px == 32) return launch_maps<norm_maps_tile_kernel<T, 32, 8>>(a, m, m.blocks, vec, pairs, s) == cudaSuccess ? TC_OK : TC_ERR_CUDA;
        if (m.px == 16) return launch_maps<norm_maps_tile_kernel<T, 16, 8>>(a, m, m.blocks, vec, pairs, s) == cudaSuccess ? TC_OK : TC_ERR_CUDA;
        if (m.px == 8) return launch_maps<norm_maps_tile_kernel<T, 8, 8>>(a, m, m.blocks, vec, pairs, s) == cudaSuccess ? TC_OK : TC_ERR_CUDA;
        return launch_first(true, norm_maps_kernel<T>, dim3((unsigned int)((a.pixels + 31) / 32)), dim3(256), 0, s, a) == cudaSuccess ? TC_OK : TC_ERR_CUDA;
    }
    if (a.c <= 64 && a.vec) return launch_norm_rows<T, 8, 1>(a, s);
    if (a.c <= 128 && a.vec) return launch_norm_rows<T, 16, 1>(a, s);
    if (a.c <= 256) return launch_norm_rows<T, 32, 1>(a, s);
    if (a.c <= 512) return launch_norm_rows<T, 32, 2>(a, s);
    tc_status st;
    if (a.c <= 1024) return launch_norm_ring<T, 2, 2>(a, s, st) ? st : launch_norm_rows<T, 128, 1>(a, s);
    if (a.c <= 2048) return launch_norm_ring<T, 4, 2>(a, s, st) ? st : launch_norm_rows<T, 256, 1>(a, s);
    if (a.c <= 4096) return launch_norm_ring<T, 8, 2>(a, s, st) ? st : launch_norm_rows<T, 256, 2>(a, s);
    if (a.c <= 8192) return launch_norm_ring<T, 16, 2>(a, s, st) ? st : launch_norm_rows<T, 512, 2>(a, s);
    return launch_norm_rows<T, 512, 4>(a, s);
}

template <typename T, int kThreadsRow, int kV>
cudaError_t launch_grad_rows(const NormGradArgs &a, int blocks, cudaStream_t s)
{
    const size_t smem = kThreadsRow <= 32 ? 2 * 8 * 256 * kV * sizeof(float) : 0;
    auto kernel = norm_rows_grad_kernel<T, kThreadsRow, kV, true>;
    if constexpr (kThreadsRow >= 32)
        if (!a.vec) kernel = norm_rows_grad_kernel<T, kThreadsRow, kV, false>;
    return launch_first(true, kernel, dim3((unsigned int)blocks), dim3(kThreadsRow <= 32 ? 256 : kThreadsRow), smem, s, a);
}
// Threads of a row of up to 256 channels.
int short_row_threads(const NormGradArgs &a) { return !a.vec || a.c > 128 ? 32 : a.c > 64 ? 16 : 8; }

// With the ring of rows where there is one: two chunks a thread of bf16, whose unpacking and sums bound it (16384x4096 205 us with one
// and 158); one of fp32, of whose rows two would not fit two blocks' rings.  Blocks of 512 threads an SM in all.
constexpr int ring_chunks(int warps, int size) { return warps <= 2 ? 1 : warps > 16 ? warps / 16 : size == 2 ? 2 : 1; }
// Rows of up to 256 kWarps channels.
template <typename T, int kWarps>
cudaError_t launch_grad(const NormGradArgs &a, int blocks, cudaStream_t s)
{
    constexpr int kRingV = ring_chunks(kWarps, sizeof(T)), kRingWarps = kWarps / kRingV;
    const RowRing r = make_ring({a.before ? a.s : nullptr, a.before ? a.dx : nullptr, a.y, a.ds, a.gate_map}, a.c, sizeof(T), a.pixels, blocks, 16 / kRingWarps, a.vec);
    if (r.stages && a.vec) return launch_ring<norm_rows_grad_ring_kernel<T, kRingWarps, kRingV, true>>(a.device, a, r, blocks, kRingWarps * 32, s);
    if constexpr (kWarps > 2)                                 // (unaligned rows of up to 512 channels: 20000x301 in fp32 51 us without and 55 with, in bf16 61 and 56)
        if (r.stages) return launch_ring<norm_rows_grad_ring_kernel<T, kRingWarps, kRingV, false>>(a.device, a, r, blocks, kRingWarps * 32, s);
    return launch_grad_rows<T, 32 * kWarps, 1>(a, blocks, s);
}

template <typename T>
tc_status gradient(const NormGradArgs &a, int blocks, int sms, cudaStream_t s)
{
    cudaError_t err = cudaSuccess;
    if (blocks == 0) {                                        // no pixels: the vectors' gradients are zero
    } else if (const MapPlan m = plan_grad_maps(a, sizeof(T), sms); a.hw > 1 && m.px) {
        const bool vec = four_pixels<T>(a.hw, a.s, a.dx, a.y, a.ds, a.gate_map), pairs = pixel_pairs<T>(a.hw, a.dh, a.dy, a.dgate_map);
        auto run = [&](auto px, auto warps) { return launch_maps<norm_maps_grad_tile_kernel<T, px.value, warps.value>>(a, m, blocks, vec, pairs, s); };
        using std::integral_constant;
        constexpr integral_constant<int, 4> w4; constexpr integral_constant<int, 8> w8; constexpr integral_constant<int, 16> w16;
        err = m.px == 64   ? m.warps == 4 ? run(integral_constant<int, 64>(), w4) : run(integral_constant<int, 64>(), w8)
              : m.px == 32 ? m.warps == 16 ? run(integral_constant<int, 32>(), w16) : run(integral_constant<int, 32>(), w8)
              : m.px == 16 ? m.warps == 16 ? run(integral_constant<int, 16>(), w16) : run(integral_constant<int, 16>(), w8)
                           : m.warps == 16 ? run(integral_constant<int, 8>(), w16) : run(integral_constant<int, 8>(), w8);
    } else if (a.hw > 1) {
        const size_t smem = (size_t)2 * a.c * sizeof(float);
        err = allow_shared<norm_maps_grad_kernel<T>>(a.device, 2 * kMostChannels * sizeof(float))
                  ? launch_first(true, norm_maps_grad_kernel<T>, dim3((unsigned int)blocks), dim3(256), smem, s, a) : cudaErrorInvalidValue;
    } else if (a.c <= 256) {
        const int threads = short_row_threads(a);
        err = threads == 8 ? launch_grad_rows<T, 8, 1>(a, blocks, s) : threads == 16 ? launch_grad_rows<T, 16, 1>(a, blocks, s) : launch_grad_rows<T, 32, 1>(a, blocks, s);
    }
    else if (a.c <= 512) err = launch_grad<T, 2>(a, blocks, s);
    else if (a.c <= 1024) err = launch_grad<T, 4>(a, blocks, s);
    else if (a.c <= 2048) err = launch_grad<T, 8>(a, blocks, s);
    else if (a.c <= 4096) err = launch_grad<T, 16>(a, blocks, s);
    else if (a.c <= 8192) err = launch_grad<T, 32>(a, blocks, s);
    else err = launch_grad_rows<T, 1024, 2>(a, blocks, s);
    if (err != cudaSuccess) { cudaGetLastError(); return TC_ERR_CUDA; }
    return launch_chained(blocks > 0, norm_vectors_kernel, dim3((unsigned int)((a.c + 31) / 32)), dim3(kVectorWarps * 32), 0, s, a, blocks) == cudaSuccess ? TC_OK : TC_ERR_CUDA;
}

}  // namespace

tc_status tc_launch_residual_norms(const NormArgs &a, int dtype, cudaStream_t s)
{
    return dtype == TC_BF16 ? norms<__nv_bfloat16>(a, s) : norms<float>(a, s);
}

// Blocks of the gradient's kernel: as many as an SM holds of its row's or tile's size.
int tc_norm_grad_blocks(const NormGradArgs &a, int dtype, int sm_count)
{
    const size_t size = dtype == TC_BF16 ? 2 : 4;
    if (a.hw > 1)
        if (const MapPlan m = plan_grad_maps(a, size, sm_count); m.px) return (int)m.blocks;
    long long rows = a.pixels, per_sm = 1;
    if (a.hw > 1) { rows = (a.pixels + 31) / 32; per_sm = 4; }
    else if (a.c <= 256) { const int each = 256 / short_row_threads(a); rows = (a.pixels + each - 1) / each; per_sm = 2; }
    else
        for (int warps = 2; warps <= 16; warps *= 2)
            if (a.c <= 256 * warps) { per_sm = 16 * ring_chunks(warps, (int)size) / warps; break; }
    const long long most = per_sm * sm_count;
    return (int)(rows < most ? rows : most);
}

tc_status tc_launch_residual_norms_backward(const NormGradArgs &a, int dtype, int blocks, int sm_count, cudaStream_t s)
{
    return dtype == TC_BF16 ? gradient<__nv_bfloat16>(a, blocks, sm_count, s) : gradient<float>(a, blocks, sm_count, s);
}
