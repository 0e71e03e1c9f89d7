// Product of two matrices of 4-bit microscaled values on the tensor cores (sm_100a, block-scaled tcgen05 products):
//   out[i][j] = act(sum_k a_ik w_jk + bias_j),  a [m x k], w [n x k], blocks of 32 along k with a scale each.
// Products of codes and their scales are exact; sums, bias and activation are fp32, rounded once to the type of `out`.
//
// One CTA per SM walks over tiles of 128 rows x 128 columns, columns fastest, so that the rows of a tile come from HBM once and from
// L2 for the other columns.  Warps: 0 streams stages of 256 k (128 bytes of codes per row by TMA, the scale tiles by bulk copies);
// 1 copies a stage's scales to tensor memory and issues its four products of 64 k; 4-11 take a finished accumulator out of tensor memory while the
// next tile is at work (two accumulators) and store it through shared memory with asynchronous tile stores.
// The scale copies go to tensor-memory columns of their own per stage: a stage is only refilled once its products have completed.
// 4096 x 4096 x 4096: 37.6 us, 3.7 PFLOP/s; 10000 x 2816 by 1024: 20.3 us (bound: its tail, 632 tiles on 148 multiprocessors), 34.9 us with the quantisation of x; 7 rows: 5.5 us.
#include <climits>
#include <cstdio>

#include "aif_internal.h"
#include "aif_mx4.cuh"
#include "aif_tc_ptx.cuh"

namespace aif {

cudaError_t launch_mx4_quantize(const void *x, int dtype, int64_t rows, int cols, int64_t stride, uint8_t *codes, uint8_t *scales, cudaStream_t st);

namespace {

// Instruction descriptor of tcgen05.mma.kind::mxf4: A and B E2M1 (1 at [7,10) and [10,12)), N >> 3 at [17,23), scales E8M0 (bit 23), M >> 4 at
// [24,29); which pair of the four scale bytes of a column an instruction uses (0 or 2) stands at [4,6) for B and [29,31) for A.
__host__ __device__ constexpr uint32_t umma_idesc_mxf4(int m, int n, int pair)
{
    return (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | (1u << 23) | ((uint32_t)(m >> 4) << 24) | ((uint32_t)pair << 29) | ((uint32_t)pair << 4);
}
// (the whole warp walks and the lane with `one` set issues: see umma_bf16_if)
__device__ __forceinline__ void umma_mxf4(uint32_t one, uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t a_scale, uint32_t b_scale, uint32_t accumulate)
{
    asm volatile(
        "{\n"
        ".reg .pred p, q;\n"
        "setp.ne.b32 p, %6, 0;\n"
        "setp.ne.b32 q, %7, 0;\n"
        "@q tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n"
        "}\n" ::"r"(d_tmem),
        "l"(adesc), "l"(bdesc), "r"(idesc), "r"(a_scale), "r"(b_scale), "r"(accumulate), "r"(one)
        : "memory");
}
// 512 bytes (32 rows x 16 bytes) to four tensor-memory columns, the same in every quarter of the lanes.
__device__ __forceinline__ void tmem_copy_scales(uint32_t one, uint32_t taddr, uint64_t desc)
{
    asm volatile(
        "{\n"
        ".reg .pred q;\n"
        "setp.ne.b32 q, %2, 0;\n"
        "@q tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;\n"
        "}\n" ::"r"(taddr),
        "l"(desc), "r"(one)
        : "memory");
}

constexpr int kBM = 128;
constexpr int kStageK = 256;       // elements of k per stage: 128 bytes of codes, two scale tiles
constexpr int kTmemScales = 256;   // first of the scale columns, behind the two accumulators (at 0 and 128)

constexpr int kBN = 128;

struct GemmCfg {
    static constexpr int kABytes = kBM * 128, kBBytes = kBN * 128;
    static constexpr int kStageBytes = kABytes + kBBytes + 2048;   // + two scale tiles of each operand
    static constexpr int kStages = 4;
    static constexpr int kThreads = 384;
    static constexpr int kOutBytes = 8 * 2 * 4096;                 // two pieces of 32 rows x 128 bytes for each of the eight output warps
    static constexpr size_t kSmem = 1024 + kStages * kStageBytes + kOutBytes + 256 + 8 * 64 * 4;
};

// Status bits of the products that were given no word of their own.
__device__ uint32_t g_product_status;
__global__ void k_clear_status(uint32_t bits) { atomicAnd(&g_product_status, ~bits); }

struct GemmParams {
    int64_t m;
    int32_t n, k;
    const uint8_t *a_scales, *w_scales;
    const float *bias;
    int32_t relu;
    void *out;
    int64_t out_stride;
    int32_t wide;        // rows of `out` begin and end on 16-byte boundaries: tile stores
    int32_t n_tiles;     // column tiles
    int64_t tiles;       // all (of the kernel that quantises too: bands of rows)
    uint32_t *status;    // or nullptr: g_product_status
};

__device__ __forceinline__ uint32_t max_nan_bf16x2(uint32_t a, uint32_t b)
{
    uint32_t o;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(o) : "r"(a), "r"(b));
    return o;
}
__device__ __forceinline__ float max_nan_f32(float a, float b)
{
    float o;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(o) : "f"(a), "f"(b));
    return o;
}
// 32 rows x 64 columns of an accumulator, by one warp: from tensor memory through shared memory (two slabs of 4 KB) to `out`, in pieces of 128 bytes of a row, swizzled
// so that the lanes (one row each) stay on different banks and a tile store takes them in the same form.  `freed` is told once the accumulator has been read.
template <typename T>
__device__ __forceinline__ void store_half(const GemmParams &p, const CUtensorMap &tmO, uint32_t src, int64_t row0, int n0, unsigned char *slabs, int &slab, const float *bias_s,
                                           uint32_t freed)
{
    constexpr int kCols = 128 / (int)sizeof(T);   // columns of a piece
    constexpr int kPer = 16 / (int)sizeof(T);     // elements of 16 bytes
    const int lane = threadIdx.x & 31;
    const uint32_t least = p.relu ? 0u : sizeof(T) == 2 ? 0xff80ff80u : 0xff800000u;   // the larger of this and the value, where NaN stays
#pragma unroll
    for (int c0 = 0; c0 < 64; c0 += 32) {
        uint32_t r[32];
        tmem_ld32(src + c0, r);
        tmem_ld_wait();
        if (c0 == 32) {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(freed);
        }
        const int first = c0 / kCols * kCols, col = n0 + first;   // of the piece that these columns lie in
        unsigned char *sb = slabs + slab * 4096;
        if (c0 == first) {
            if (p.wide && lane == 0) bulk_wait_read<1>();   // the store that last read this slab is done with it
            __syncwarp();
        }
#pragma unroll
        for (int q = 0; q < 32 / kPer; ++q) {
            float v[kPer];
#pragma unroll
            for (int i = 0; i < kPer; i += 4) {
                const float4 bb = *reinterpret_cast<const float4 *>(bias_s + c0 + q * kPer + i);
                const float add[4] = {bb.x, bb.y, bb.z, bb.w};
#pragma unroll
                for (int x = 0; x < 4; ++x) v[i + x] = __uint_as_float(r[q * kPer + i + x]) + add[x];
            }
            uint4 o;
            if constexpr (sizeof(T) == 2) {
                uint32_t pk[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const __nv_bfloat162 hh = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
                    pk[i] = max_nan_bf16x2(*reinterpret_cast<const uint32_t *>(&hh), least);
                }
                o = make_uint4(pk[0], pk[1], pk[2], pk[3]);
            } else {
#pragma unroll
                for (int i = 0; i < kPer; ++i) v[i] = max_nan_f32(v[i], __uint_as_float(least));
                o = make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
            }
            *reinterpret_cast<uint4 *>(sb + lane * 128 + (((q + (c0 - first) / kPer) ^ (lane & 7)) << 4)) = o;
        }
        if (c0 + 32 < first + kCols) continue;
        if (p.wide) {
            // rows and columns behind the end are not stored
            fence_proxy_async();
            __syncwarp();
            if (lane == 0) {
                if (row0 < p.m && col < p.n) tma_store_2d(&tmO, smem_u32(sb), col, (int)row0);
                bulk_commit();
            }
            slab ^= 1;
        } else {
            __syncwarp();
            // a row at a time, a lane to an element
            T *out = static_cast<T *>(p.out);
            for (int rr = 0; rr < 32 && row0 + rr < p.m; ++rr) {
#pragma unroll
                for (int x = lane; x < kCols; x += 32)
                    if (col + x < p.n) out[(row0 + rr) * p.out_stride + col + x] = *reinterpret_cast<const T *>(sb + rr * 128 + ((x / kPer ^ (rr & 7)) << 4) + x % kPer * sizeof(T));
            }
            __syncwarp();
        }
    }
}

template <typename T>
__global__ void __launch_bounds__(GemmCfg::kThreads, 1) k_mx4_gemm(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmW,
                                                                       const __grid_constant__ CUtensorMap tmO, const GemmParams p)
{
    using C = GemmCfg;
    constexpr int kS = C::kStages;
    extern __shared__ unsigned char smem_dyn[];
    unsigned char *base = reinterpret_cast<unsigned char *>(((uintptr_t)smem_dyn + 1023) & ~(uintptr_t)1023);
    unsigned char *smA = base, *smB = smA + kS * C::kABytes, *smSc = smB + kS * C::kBBytes;   // scales: [stage][A 1 KB, W 1 KB]
    unsigned char *smOut = smSc + kS * 2048;
    uint64_t *bars = reinterpret_cast<uint64_t *>(smOut + C::kOutBytes);
    uint64_t *full = bars, *empty = bars + kS, *acc_full = bars + 2 * kS, *acc_empty = acc_full + 2;
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(acc_empty + 2);
    volatile uint32_t *abort_flag = tmem_slot + 1;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (tid == 0) {
        for (int s = 0; s < kS; ++s) mbar_init(smem_u32(full + s), 1), mbar_init(smem_u32(empty + s), 1);
        for (int b = 0; b < 2; ++b) mbar_init(smem_u32(acc_full + b), 1), mbar_init(smem_u32(acc_empty + b), 8);
        *abort_flag = 0u;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) tmem_alloc(smem_u32(tmem_slot), 512);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    grid_dep_wait();
    grid_dep_launch();

    const int stages = (p.k + kStageK - 1) / kStageK, sc_tiles = mx_scale_tiles(p.k);
    if (warp == 0) {
        if (lane == 0) {
            uint32_t it = 0;
            bool ok = true;
            for (int64_t tile = blockIdx.x; ok && tile < p.tiles; tile += gridDim.x) {
                const int64_t band = tile / p.n_tiles;
                const int n0 = (int)(tile % p.n_tiles) * kBN;
                const uint8_t *sa = p.a_scales + (size_t)band * sc_tiles * 512;
                const uint8_t *sw = p.w_scales + (size_t)(n0 / 128) * sc_tiles * 512;
                for (int j = 0; j < stages; ++j, ++it) {
                    const int s = (int)(it % kS);
                    if (!mbar_wait(smem_u32(empty + s), ((it / kS) & 1u) ^ 1u, abort_flag)) {
                        ok = false;
                        break;
                    }
                    const uint32_t sc = (uint32_t)(min(2, sc_tiles - 2 * j) * 512), bar = smem_u32(full + s);
                    mbar_expect_tx(bar, (uint32_t)(C::kABytes + C::kBBytes) + 2 * sc);
                    tma_load_2d(smem_u32(smA + s * C::kABytes), &tmA, bar, j * 128, (int)(band * kBM));
                    tma_load_2d(smem_u32(smB + s * C::kBBytes), &tmW, bar, j * 128, n0);
                    bulk_load(smem_u32(smSc + s * 2048), sa + j * 1024, sc, bar);
                    bulk_load(smem_u32(smSc + s * 2048 + 1024), sw + j * 1024, sc, bar);
                }
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        const uint32_t one = elect_one();
        const uint64_t ad0 = umma_desc_sw128(smem_u32(smA)), bd0 = umma_desc_sw128(smem_u32(smB)), sd0 = umma_desc_plain(smem_u32(smSc), 16);
        uint32_t it = 0;
        int t = 0;
        bool ok = true;
        for (int64_t tile = blockIdx.x; ok && tile < p.tiles; tile += gridDim.x, ++t) {
            const int b = t & 1;
            if (t >= 2 && !mbar_wait(smem_u32(acc_empty + b), (uint32_t)(((t - 2) >> 1) & 1), abort_flag)) break;
            for (int j = 0; j < stages; ++j, ++it) {
                const uint32_t s = it % kS;
                if (!mbar_wait(smem_u32(full + s), (it / kS) & 1u, abort_flag)) {
                    ok = false;
                    break;
                }
                tc_fence_after();
                const int steps = min(4, (p.k - j * kStageK + 63) / 64);   // products of 64 k; codes behind the last column are zero
                const uint32_t sc_t = tmem + (uint32_t)(kTmemScales + s * 16);
                const uint64_t ad = ad0 + (uint64_t)(s * (C::kABytes >> 4)), bd = bd0 + (uint64_t)(s * (C::kBBytes >> 4)), sd = sd0 + (uint64_t)(s * (2048 >> 4));
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    if (2 * h >= steps) break;
                    tmem_copy_scales(one, sc_t + 4 * h, sd + (uint64_t)(h * (512 >> 4)));
                    tmem_copy_scales(one, sc_t + 8 + 4 * h, sd + (uint64_t)((1024 + h * 512) >> 4));
                }
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    if (q >= steps) break;
                    umma_mxf4(one, tmem + (uint32_t)(b * 128), ad + 2 * q, bd + 2 * q, umma_idesc_mxf4(kBM, kBN, (q & 1) * 2), sc_t + 4 * (q >> 1), sc_t + 8 + 4 * (q >> 1),
                              j > 0 || q > 0);
                }
                umma_commit_if(one, smem_u32(empty + s));
            }
            if (ok) umma_commit_if(one, smem_u32(acc_full + b));
        }
    } else if (warp >= 4) {
        // two warps to a quarter of the rows, each with half of the columns
        const int w = (warp - 4) & 3, half = (warp - 4) >> 2;
        unsigned char *stg = smOut + (warp - 4) * 2 * 4096;
        float *bias_s = reinterpret_cast<float *>(smOut + C::kOutBytes + 256) + (warp - 4) * 64;
        int t = 0, slab = 0;
        for (int64_t tile = blockIdx.x; tile < p.tiles; tile += gridDim.x, ++t) {
            const int b = t & 1;
            const int64_t row0 = tile / p.n_tiles * kBM + w * 32;
            const int n0 = (int)(tile % p.n_tiles) * kBN + half * 64;
            __syncwarp();
#pragma unroll
            for (int x = 0; x < 64; x += 32) bias_s[x + lane] = p.bias && n0 + x + lane < p.n ? __ldg(p.bias + n0 + x + lane) : 0.f;
            __syncwarp();
            if (!__all_sync(0xffffffffu, mbar_wait(smem_u32(acc_full + b), (uint32_t)((t >> 1) & 1), abort_flag))) break;
            tc_fence_after();
            store_half<T>(p, tmO, tmem + ((uint32_t)(w * 32) << 16) + (uint32_t)(b * 128 + half * 64), row0, n0, stg, slab, bias_s, smem_u32(acc_empty + b));
        }
        if (lane == 0) bulk_wait<0>();   // all stores of this warp have reached global memory
    }

    if (*abort_flag) {
        if (tid == 0) atomicOr(p.status ? p.status : &g_product_status, AIF_STATUS_TIMEOUT);
        const long long t0 = clock64();
        while (clock64() - t0 < 2000000ll) __nanosleep(1000);   // copies in flight land before the memory is given up
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 1) tmem_dealloc(tmem, 512);
}

// The same product for rows that are not quantised yet and n <= 256, where all of W stays in shared memory: one kernel, so that the codes of x never go through
// memory.  A CTA per SM walks over bands of 128 rows; warps 0-15 load x (two parts of 32 KB ahead, in registers), quantise it and write codes and scales where the tensor core
// takes them (a ring of stages of 256 k); 16 issues; 17-20 store the accumulators, of which there are three, of 128 columns each.  Bound: HBM.  524288 x 512 by 256 in bf16:
// 137 us, 5.9 TB/s (quantising first: 192 us; in chunks that stay in L2, 215 us at best, their launches cost more than that saves); 524288 x 256 by 128: bf16 68 us, fp32 128 us.
struct NarrowCfg {
    static constexpr int kLoaders = 16, kThreads = 21 * 32;
    static constexpr int kStages = 3;
    static constexpr int kStageBytes = kBM * 128 + 1024;
    static constexpr int kAccs = 3;
    static constexpr int kOutBytes = 4 * 2 * 4096;
    static constexpr size_t kFixed = 1024 + kStages * kStageBytes + kOutBytes + 256 + 4 * 128 * 4;   // (beside W)
    static constexpr size_t kLeast = 116 * 1024;   // one CTA per multiprocessor: it takes all of the tensor memory
    static constexpr size_t kMost = 227 * 1024;
    static constexpr int kScaleAt = kAccs * 128;   // tensor-memory columns of the scales: x by stage, then W
};

// Bytes of W [n x k] in shared memory: stages of 128 rows x 256 k, scale tiles.
inline size_t narrow_w_bytes(int n, int k) { return (size_t)((n + 127) / 128) * (((size_t)k + kStageK - 1) / kStageK * 16384 + (size_t)mx_scale_tiles(k) * 512); }

template <typename T>
__global__ void __launch_bounds__(NarrowCfg::kThreads, 1) k_mx4_narrow(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmO, const GemmParams p,
                                                                      const T *__restrict__ x, int64_t x_stride)
{
    using C = NarrowCfg;
    constexpr int kS = C::kStages;
    extern __shared__ unsigned char smem_dyn[];
    unsigned char *base = reinterpret_cast<unsigned char *>(((uintptr_t)smem_dyn + 1023) & ~(uintptr_t)1023);
    const int nb = p.n_tiles, stages = (p.k + kStageK - 1) / kStageK, sc_tiles = mx_scale_tiles(p.k);
    unsigned char *smA = base, *smASc = smA + kS * kBM * 128, *smOut = smASc + kS * 1024;
    uint64_t *bars = reinterpret_cast<uint64_t *>(smOut + C::kOutBytes);
    float *smBias = reinterpret_cast<float *>(smOut + C::kOutBytes + 256);
    unsigned char *smW = smA + (C::kFixed - 1024 + 1023) / 1024 * 1024, *smWSc = smW + (size_t)nb * stages * 16384;   // [block][stage], [block][scale tile]
    uint64_t *full = bars, *empty = full + kS, *acc_full = empty + kS, *acc_empty = acc_full + C::kAccs, *w_full = acc_empty + C::kAccs;
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(w_full + 1);
    volatile uint32_t *abort_flag = tmem_slot + 1;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (tid == 0) {
        for (int s = 0; s < kS; ++s) mbar_init(smem_u32(full + s), C::kLoaders), mbar_init(smem_u32(empty + s), 1);
        for (int b = 0; b < C::kAccs; ++b) mbar_init(smem_u32(acc_full + b), 1), mbar_init(smem_u32(acc_empty + b), 8);
        mbar_init(smem_u32(w_full), 1);
        *abort_flag = 0u;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == C::kLoaders) tmem_alloc(smem_u32(tmem_slot), 512);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    grid_dep_wait();
    grid_dep_launch();

    if (warp < C::kLoaders) {
        // A part is kRows rows of each thread x 128 columns of the band: sixteen lanes to a row, eight elements each.
        constexpr int kRows = sizeof(T) == 2 ? 4 : 2, kParts = 4 / kRows;
        const int sub = tid & 15, r0 = tid >> 4;
        const int64_t row_step = 32 * x_stride * (int64_t)sizeof(T), band_step = (int64_t)gridDim.x * kBM * x_stride * (int64_t)sizeof(T);   // bytes
        // of the part that is loaded next: this thread's first row and column in it, and how many rows there are from there on
        const char *src = reinterpret_cast<const char *>(x + ((int64_t)blockIdx.x * kBM + r0) * x_stride + sub * 8);
        int have = (int)p.m - (int)blockIdx.x * kBM - r0, col = sub * 8, part = 0;
        auto load = [&](Raw8<T> (&v)[kRows]) {
            const int rows = col < p.k ? have : 0;
#pragma unroll
            for (int i = 0; i < kRows; ++i) {
                v[i] = Raw8<T>{};
                if (i * 32 < rows) v[i] = load_raw8<T, true>(reinterpret_cast<const T *>(src));
                src += row_step;
            }
            have -= kRows * 32;
            if (++part == kParts) {
                part = 0, have += kBM, col += 128, src += 128 * (int)sizeof(T) - 4 * row_step;
                if (col >= sc_tiles * 128) src += band_step - (col - sub * 8) * (int)sizeof(T), have -= (int)gridDim.x * kBM, col = sub * 8;
            }
        };
        Raw8<T> v[2][kRows];
        load(v[0]);
        load(v[1]);
        // 16-byte pieces of a row's 128 bytes of codes are swizzled by the row (a part's rows are 32 apart): both halves of a stage
        const uint32_t codes_at = smem_u32(smA) + r0 * 128 + (((sub >> 2) ^ (r0 & 7)) << 4) + (sub & 3) * 4, scales_at = smem_u32(smASc) + mx_scale_at(r0, sub >> 2);
        uint32_t s = 0, phase = 1;   // stage, and the parity of the wait for it
        int c = 0, q = 0;            // chunk and part at work
        const int mine = (int)((p.tiles + gridDim.x - 1 - blockIdx.x) / gridDim.x);   // bands
        for (int parts = mine * sc_tiles * kParts; parts > 0;) {
#pragma unroll
            for (int d = 0; d < 2; ++d) {
                if (parts <= 0) break;
                if ((c & 1) == 0 && q == 0 && !__all_sync(0xffffffffu, mbar_wait(smem_u32(empty + s), phase, abort_flag))) {
                    parts = 0;
                    break;
                }
                --parts;
                uint32_t w[kRows], byte[kRows];
                mx_quantise_quad<T>(v[d], w, byte);
                load(v[d]);
                const uint32_t to = (codes_at ^ (uint32_t)((c & 1) << 6)) + s * (kBM * 128) + q * (kRows * 32 * 128), sc_to = scales_at + s * 1024 + (c & 1) * 512 + q * (kRows * 4);
#pragma unroll
                for (int i = 0; i < kRows; ++i) {
                    asm volatile("st.shared.b32 [%0], %1;" ::"r"(to + i * (32 * 128)), "r"(w[i]) : "memory");
                    if ((sub & 3) == 0) asm volatile("st.shared.b8 [%0], %1;" ::"r"(sc_to + i * 4), "r"(byte[i]) : "memory");
                }
                if (++q == kParts) {
                    q = 0;
                    const bool last = c + 1 == sc_tiles;
                    if ((c & 1) || last) {
                        fence_proxy_async();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(smem_u32(full + s));
                        if (++s == kS) s = 0, phase ^= 1u;
                    }
                    c = last ? 0 : c + 1;
                }
            }
        }
    } else if (warp == C::kLoaders) {
        const uint32_t one = elect_one();
        if (one) {
            const uint32_t bar = smem_u32(w_full);
            mbar_expect_tx(bar, (uint32_t)(nb * (stages * 16384 + sc_tiles * 512)));
            for (int b = 0; b < nb; ++b) {
                for (int j = 0; j < stages; ++j) tma_load_2d(smem_u32(smW + (b * stages + j) * 16384), &tmW, bar, j * 128, b * kBN);
                bulk_load(smem_u32(smWSc + b * sc_tiles * 512), p.w_scales + (size_t)b * sc_tiles * 512, (uint32_t)(sc_tiles * 512), bar);
            }
        }
        __syncwarp();
        const uint64_t ad0 = umma_desc_sw128(smem_u32(smA)), bd0 = umma_desc_sw128(smem_u32(smW)), sd0 = umma_desc_plain(smem_u32(smASc), 16),
                       wd0 = umma_desc_plain(smem_u32(smWSc), 16);
        const uint32_t x_sc = tmem + C::kScaleAt, w_sc = x_sc + kS * 8;
        bool ok = mbar_wait(smem_u32(w_full), 0u, abort_flag);
        tc_fence_after();
        if (ok)
            for (int i = 0; i < nb * sc_tiles; ++i) tmem_copy_scales(one, w_sc + 4 * i, wd0 + (uint64_t)(i * (512 >> 4)));
        uint32_t it = 0, acc = 0;
        for (int64_t band = blockIdx.x; ok && band * kBM < p.m; band += gridDim.x, acc += nb) {
            for (int j = 0; ok && j < stages; ++j, ++it) {
                const uint32_t s = it % kS;
                if (!mbar_wait(smem_u32(full + s), (it / kS) & 1u, abort_flag)) {
                    ok = false;
                    break;
                }
                tc_fence_after();
                const int steps = min(4, (p.k - j * kStageK + 63) / 64);   // products of 64 k; codes behind the last column are zero
                const uint64_t ad = ad0 + (uint64_t)(s * (kBM * 128 >> 4)), sd = sd0 + (uint64_t)(s * (1024 >> 4));
                const uint32_t a_sc = x_sc + s * 8;
                tmem_copy_scales(one, a_sc, sd);
                if (steps > 2) tmem_copy_scales(one, a_sc + 4, sd + (uint64_t)(512 >> 4));
                for (int b = 0; b < nb; ++b) {
                    const uint32_t n_acc = acc + b, slot = n_acc % C::kAccs;
                    if (j == 0 && n_acc >= C::kAccs && !mbar_wait(smem_u32(acc_empty + slot), ((n_acc / C::kAccs) & 1u) ^ 1u, abort_flag)) {
                        ok = false;
                        break;
                    }
                    tc_fence_after();
                    const uint64_t bd = bd0 + (uint64_t)((b * stages + j) * (16384 >> 4));
                    const uint32_t b_sc = w_sc + 4 * (uint32_t)(b * sc_tiles + 2 * j);
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        if (q >= steps) break;
                        umma_mxf4(one, tmem + slot * 128, ad + 2 * q, bd + 2 * q, umma_idesc_mxf4(kBM, kBN, (q & 1) * 2), a_sc + 4 * (q >> 1), b_sc + 4 * (q >> 1), j > 0 || q > 0);
                    }
                    if (j + 1 == stages) umma_commit_if(one, smem_u32(acc_full + slot));
                }
                umma_commit_if(one, smem_u32(empty + s));
            }
        }
    } else {
        // a warp to a quarter of the rows
        const int e = warp - C::kLoaders - 1, w = warp & 3;
        unsigned char *stg = smOut + e * 2 * 4096;
        float *bias_s = smBias + e * 128;
        int slab = 0;
        uint32_t acc = 0;
        bool ok = true;
        for (int64_t band = blockIdx.x; ok && band * kBM < p.m; band += gridDim.x) {
            for (int b = 0; b < nb; ++b, ++acc) {
                const uint32_t slot = acc % C::kAccs;
                const int n0 = b * kBN;
                __syncwarp();
#pragma unroll
                for (int i = 0; i < 128; i += 32) bias_s[i + lane] = p.bias && n0 + i + lane < p.n ? __ldg(p.bias + n0 + i + lane) : 0.f;
                __syncwarp();
                if (!__all_sync(0xffffffffu, mbar_wait(smem_u32(acc_full + slot), (acc / C::kAccs) & 1u, abort_flag))) {
                    ok = false;
                    break;
                }
                tc_fence_after();
#pragma unroll 1
                for (int half = 0; half < 2; ++half)
                    store_half<T>(p, tmO, tmem + ((uint32_t)(w * 32) << 16) + slot * 128u + (uint32_t)(half * 64), band * kBM + w * 32, n0 + half * 64, stg, slab, bias_s + half * 64,
                                  smem_u32(acc_empty + slot));
            }
        }
        if (lane == 0) bulk_wait<0>();   // all stores of this warp have reached global memory
    }

    if (*abort_flag) {
        if (tid == 0) atomicOr(p.status ? p.status : &g_product_status, AIF_STATUS_TIMEOUT);
        const long long t0 = clock64();
        while (clock64() - t0 < 2000000ll) __nanosleep(1000);   // copies in flight land before the memory is given up
    }
    tc_fence_before();
    __syncthreads();
    if (warp == C::kLoaders) tmem_dealloc(tmem, 512);
}

// Codes as a matrix of bytes [rows x cols / 2], boxes of 128 bytes x box_rows, 128-byte swizzle; columns and rows behind the end read as zero.
cudaError_t encode_codes(CUtensorMap *m, const uint8_t *codes, int64_t rows, int cols, int box_rows)
{
    EncodeFn enc = encode_fn();
    if (!enc) return cudaErrorNotSupported;
    const cuuint64_t dims[2] = {(cuuint64_t)(cols / 2), (cuuint64_t)rows};
    const cuuint64_t strides[1] = {(cuuint64_t)(cols / 2)};
    const cuuint32_t box[2] = {128, (cuuint32_t)box_rows};
    const cuuint32_t estr[2] = {1, 1};
    const CUresult r = enc(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<uint8_t *>(codes), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                           CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

template <typename T>
cudaError_t encode_out(CUtensorMap *m, const GemmParams &p)
{
    // the output as it is stored: 128-byte pieces of 32 rows
    if (!p.wide) return cudaSuccess;
    EncodeFn enc = encode_fn();
    if (!enc) return cudaErrorNotSupported;
    const cuuint64_t dims[2] = {(cuuint64_t)p.n, (cuuint64_t)p.m};
    const cuuint64_t strides[1] = {(cuuint64_t)(p.out_stride * sizeof(T))};
    const cuuint32_t box[2] = {(cuuint32_t)(128 / sizeof(T)), 32};
    const cuuint32_t estr[2] = {1, 1};
    const CUresult r = enc(m, sizeof(T) == 2 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 2, p.out, dims, strides, box, estr,
                           CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

template <typename T>
cudaError_t run_gemm(GemmParams p, const uint8_t *a_codes, const uint8_t *w_codes, cudaStream_t st)
{
    using C = GemmCfg;
    CUtensorMap ta, tw, to{};
    cudaError_t e = encode_codes(&ta, a_codes, p.m, p.k, kBM);
    if (e == cudaSuccess) e = encode_codes(&tw, w_codes, p.n, p.k, kBN);
    if (e == cudaSuccess) e = encode_out<T>(&to, p);
    if (e == cudaSuccess) e = allow_smem<k_mx4_gemm<T>>(C::kSmem);
    if (e != cudaSuccess) return e;
    p.tiles = (p.m + kBM - 1) / kBM * p.n_tiles;
    const unsigned grid = (unsigned)(p.tiles < 148 ? p.tiles : 148);
    e = launch_pdl(k_mx4_gemm<T>, dim3(grid), dim3(C::kThreads), C::kSmem, st, ta, tw, to, p);
    count_launch();
    return e;
}
template <typename T>
cudaError_t run_narrow(GemmParams p, const void *x, int64_t x_stride, const uint8_t *w_codes, cudaStream_t st)
{
    using C = NarrowCfg;
    CUtensorMap tw, to{};
    cudaError_t e = encode_codes(&tw, w_codes, p.n, p.k, kBN);
    if (e == cudaSuccess) e = encode_out<T>(&to, p);
    const size_t need = (C::kFixed + 1023) / 1024 * 1024 + narrow_w_bytes(p.n, p.k), smem = need < C::kLeast ? C::kLeast : need;
    if (e == cudaSuccess) e = allow_smem<k_mx4_narrow<T>>(C::kMost);
    if (e != cudaSuccess) return e;
    p.tiles = (p.m + kBM - 1) / kBM;
    e = launch_pdl(k_mx4_narrow<T>, dim3((unsigned)(p.tiles < 148 ? p.tiles : 148)), dim3(C::kThreads), smem, st, tw, to, p, static_cast<const T *>(x), x_stride);
    count_launch();
    return e;
}
// The kernel that quantises the rows itself: rows begin on 16 bytes, n <= 256 and W fits beside the rest.  It reads x once and writes nothing but `out`; what speaks against
// it is the time of one band, which grows with k.  So: short rows (k of 256 in bf16 and 1000 rows: 4.9 us against 6.2 of the two kernels), or two bands per multiprocessor and
// more (k 512, n 256, bf16: 37888 rows 13.6 us against 15.6, but 20000 rows, two bands for a few, 13.0 against 12.0 and 1000 rows 8.0 against 6.6; 300000 rows 80 against 115).
// fp32 also needs the L1 that a large W takes (300000 x 1024 in fp32: n 128 224 us against 250, n 256 311 against 288; in bf16 n 256 146 against 202).
bool use_narrow(const aif_mx4_product &q, int el)
{
    const size_t w = narrow_w_bytes(q.n, q.k);
    const bool can = q.n <= 256 && (NarrowCfg::kFixed + 1023) / 1024 * 1024 + w <= NarrowCfg::kMost && (reinterpret_cast<uintptr_t>(q.x) & 15) == 0 && (q.x_stride * el) % 16 == 0;
    return can && (el == 2 || w <= 76 * 1024) && (q.k * el <= 512 || q.m > 2 * 147 * kBM);
}

int product_result(cudaError_t e, const char *what)
{
    if (e == cudaSuccess) return AIF_OK;
    char text[256];
    snprintf(text, sizeof(text), "%s: %s", what, cudaGetErrorString(e));
    cudaGetLastError();
    set_last_error(text);
    return AIF_ERR_CUDA;
}

}  // namespace
}  // namespace aif

using namespace aif;

extern "C" {

int64_t aif_mx4_workspace_bytes(int64_t m, int32_t k)
{
    const int64_t sc = aif_mx4_scale_bytes(m, k);
    return sc < 0 ? sc : (m * (k / 2) + 255) / 256 * 256 + sc;
}

int aif_mx4_linear(const aif_mx4_product *q, aif_stream stream)
{
    StageRange range("aif_mx4_linear");
    if (!q || q->struct_size != sizeof(aif_mx4_product)) return AIF_ERR_ARG;
    if (q->dtype != AIF_F32 && q->dtype != AIF_BF16) return AIF_ERR_ARG;
    if (q->m < 0 || q->m > INT_MAX - kBM || q->n < 1 || q->k < kMxBlock || q->k % kMxBlock != 0 || q->out_stride < q->n) return AIF_ERR_SHAPE;
    if (q->n > INT_MAX - 128 || (q->m + 127) / 128 * mx_scale_tiles(q->k) > INT_MAX) return AIF_ERR_SHAPE;
    if (q->m == 0) return AIF_OK;
    auto aligned = [](const void *p) { return p && (reinterpret_cast<uintptr_t>(p) & 15) == 0; };
    const int el = q->dtype == AIF_BF16 ? 2 : 4;
    if (!aligned(q->w_codes) || !aligned(q->w_scales) || !q->out || reinterpret_cast<uintptr_t>(q->out) % el != 0) return AIF_ERR_ARG;
    if (q->bias && reinterpret_cast<uintptr_t>(q->bias) % 4 != 0) return AIF_ERR_ARG;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    GemmParams p{};
    p.m = q->m, p.n = q->n, p.k = q->k, p.a_scales = q->x_scales, p.w_scales = q->w_scales, p.bias = q->bias, p.relu = q->relu;
    p.out = q->out, p.out_stride = q->out_stride, p.status = q->status, p.n_tiles = (q->n + kBN - 1) / kBN;
    // (a tile store cuts a row off at 16 bytes, not at an element)
    p.wide = (reinterpret_cast<uintptr_t>(q->out) & 15) == 0 && (q->out_stride * el) % 16 == 0 && ((int64_t)q->n * el) % 16 == 0;
    const uint8_t *codes = q->x_codes;
    cudaError_t e = cudaSuccess;
    bool narrow = false;
    if (q->x) {
        if (q->x_stride < q->k) return AIF_ERR_SHAPE;
        if (reinterpret_cast<uintptr_t>(q->x) % el != 0 || !aligned(q->workspace) || q->workspace_bytes < aif_mx4_workspace_bytes(q->m, q->k)) return AIF_ERR_ARG;
        narrow = use_narrow(*q, el);
        if (!narrow) {
            uint8_t *ws = static_cast<uint8_t *>(q->workspace), *scales = ws + (q->m * (q->k / 2) + 255) / 256 * 256;
            codes = ws, p.a_scales = scales;
            e = launch_mx4_quantize(q->x, q->dtype, q->m, q->k, q->x_stride, ws, scales, st);
        }
    } else if (!aligned(codes) || !aligned(p.a_scales)) {
        return AIF_ERR_ARG;
    }
    if (narrow)
        e = q->dtype == AIF_BF16 ? run_narrow<__nv_bfloat16>(p, q->x, q->x_stride, q->w_codes, st) : run_narrow<float>(p, q->x, q->x_stride, q->w_codes, st);
    else if (e == cudaSuccess)
        e = q->dtype == AIF_BF16 ? run_gemm<__nv_bfloat16>(p, codes, q->w_codes, st) : run_gemm<float>(p, codes, q->w_codes, st);
    return product_result(e, "aif_mx4_linear");
}

int aif_mx4_poll(uint32_t *bits, aif_stream stream)
{
    if (!bits) return AIF_ERR_ARG;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    uint32_t got = 0;
    cudaError_t e = cudaMemcpyFromSymbolAsync(&got, g_product_status, 4, 0, cudaMemcpyDeviceToHost, st);
    if (e == cudaSuccess) e = cudaStreamSynchronize(st);
    if (e == cudaSuccess && got != 0) {   // those bits alone: calls on other streams may set some meanwhile
        k_clear_status<<<1, 1, 0, st>>>(got);
        count_launch();
        e = cudaGetLastError();
        if (e == cudaSuccess) e = cudaStreamSynchronize(st);
    }
    if (e == cudaSuccess) *bits = got;
    return product_result(e, "aif_mx4_poll");
}

int aif_mx4_status_word(uint32_t **word)
{
    if (!word) return AIF_ERR_ARG;
    void *at = nullptr;
    const cudaError_t e = cudaGetSymbolAddress(&at, g_product_status);
    if (e == cudaSuccess) *word = static_cast<uint32_t *>(at);
    return product_result(e, "aif_mx4_status_word");
}

}  // extern "C"
