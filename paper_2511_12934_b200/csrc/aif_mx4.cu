// Quantisation of matrices to 4-bit microscaled values and back (see aif_mx4.cuh for the format).
//
// Both are one pass over the data, bound by HBM.  A CTA takes 128 rows x 128 columns, the region of one 512-byte tile of scale
// bytes, so that the tile leaves in one coalesced store; sixteen lanes read 256 (bf16) consecutive bytes of a row, four of them share a block.
// 524288 x 512: bf16 120 us (5.7 TB/s) and back 137 us (4.9 TB/s), fp32 173 us (7.0 TB/s; part of it still in L2 from the call before) and back 240 us (5.1 TB/s).
#include <climits>
#include <cstdio>

#include "aif_internal.h"
#include "aif_mx4.cuh"
#include "aif_tc_ptx.cuh"

namespace aif {
namespace {

constexpr int kTile = 128;

template <typename T, bool ALIGNED>
__global__ void __launch_bounds__(256) k_mx4_quantize(const T *__restrict__ x, int64_t rows, int cols, int64_t stride, uint8_t *__restrict__ codes,
                                                      uint8_t *__restrict__ scales)
{
    __shared__ __align__(16) uint8_t tile[512];
    grid_dep_wait();
    const int kt = mx_scale_tiles(cols);
    const int64_t band = blockIdx.x / kt;
    const int t = (int)(blockIdx.x % kt);
    const int tid = threadIdx.x, sub = tid & 15;
    const int col = t * kTile + sub * 8;
    // four rows of a thread in flight at a time
#pragma unroll
    for (int i0 = 0; i0 < 8; i0 += 4) {
        Raw8<T> v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t row = band * kTile + (i0 + i) * 16 + (tid >> 4);
            v[i] = Raw8<T>{};
            if (row < rows && col < cols) v[i] = load_raw8<T, ALIGNED>(x + row * stride + col);
        }
        uint32_t w[4], byte[4];
        mx_quantise_quad<T>(v, w, byte);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = (i0 + i) * 16 + (tid >> 4);
            const int64_t row = band * kTile + r;
            const bool in = row < rows && col < cols;   // the four lanes of a block agree: cols is a multiple of 32
            if (in) *reinterpret_cast<uint32_t *>(codes + row * (cols / 2) + col / 2) = w[i];
            if ((sub & 3) == 0) tile[mx_scale_at(r, sub >> 2)] = (uint8_t)(in ? byte[i] : 0u);   // padding: 2^-127, which times a zero code is nothing
        }
    }
    // The product that may follow takes its place beside the last CTAs: 37.1 us against 38.4 (10000 x 2816 by 1024, with the product); in
    // a grid of many waves its CTAs would take the place of this kernel's (524288 x 512 by 256: 207 us against 203.6).
    if (gridDim.x <= 2 * 8 * 148) grid_dep_launch();
    __syncthreads();
    if (tid < 32) reinterpret_cast<uint4 *>(scales + (size_t)blockIdx.x * 512)[tid] = reinterpret_cast<const uint4 *>(tile)[tid];
}

template <typename T, bool ALIGNED>
__global__ void __launch_bounds__(256) k_mx4_dequantize(const uint8_t *__restrict__ codes, const uint8_t *__restrict__ scales, int64_t rows, int cols,
                                                        T *__restrict__ out, int64_t stride)
{
    __shared__ __align__(16) uint8_t tile[512];
    const int kt = mx_scale_tiles(cols);
    const int64_t band = blockIdx.x / kt;
    const int t = (int)(blockIdx.x % kt);
    const int tid = threadIdx.x, sub = tid & 15;
    const int col = t * kTile + sub * 8;
    if (tid < 32) reinterpret_cast<uint4 *>(tile)[tid] = __ldg(reinterpret_cast<const uint4 *>(scales + (size_t)blockIdx.x * 512) + tid);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int r = i * 16 + (tid >> 4);
        const int64_t row = band * kTile + r;
        if (row < rows && col < cols) {
            float v[8];
            mx_values8(__ldg(reinterpret_cast<const uint32_t *>(codes + row * (cols / 2) + col / 2)), mx_scale(tile[mx_scale_at(r, sub >> 2)]), v);
            store8<T, ALIGNED>(out + row * stride + col, v);
        }
    }
}

bool aligned16(const void *p, int64_t stride_bytes) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0 && (stride_bytes & 15) == 0; }

int check_matrix(int32_t dtype, int64_t rows, int32_t cols, int64_t stride)
{
    if (dtype != AIF_F32 && dtype != AIF_BF16) return AIF_ERR_ARG;
    if (rows < 0 || cols < kMxBlock || cols % kMxBlock != 0 || stride < cols) return AIF_ERR_SHAPE;
    // one CTA per tile of 128 x 128: as many as a grid has
    if ((rows + kTile - 1) / kTile * mx_scale_tiles(cols) > INT_MAX) return AIF_ERR_SHAPE;
    return AIF_OK;
}

int launched(cudaError_t e, const char *what)
{
    if (e == cudaSuccess) return AIF_OK;
    char text[256];
    snprintf(text, sizeof(text), "%s: %s", what, cudaGetErrorString(e));
    set_last_error(text);
    return AIF_ERR_CUDA;
}

}  // namespace

cudaError_t launch_mx4_quantize(const void *x, int dtype, int64_t rows, int cols, int64_t stride, uint8_t *codes, uint8_t *scales, cudaStream_t st)
{
    const unsigned grid = (unsigned)((rows + kTile - 1) / kTile * mx_scale_tiles(cols));
    const bool al = aligned16(x, stride * (dtype == AIF_BF16 ? 2 : 4));
    // At most a CTA per multiprocessor: their launch overlaps the end of the kernel before (7 x 2816 by 1024 in a run of layers: 8.1 us against 8.5).  Beyond that the CTAs
    // share multiprocessors that are still set up for the shared memory of the product before: 13.4 us against 11.1 for 4001 x 1024 by 520, 172 against 160 for
    // 524288 x 256 by 128 in fp32.
    auto go = [&](auto kernel, auto *p) {
        if (grid <= 148) return launch_pdl(kernel, dim3(grid), dim3(256), 0, st, p, rows, cols, stride, codes, scales);
        kernel<<<grid, 256, 0, st>>>(p, rows, cols, stride, codes, scales);
        return cudaGetLastError();
    };
    cudaError_t e;
    if (dtype == AIF_BF16) {
        auto *p = static_cast<const __nv_bfloat16 *>(x);
        e = al ? go(k_mx4_quantize<__nv_bfloat16, true>, p) : go(k_mx4_quantize<__nv_bfloat16, false>, p);
    } else {
        auto *p = static_cast<const float *>(x);
        e = al ? go(k_mx4_quantize<float, true>, p) : go(k_mx4_quantize<float, false>, p);
    }
    count_launch();
    return e;
}

}  // namespace aif

using namespace aif;

extern "C" {

int64_t aif_mx4_scale_bytes(int64_t rows, int32_t cols)
{
    if (rows < 0 || cols < kMxBlock || cols % kMxBlock != 0) return AIF_ERR_SHAPE;
    return (rows + kTile - 1) / kTile * mx_scale_tiles(cols) * 512;
}

int aif_mx4_quantize(const void *x, int32_t dtype, int64_t rows, int32_t cols, int64_t x_stride, uint8_t *codes, uint8_t *scales, aif_stream stream)
{
    StageRange range("aif_mx4_quantize");
    const int rc = check_matrix(dtype, rows, cols, x_stride);
    if (rc != AIF_OK) return rc;
    if (rows == 0) return AIF_OK;
    if (!x || !codes || !scales || !aligned16(codes, 0) || !aligned16(scales, 0)) return AIF_ERR_ARG;
    if (reinterpret_cast<uintptr_t>(x) % (dtype == AIF_BF16 ? 2 : 4) != 0) return AIF_ERR_ARG;
    return launched(launch_mx4_quantize(x, dtype, rows, cols, x_stride, codes, scales, reinterpret_cast<cudaStream_t>(stream)), "aif_mx4_quantize");
}

int aif_mx4_dequantize(const uint8_t *codes, const uint8_t *scales, int64_t rows, int32_t cols, void *out, int32_t dtype, int64_t out_stride,
                       aif_stream stream)
{
    StageRange range("aif_mx4_dequantize");
    const int rc = check_matrix(dtype, rows, cols, out_stride);
    if (rc != AIF_OK) return rc;
    if (rows == 0) return AIF_OK;
    if (!out || !codes || !scales || !aligned16(codes, 0) || !aligned16(scales, 0)) return AIF_ERR_ARG;
    const int el = dtype == AIF_BF16 ? 2 : 4;
    if (reinterpret_cast<uintptr_t>(out) % el != 0) return AIF_ERR_ARG;
    const unsigned grid = (unsigned)((rows + kTile - 1) / kTile * mx_scale_tiles(cols));
    const bool al = aligned16(out, out_stride * el);
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    auto go = [&](auto kernel, auto *p) { kernel<<<grid, 256, 0, st>>>(codes, scales, rows, cols, p, out_stride); };
    if (dtype == AIF_BF16) {
        auto *p = static_cast<__nv_bfloat16 *>(out);
        al ? go(k_mx4_dequantize<__nv_bfloat16, true>, p) : go(k_mx4_dequantize<__nv_bfloat16, false>, p);
    } else {
        auto *p = static_cast<float *>(out);
        al ? go(k_mx4_dequantize<float, true>, p) : go(k_mx4_dequantize<float, false>, p);
    }
    count_launch();
    return launched(cudaGetLastError(), "aif_mx4_dequantize");
}

}  // extern "C"
