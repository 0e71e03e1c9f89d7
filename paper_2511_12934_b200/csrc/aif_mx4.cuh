// 4-bit microscaled values: E2M1 codes (sign, two exponent bits, one mantissa bit: 0, .5, 1, 1.5, 2, 3, 4, 6) in blocks of 32
// that share a power of two, kept as a byte b = exponent + 127 (E8M0).  Two codes to a byte, the first in the low half.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace aif {
namespace {

constexpr int kMxBlock = 32;      // elements that share a scale
constexpr uint32_t kMxNan = 255;  // scale byte of a block that holds an infinity or NaN: every value of it is NaN

// Scale byte of a block whose largest magnitude has this exponent field: the exponent of the largest value less the two of
// the largest code, never below 2^-127.  A plain difference of exponent fields, subnormal blocks included.
__device__ __forceinline__ uint32_t mx_scale_byte(uint32_t field)
{
    return field == 255u ? kMxNan : field > 2u ? field - 2u : 0u;
}
// 2^(127 - byte) for the byte of a block without infinities; its products with the block's elements are exact.
__device__ __forceinline__ float mx_inverse_scale(uint32_t byte) { return byte == kMxNan ? 0.f : __uint_as_float((254u - byte) << 23); }
// 2^(byte - 127); NaN for kMxNan.
__device__ __forceinline__ float mx_scale(uint32_t byte)
{
    return __uint_as_float(byte == 0u ? 0x00400000u : byte == kMxNan ? 0x7fffffffu : byte << 23);
}

// Eight values -> eight codes, to nearest (ties to the code with a zero mantissa bit), saturating at +-6.
__device__ __forceinline__ uint32_t mx_encode8(const float (&v)[8])
{
    uint32_t w;
    asm("{\n"
        ".reg .b8 a, b, c, d;\n"
        "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n"
        "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n"
        "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n"
        "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n"
        "mov.b32 %0, {a, b, c, d};\n"
        "}\n"
        : "=r"(w)
        : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
    return w;
}
// Eight codes -> four pairs of fp16 (exact, unscaled): o[i] = values 2 i and 2 i + 1.
__device__ __forceinline__ void mx_decode8_f16(uint32_t w, uint32_t (&o)[4])
{
    asm("{\n"
        ".reg .b8 a, b, c, d;\n"
        "mov.b32 {a, b, c, d}, %4;\n"
        "cvt.rn.f16x2.e2m1x2 %0, a;\n"
        "cvt.rn.f16x2.e2m1x2 %1, b;\n"
        "cvt.rn.f16x2.e2m1x2 %2, c;\n"
        "cvt.rn.f16x2.e2m1x2 %3, d;\n"
        "}\n"
        : "=r"(o[0]), "=r"(o[1]), "=r"(o[2]), "=r"(o[3])
        : "r"(w));
}
__device__ __forceinline__ float2 half2_to_float2(uint32_t h) { return __half22float2(*reinterpret_cast<const __half2 *>(&h)); }

// Eight consecutive elements of storage type T as they are stored.  ALIGNED: the address is a multiple of 16 bytes.
template <typename T>
struct Raw8 {
    uint32_t w[2 * sizeof(T)];
};
template <typename T, bool ALIGNED>
__device__ __forceinline__ Raw8<T> load_raw8(const T *p)
{
    Raw8<T> r;
    if constexpr (!ALIGNED) {
        if constexpr (sizeof(T) == 2) {
            const uint16_t *q = reinterpret_cast<const uint16_t *>(p);
#pragma unroll
            for (int i = 0; i < 4; ++i) r.w[i] = (uint32_t)__ldg(q + 2 * i) | (uint32_t)__ldg(q + 2 * i + 1) << 16;
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) r.w[i] = __float_as_uint(__ldg(p + i));
        }
    } else {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
            const uint4 x = __ldg(reinterpret_cast<const uint4 *>(p) + i);
            r.w[4 * i] = x.x, r.w[4 * i + 1] = x.y, r.w[4 * i + 2] = x.z, r.w[4 * i + 3] = x.w;
        }
    }
    return r;
}
template <typename T>
__device__ __forceinline__ void widen8(const Raw8<T> &r, float (&v)[8])
{
    if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[2 * i] = __uint_as_float(r.w[i] << 16), v[2 * i + 1] = __uint_as_float(r.w[i] & 0xffff0000u);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(r.w[i]);
    }
}
template <typename T, bool ALIGNED>
__device__ __forceinline__ void load8(const T *p, float (&v)[8])
{
    widen8<T>(load_raw8<T, ALIGNED>(p), v);
}
template <typename T, bool ALIGNED>
__device__ __forceinline__ void store8(T *p, const float (&v)[8])
{
    if constexpr (!ALIGNED) {
#pragma unroll
        for (int i = 0; i < 8; ++i) p[i] = (T)v[i];
    } else if constexpr (sizeof(T) == 2) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
            w[i] = *reinterpret_cast<const uint32_t *>(&h);
        }
        *reinterpret_cast<uint4 *>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    } else {
        reinterpret_cast<float4 *>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
        reinterpret_cast<float4 *>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
    }
}

// Larger of two pairs of bf16 magnitudes, NaN is the largest; signs mean nothing.
__device__ __forceinline__ uint32_t max_abs_bf16x2(uint32_t a, uint32_t b)
{
    uint32_t o;
    asm("max.NaN.xorsign.abs.bf16x2 %0, %1, %2;" : "=r"(o) : "r"(a), "r"(b));
    return o;
}
__device__ __forceinline__ float max_abs_f32(float a, float b)
{
    float o;
    asm("max.NaN.xorsign.abs.f32 %0, %1, %2;" : "=f"(o) : "f"(a), "f"(b));
    return o;
}
// Two bf16 values times a power of two (its upper half), exactly, as fp32; -0 stays.
__device__ __forceinline__ void scale_bf16x2(uint32_t x, uint32_t power, float &lo, float &hi)
{
    asm("{\n"
        ".reg .b16 l, h, none, p;\n"
        "mov.b32 {l, h}, %2;\n"
        "mov.b32 {none, p}, %3;\n"
        "fma.rn.f32.bf16 %0, l, p, %4;\n"
        "fma.rn.f32.bf16 %1, h, p, %4;\n"
        "}\n"
        : "=f"(lo), "=f"(hi)
        : "r"(x), "r"(power), "f"(-0.f));
}
// Four neighbouring lanes (4 i .. 4 i + 3, converged) quantise the 32 elements of each of N blocks, eight each: the lane's codes, and the blocks' scale bytes.  Blocks go in
// pairs: their largest magnitudes (the upper 16 bits say all that is needed of them) share a register on their way through the lanes.
template <typename T, int N>
__device__ __forceinline__ void mx_quantise_quad(const Raw8<T> (&x)[N], uint32_t (&w)[N], uint32_t (&byte)[N])
{
    static_assert(N % 2 == 0, "blocks go in pairs");
#pragma unroll
    for (int n = 0; n < N; n += 2) {
        uint32_t top;   // of block n in the lower half
        if constexpr (sizeof(T) == 2) {
            uint32_t m[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) m[i] = max_abs_bf16x2(max_abs_bf16x2(x[n + i].w[0], x[n + i].w[1]), max_abs_bf16x2(x[n + i].w[2], x[n + i].w[3]));
            top = max_abs_bf16x2(__byte_perm(m[0], m[1], 0x5410), __byte_perm(m[0], m[1], 0x7632));
        } else {
            float m[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                m[i] = __uint_as_float(x[n + i].w[0]);
#pragma unroll
                for (int e = 1; e < 8; ++e) m[i] = max_abs_f32(m[i], __uint_as_float(x[n + i].w[e]));
            }
            top = __byte_perm(__float_as_uint(m[0]), __float_as_uint(m[1]), 0x7632);
        }
        top = max_abs_bf16x2(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = max_abs_bf16x2(top, __shfl_xor_sync(0xffffffffu, top, 2));
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t b = mx_scale_byte((top >> (i ? 23 : 7)) & 0xffu), inv = __float_as_uint(mx_inverse_scale(b));
            float v[8];
            if constexpr (sizeof(T) == 2) {
#pragma unroll
                for (int e = 0; e < 4; ++e) scale_bf16x2(x[n + i].w[e], inv, v[2 * e], v[2 * e + 1]);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = __uint_as_float(x[n + i].w[e]) * __uint_as_float(inv);
            }
            const uint32_t codes = mx_encode8(v);
            w[n + i] = b == kMxNan ? 0u : codes, byte[n + i] = b;
        }
    }
}
// The values of eight codes of a block with this scale.
__device__ __forceinline__ void mx_values8(uint32_t codes, float scale, float (&v)[8])
{
    uint32_t h[4];
    mx_decode8_f16(codes, h);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = half2_to_float2(h[i]);
        v[2 * i] = f.x * scale, v[2 * i + 1] = f.y * scale;
    }
}

__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t a, uint32_t b)
{
    uint32_t o;
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(o) : "r"(a), "r"(b));
    return o;
}

// Eight codes to four bf16 pairs.  A code's exponent and mantissa bits are put where bf16 has its lowest exponent bits and its highest mantissa bit:
// the value times 2^-126, subnormal codes included, and one exact multiplication by 2^126 times the block's scale makes it the value.
// Scales beyond 2 (byte > 128) would need a factor beyond the largest power of two: they take two steps.
struct UnpackScale {
    uint32_t first, second;   // bf16 pairs
    bool two;
    __device__ __forceinline__ explicit UnpackScale(uint32_t byte)
    {
        two = byte > 128u;
        const uint32_t f = two ? 253u << 7 : (byte + 126u) << 7, s = byte == kMxNan ? 0x7fffu : byte << 7;
        first = f | (f << 16), second = s | (s << 16);
    }
};
// (times the first factor alone)
__device__ __forceinline__ uint4 unpack8_first(uint32_t w, uint32_t first)
{
    uint4 o;
    o.x = ((w << 12) & 0x80008000u) | ((w << 6) & 0x01c001c0u);
    o.y = ((w << 8) & 0x80008000u) | ((w << 2) & 0x01c001c0u);
    o.z = ((w << 4) & 0x80008000u) | ((w >> 2) & 0x01c001c0u);
    o.w = (w & 0x80008000u) | ((w >> 6) & 0x01c001c0u);
    o.x = mul_bf16x2(o.x, first), o.y = mul_bf16x2(o.y, first), o.z = mul_bf16x2(o.z, first), o.w = mul_bf16x2(o.w, first);
    return o;
}
__device__ __forceinline__ uint4 unpack8(uint32_t w, const UnpackScale &s)
{
    uint4 o = unpack8_first(w, s.first);
    if (s.two) o.x = mul_bf16x2(o.x, s.second), o.y = mul_bf16x2(o.y, s.second), o.z = mul_bf16x2(o.z, s.second), o.w = mul_bf16x2(o.w, s.second);
    return o;
}

// Scale bytes of a matrix lie in tiles of 128 rows x 4 blocks, 512 bytes each, the tiles of a band of 128 rows one after the other:
// byte (row, block) at (row / 128 * tiles + block / 4) * 512 + row % 32 * 16 + row % 128 / 32 * 4 + block % 4, which is the order in
// which the block-scaled products read 32 rows x 16 bytes into tensor memory.
__host__ __device__ __forceinline__ int mx_scale_tiles(int cols) { return (cols + 4 * kMxBlock - 1) / (4 * kMxBlock); }
__device__ __forceinline__ int mx_scale_at(int row_in_band, int block_in_tile) { return (row_in_band & 31) * 16 + (row_in_band >> 5) * 4 + block_in_tile; }

}  // namespace
}  // namespace aif
