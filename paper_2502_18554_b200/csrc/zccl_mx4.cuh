// Microscaled 4-bit floating point: the arithmetic of a block and the layout of the scales.  Not installed.
#pragma once
#include "zccl_device.cuh"

#include <cuda_bf16.h>
#include <cuda_fp16.h>

namespace zccl {

constexpr int kMxBlock = 32;              // elements that share a scale
constexpr int kMxGroup = 4 * kMxBlock;    // elements of a row that a tile of scales covers
constexpr int kMxBand = 128;              // rows that a tile of scales covers
constexpr int kMxTileBytes = 512;
constexpr size_t kMxMaxGroups = 0x7FFFFFFFu;   // (row, group) pairs are counted in 32 bits: 2^38 elements

__host__ __device__ inline size_t mx_blocks(size_t cols) { return (cols + kMxBlock - 1) / kMxBlock; }
__host__ __device__ inline size_t mx_groups(size_t cols) { return (cols + kMxGroup - 1) / kMxGroup; }
__host__ __device__ inline size_t mx_bands(size_t rows) { return (rows + kMxBand - 1) / kMxBand; }

namespace {

// Where the four scales of group g of row r begin.
__device__ __forceinline__ size_t mx_scale_at(uint32_t r, uint32_t g, uint32_t groups)
{
    return ((size_t)(r >> 7) * groups + g) * kMxTileBytes + (r & 31u) * 16u + ((r >> 5) & 3u) * 4u;
}

__device__ __forceinline__ float mx_float(float v) { return v; }
__device__ __forceinline__ float mx_float(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float mx_float(__half v) { return __half2float(v); }
template <class T> __device__ __forceinline__ T mx_round(float v);
template <> __device__ __forceinline__ float mx_round<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 mx_round<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half mx_round<__half>(float v) { return __float2half_rn(v); }

// 4 or 8 values of a vector load, in binary32.
template <class T> struct MxPack { T v[16 / sizeof(T)]; };

// The biased exponent of a block whose largest magnitude has the bits `top`: floor(log2) is the exponent field, and a field
// below 2 (e below -127, subnormal numbers and zero among them) ends at 0.  255 where `top` is no finite number.
__device__ __forceinline__ uint32_t mx_exponent(uint32_t top)
{
    const uint32_t field = top >> 23;
    return field == 255u ? 255u : field < 2u ? 0u : field - 2u;
}
// 2^-e, exact: 254 - s is a normal number's field for every finite s <= 252.  0 for a block of NaN, whose codes are zeros.
__device__ __forceinline__ float mx_inverse(uint32_t s) { return __uint_as_float(s == 255u ? 0u : (254u - s) << 23); }
// 2^e; e = -127 is a subnormal number
__device__ __forceinline__ float mx_scale(uint32_t s) { return __uint_as_float(s == 0u ? 0x00400000u : s == 255u ? 0x7FC00000u : s << 23); }

// Eight values of a block, already times 2^-e, as eight codes (the conversion rounds to nearest, ties to even, and ends at 6).
__device__ __forceinline__ uint32_t mx_encode8(const float (&v)[8])
{
    uint32_t w;
    asm("{\n\t.reg .b8 a, b, c, d;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
        "mov.b32 %0, {a, b, c, d};\n\t}"
        : "=r"(w)
        : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
    return w;
}
// Two elements of a 16-bit type in a word, or of binary32 in two.
template <class T> struct MxTwo { uint32_t w; };
template <> struct MxTwo<float> { float a, b; };

// Largest magnitudes so far of the two places, as bits: a NaN stays, above infinity.
template <class T> struct MxTop { uint32_t w = 0; };
template <> struct MxTop<float> { float a = 0.0f, b = 0.0f; };
__device__ __forceinline__ void mx_top(MxTop<__nv_bfloat16>& top, const MxTwo<__nv_bfloat16>& v)
{
    asm("{\n\t.reg .b32 a;\n\tabs.bf16x2 a, %1;\n\tmax.NaN.bf16x2 %0, %0, a;\n\t}" : "+r"(top.w) : "r"(v.w));
}
__device__ __forceinline__ void mx_top(MxTop<__half>& top, const MxTwo<__half>& v)
{
    asm("{\n\t.reg .b32 a;\n\tabs.f16x2 a, %1;\n\tmax.NaN.f16x2 %0, %0, a;\n\t}" : "+r"(top.w) : "r"(v.w));
}
__device__ __forceinline__ void mx_top(MxTop<float>& top, const MxTwo<float>& v)
{
    asm("max.NaN.f32 %0, %0, %1;" : "+f"(top.a) : "f"(fabsf(v.a)));
    asm("max.NaN.f32 %0, %0, %1;" : "+f"(top.b) : "f"(fabsf(v.b)));
}
// The bits of a magnitude in binary32.
template <class T> __device__ __forceinline__ uint32_t mx_bits(uint32_t half);
template <> __device__ __forceinline__ uint32_t mx_bits<__nv_bfloat16>(uint32_t half) { return half << 16; }
template <> __device__ __forceinline__ uint32_t mx_bits<__half>(uint32_t half) { return __float_as_uint(__half2float(__ushort_as_half((unsigned short)half))); }
template <class T> __device__ __forceinline__ uint32_t mx_first(const MxTop<T>& top) { return mx_bits<T>(top.w & 0xFFFFu); }
template <class T> __device__ __forceinline__ uint32_t mx_second(const MxTop<T>& top) { return mx_bits<T>(top.w >> 16); }
__device__ __forceinline__ uint32_t mx_first(const MxTop<float>& top) { return __float_as_uint(top.a); }
__device__ __forceinline__ uint32_t mx_second(const MxTop<float>& top) { return __float_as_uint(top.b); }

// Both elements times their powers of two, as binary32 (what falls below its range is far below the smallest code's half).  bfloat16 has binary32's exponents, so
// its powers are bfloat16 too and one instruction converts and multiplies (8192 x 8192 along rows 25.8 us; multiplied in pairs and then taken apart 27.2 us).
template <class T>
__device__ __forceinline__ void mx_scaled(const MxTwo<T>& v, float first, float second, uint32_t, float& a, float& b)
{
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&v.w));
    a = f.x * first;
    b = f.y * second;
}
__device__ __forceinline__ void mx_scaled(const MxTwo<float>& v, float first, float second, uint32_t, float& a, float& b)
{
    a = v.a * first;
    b = v.b * second;
}
__device__ __forceinline__ void mx_scaled(const MxTwo<__nv_bfloat16>& v, float, float, uint32_t both, float& a, float& b)
{
    asm("{\n\t.reg .b16 l, h, s, t;\n\tmov.b32 {l, h}, %2;\n\tmov.b32 {s, t}, %3;\n\tfma.rn.f32.bf16 %0, l, s, %4;\n\tfma.rn.f32.bf16 %1, h, t, %4;\n\t}"
        : "=f"(a), "=f"(b) : "r"(v.w), "r"(both), "f"(-0.0f));
}
// 2^-e of two places as a pair of bfloat16.
__device__ __forceinline__ uint32_t mx_pair(float first, float second) { return __float_as_uint(first) >> 16 | (__float_as_uint(second) & 0xFFFF0000u); }

// Eight neighbouring elements of a row; what lies behind `cols` counts as zero.  The row is not __restrict__ (see zccl_mx4.cu).
template <class T, bool VEC>
__device__ __forceinline__ void load8(const T* row, uint32_t at, uint32_t cols, MxTwo<T> (&v)[4])
{
    if (VEC && at + 8 <= cols) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) reinterpret_cast<uint4*>(v)[i] = __ldcs(reinterpret_cast<const uint4*>(row + at) + i);
    } else {
        T e[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) e[i] = at + i < cols ? row[at + i] : mx_round<T>(0.0f);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = *reinterpret_cast<const MxTwo<T>*>(&e[2 * i]);
    }
}

// One code (four bits): magnitudes 0 ... 3 are halves of their index, 4 ... 7 have two mantissas to a binade.
__device__ __forceinline__ float mx_decode1(uint32_t code)
{
    const uint32_t m = code & 7u;
    // E2M1 moved to binary32's exponent and mantissa is the value times 2^-126, its subnormal number one of binary32's
    return __uint_as_float(m << 22 | (code & 8u) << 28) * 0x1p126f;
}
// Eight codes as the numbers that E2M1 gives them (without the block's scale).
__device__ __forceinline__ void mx_decode8(uint32_t w, float (&v)[8])
{
    uint32_t h[4];
    asm("{\n\t.reg .b8 a, b, c, d;\n\t"
        "mov.b32 {a, b, c, d}, %4;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, a;\n\t"
        "cvt.rn.f16x2.e2m1x2 %1, b;\n\t"
        "cvt.rn.f16x2.e2m1x2 %2, c;\n\t"
        "cvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3]) : "r"(w));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h[i]));
        v[2 * i] = f.x;
        v[2 * i + 1] = f.y;
    }
}

// Four lanes' block, eight elements to a lane: the lane's codes, and the block's biased exponent.
template <class T>
__device__ __forceinline__ uint32_t quantize_block(const MxTwo<T> (&v)[4], uint32_t& s)
{
    MxTop<T> two;
#pragma unroll
    for (int i = 0; i < 4; ++i) mx_top(two, v[i]);
    uint32_t top = max(mx_first(two), mx_second(two));
    top = max(top, __shfl_xor_sync(kFull, top, 1));
    top = max(top, __shfl_xor_sync(kFull, top, 2));
    s = mx_exponent(top);
    const float inverse = mx_inverse(s);
    const uint32_t both = mx_pair(inverse, inverse);
    float f[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) mx_scaled(v[i], inverse, inverse, both, f[2 * i], f[2 * i + 1]);
    return s == 255u ? 0u : mx_encode8(f);
}
// Sixteen lanes' run of 128 elements: the lane's codes, and in `four` the run's four biased exponents as a word (every lane's).
template <class T>
__device__ __forceinline__ uint32_t quantize_run(const MxTwo<T> (&v)[4], uint32_t sub, uint32_t& four)
{
    uint32_t s;
    const uint32_t w = quantize_block(v, s);
    four = s << (8 * (sub >> 2));
    four |= __shfl_xor_sync(kFull, four, 4);
    four |= __shfl_xor_sync(kFull, four, 8);
    return w;
}

}  // namespace
}  // namespace zccl
