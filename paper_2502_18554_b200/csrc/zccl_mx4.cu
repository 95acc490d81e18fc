// Quantisation to microscaled 4-bit floating point, along the rows or along the columns, and back.
#include "../../include/zccl.h"
#include "zccl_mx4.cuh"

#include <algorithm>

namespace zccl {
namespace {

constexpr int kMxThreads = 256;

// Eight neighbouring elements of a row, in binary32; what lies behind `cols` counts as zero.
template <class T, bool VEC>
__device__ __forceinline__ void load8(const T* __restrict__ row, uint32_t at, uint32_t cols, float (&v)[8])
{
    constexpr int kPer = 16 / sizeof(T);
    if (VEC && at + 8 <= cols) {
#pragma unroll
        for (int i = 0; i < 8 / kPer; ++i) {
            const uint4 raw = __ldcs(reinterpret_cast<const uint4*>(row + at) + i);
            const MxPack<T> p = *reinterpret_cast<const MxPack<T>*>(&raw);
#pragma unroll
            for (int j = 0; j < kPer; ++j) v[kPer * i + j] = mx_float(p.v[j]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = at + i < cols ? mx_float(row[at + i]) : 0.0f;
    }
}

__device__ __forceinline__ uint32_t top_of(const float (&v)[8])
{
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(v[i]) & 0x7FFFFFFFu);
    return top;
}

// Rows: 16 lanes take a group of 128 neighbouring elements (four blocks, one word of scales), a lane eight of them, so
// loads are 16 bytes a lane and codes leave as whole lines.  Groups of the rows that fill the last band up, and blocks
// behind the last, are quantised as zeros: only their scales are written.
template <class T, bool VEC>
__global__ void __launch_bounds__(kMxThreads) mx_quantize_rows_kernel(const T* __restrict__ x, uint32_t rows, uint32_t cols, size_t pitch,
                                                                       uint32_t blocks, uint32_t groups, uint32_t total, uint32_t step_row, uint32_t step_group,
                                                                       uint32_t* __restrict__ codes, unsigned char* __restrict__ scales)
{
    pdl_enter();
    const uint32_t sub = threadIdx.x & 15u;
    uint32_t u = blockIdx.x * (kMxThreads / 16) + (threadIdx.x >> 4);
    uint32_t r = u / groups, g = u - r * groups;
    const uint32_t stride = gridDim.x * (kMxThreads / 16);
    // whole warps go round together: the last round's idle half takes part in the exchanges with zeros
    for (uint32_t first = u & ~1u; first < total; first += stride, u += stride) {
        float v[8];
        const uint32_t at = g * kMxGroup + sub * 8;
        if (u < total && r < rows && at < cols) load8<T, VEC>(x + (size_t)r * pitch, at, cols, v);
        else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = 0.0f;
        }
        uint32_t top = top_of(v);
        top = max(top, __shfl_xor_sync(kFull, top, 1));
        top = max(top, __shfl_xor_sync(kFull, top, 2));
        const uint32_t s = mx_exponent(top);
        const uint32_t w = s == 255u ? 0u : mx_encode8(v, mx_inverse(s));
        uint32_t four = s << (8 * (sub >> 2));
        four |= __shfl_xor_sync(kFull, four, 4);
        four |= __shfl_xor_sync(kFull, four, 8);
        if (u < total) {
            if (r < rows && (at >> 5) < blocks) codes[((size_t)r * blocks + (at >> 5)) * 4 + (sub & 3u)] = w;
            if (sub == 0) *reinterpret_cast<uint32_t*>(scales + mx_scale_at(r, g, groups)) = four;
        }
        r += step_row;
        g += step_group;
        if (g >= groups) { g -= groups; ++r; }
    }
}

// Columns: the form of the transpose.  A warp takes 32 rows x 64 columns (a lane two columns, so a row's load is one line
// of 16-bit elements), a CTA the four blocks of a word of scales.  A lane then holds whole blocks: no exchange, and a
// block's codes leave as 16 bytes; the four warps' fill a sector pair of the same row of the output.
template <class T, bool VEC>
__global__ void __launch_bounds__(128) mx_quantize_columns_kernel(const T* __restrict__ x, uint32_t rows, uint32_t cols, size_t pitch, uint32_t blocks,
                                                                   uint32_t groups, uint32_t across, uint4* __restrict__ codes, unsigned char* __restrict__ scales)
{
    pdl_enter();
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31u;
    const uint32_t g = blockIdx.x / across;
    const uint32_t c = (blockIdx.x - g * across) * 64 + lane * 2;
    const uint32_t b = g * 4 + warp;
    const uint32_t r0 = b * kMxBlock;
    __shared__ __align__(4) unsigned char sh[64][4];
    uint32_t top0 = 0, top1 = 0;
    T v0[kMxBlock], v1[kMxBlock];
    const bool any = c < cols, both = c + 1 < cols;
#pragma unroll
    for (int i = 0; i < kMxBlock; ++i) {
        const T* p = x + (size_t)(r0 + i) * pitch + c;
        v0[i] = v1[i] = mx_round<T>(0.0f);
        if (any && r0 + i < rows) {
            if (VEC && both) {
                struct alignas(2 * sizeof(T)) Two { T a, b; };
                const Two two = *reinterpret_cast<const Two*>(p);
                v0[i] = two.a;
                v1[i] = two.b;
            } else {
                v0[i] = p[0];
                if (both) v1[i] = p[1];
            }
        }
    }
#pragma unroll
    for (int i = 0; i < kMxBlock; ++i) {
        top0 = max(top0, __float_as_uint(mx_float(v0[i])) & 0x7FFFFFFFu);
        top1 = max(top1, __float_as_uint(mx_float(v1[i])) & 0x7FFFFFFFu);
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const uint32_t s = mx_exponent(j ? top1 : top0);
        const float inverse = mx_inverse(s);
        uint32_t w[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            float f[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = mx_float(j ? v1[8 * q + i] : v0[8 * q + i]);
            w[q] = s == 255u ? 0u : mx_encode8(f, inverse);
        }
        if (c + j < cols && b < blocks) codes[(size_t)(c + j) * blocks + b] = make_uint4(w[0], w[1], w[2], w[3]);
        sh[lane * 2 + j][warp] = (unsigned char)s;
    }
    __syncthreads();
    if (threadIdx.x < 64) {
        const uint32_t column = (blockIdx.x - g * across) * 64 + threadIdx.x;
        *reinterpret_cast<uint32_t*>(scales + mx_scale_at(column, g, groups)) = *reinterpret_cast<const uint32_t*>(sh[threadIdx.x]);
    }
}

template <class T, bool VEC>
__global__ void __launch_bounds__(kMxThreads) mx_dequantize_kernel(const uint32_t* __restrict__ codes, const unsigned char* __restrict__ scales, uint32_t rows,
                                                                    uint32_t cols, uint32_t blocks, uint32_t groups, uint32_t total, uint32_t step_row,
                                                                    uint32_t step_group, T* __restrict__ y, size_t pitch)
{
    pdl_enter();
    const uint32_t sub = threadIdx.x & 15u;
    uint32_t u = blockIdx.x * (kMxThreads / 16) + (threadIdx.x >> 4);
    uint32_t r = u / groups, g = u - r * groups;
    const uint32_t stride = gridDim.x * (kMxThreads / 16);
    for (; u < total; u += stride) {
        const uint32_t at = g * kMxGroup + sub * 8;
        if (at < cols) {
            const uint32_t w = __ldcs(codes + ((size_t)r * blocks + (at >> 5)) * 4 + (sub & 3u));
            const uint32_t s = scales[mx_scale_at(r, g, groups) + (sub >> 2)];
            float v[8];
            mx_decode8(w, mx_scale(s), v);
            T* out = y + (size_t)r * pitch + at;
            constexpr int kPer = 16 / sizeof(T);
            if (VEC && at + 8 <= cols) {
#pragma unroll
                for (int i = 0; i < 8 / kPer; ++i) {
                    MxPack<T> p;
#pragma unroll
                    for (int j = 0; j < kPer; ++j) p.v[j] = mx_round<T>(v[kPer * i + j]);
                    reinterpret_cast<uint4*>(out)[i] = *reinterpret_cast<const uint4*>(&p);
                }
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (at + i < cols) out[i] = mx_round<T>(v[i]);
            }
        }
        r += step_row;
        g += step_group;
        if (g >= groups) { g -= groups; ++r; }
    }
}

struct Rounds {
    unsigned ctas;
    uint32_t step_row, step_group;
};
// As many CTAs as there is work for, at most `most`, and how far (row, group) moves from round to round.
Rounds rounds_of(size_t total, uint32_t groups, size_t most)
{
    const size_t per = kMxThreads / 16;
    const unsigned ctas = (unsigned)std::min((total + per - 1) / per, most);
    const uint32_t stride = ctas * (uint32_t)per;
    return {ctas, stride / groups, stride % groups};
}

template <class T>
int quantize(const T* x, size_t rows, size_t cols, size_t pitch, bool transpose, void* codes, void* scales, cudaStream_t st)
{
    const uintptr_t at = (uintptr_t)x;
    cudaError_t e;
    if (transpose) {
        const size_t blocks = mx_blocks(rows), groups = mx_groups(rows), across = mx_bands(cols) * 2;
        if (groups * across > kMxMaxGroups) return ZCCL_E_ARG;
        const bool vec = at % (2 * sizeof(T)) == 0 && pitch % 2 == 0;
        e = launch_k(vec ? mx_quantize_columns_kernel<T, true> : mx_quantize_columns_kernel<T, false>, dim3((unsigned)(groups * across)), dim3(128), 0, st,
                     x, (uint32_t)rows, (uint32_t)cols, pitch, (uint32_t)blocks, (uint32_t)groups, (uint32_t)across, (uint4*)codes, (unsigned char*)scales);
    } else {
        const size_t blocks = mx_blocks(cols), groups = mx_groups(cols), total = mx_bands(rows) * kMxBand * groups;
        if (total > kMxMaxGroups) return ZCCL_E_ARG;
        const bool vec = at % 16 == 0 && pitch * sizeof(T) % 16 == 0;
        const Rounds k = rounds_of(total, (uint32_t)groups, 1u << 16);
        e = launch_k(vec ? mx_quantize_rows_kernel<T, true> : mx_quantize_rows_kernel<T, false>, dim3(k.ctas), dim3(kMxThreads), 0, st, x, (uint32_t)rows,
                     (uint32_t)cols, pitch, (uint32_t)blocks, (uint32_t)groups, (uint32_t)total, k.step_row, k.step_group, (uint32_t*)codes, (unsigned char*)scales);
    }
    if (e == cudaSuccess) count_launches(1);
    return e == cudaSuccess ? ZCCL_OK : ZCCL_E_CUDA;
}

template <class T>
int dequantize(const void* codes, const void* scales, size_t rows, size_t cols, T* y, size_t pitch, cudaStream_t st)
{
    const size_t blocks = mx_blocks(cols), groups = mx_groups(cols), total = rows * groups;
    if (total > kMxMaxGroups) return ZCCL_E_ARG;
    const bool vec = (uintptr_t)y % 16 == 0 && pitch * sizeof(T) % 16 == 0;
    const Rounds k = rounds_of(total, (uint32_t)groups, 1u << 16);
    const cudaError_t e = launch_k(vec ? mx_dequantize_kernel<T, true> : mx_dequantize_kernel<T, false>, dim3(k.ctas), dim3(kMxThreads), 0, st,
                                   (const uint32_t*)codes, (const unsigned char*)scales, (uint32_t)rows, (uint32_t)cols, (uint32_t)blocks, (uint32_t)groups,
                                   (uint32_t)total, k.step_row, k.step_group, y, pitch);
    if (e == cudaSuccess) count_launches(1);
    return e == cudaSuccess ? ZCCL_OK : ZCCL_E_CUDA;
}

constexpr size_t kMost = 0x7FFFFF00u;   // rows and columns are counted in 32 bits

bool aligned(const void* p, size_t to) { return p && (uintptr_t)p % to == 0; }
bool matrix_ok(const void* x, int type, size_t rows, size_t cols, size_t pitch)
{
    if (type < ZCCL_F32 || type > ZCCL_F16) return false;
    return aligned(x, type == ZCCL_F32 ? 4 : 2) && rows <= kMost && cols <= kMost && pitch >= cols;
}

}  // namespace
}  // namespace zccl

using namespace zccl;

extern "C" {

size_t zccl_mx4_code_bytes(size_t rows, size_t cols) { return rows * mx_blocks(cols) * 16; }

size_t zccl_mx4_scale_bytes(size_t rows, size_t cols) { return mx_bands(rows) * mx_groups(cols) * kMxTileBytes; }

int zccl_mx4_quantize(const void* x, int type, size_t rows, size_t cols, size_t pitch, int transpose, void* codes, void* scales, void* stream)
{
    if (rows == 0 || cols == 0) return type < ZCCL_F32 || type > ZCCL_F16 ? ZCCL_E_ARG : ZCCL_OK;
    if (!matrix_ok(x, type, rows, cols, pitch) || !aligned(codes, 16) || !aligned(scales, 16)) return ZCCL_E_ARG;
    cudaStream_t st = (cudaStream_t)stream;
    if (type == ZCCL_F32) return quantize((const float*)x, rows, cols, pitch, transpose != 0, codes, scales, st);
    if (type == ZCCL_BF16) return quantize((const __nv_bfloat16*)x, rows, cols, pitch, transpose != 0, codes, scales, st);
    return quantize((const __half*)x, rows, cols, pitch, transpose != 0, codes, scales, st);
}

int zccl_mx4_dequantize(const void* codes, const void* scales, size_t rows, size_t cols, void* y, int type, size_t pitch, void* stream)
{
    if (rows == 0 || cols == 0) return type < ZCCL_F32 || type > ZCCL_F16 ? ZCCL_E_ARG : ZCCL_OK;
    if (!matrix_ok(y, type, rows, cols, pitch) || !aligned(codes, 16) || !aligned(scales, 16)) return ZCCL_E_ARG;
    cudaStream_t st = (cudaStream_t)stream;
    if (type == ZCCL_F32) return dequantize(codes, scales, rows, cols, (float*)y, pitch, st);
    if (type == ZCCL_BF16) return dequantize(codes, scales, rows, cols, (__nv_bfloat16*)y, pitch, st);
    return dequantize(codes, scales, rows, cols, (__half*)y, pitch, st);
}

}  // extern "C"
