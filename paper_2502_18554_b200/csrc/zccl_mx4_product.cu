// Product of two operands in microscaled 4-bit floating point, Y = A B^T, on the tensor cores' block-scaled instruction: codes and
// scales go from memory to shared memory to the tensor core as they are, sums are kept in binary32.
#include "../../include/zccl.h"
#include "zccl_mx4.cuh"
#include "zccl_tcgen05.cuh"

#include <cuda.h>

#include <algorithm>
#include <mutex>

namespace zccl {
namespace {

constexpr int kRows = 128;                    // rows of a tile: the tensor core's lanes
constexpr int kDepth = 256;                   // elements along the contraction per stage: 128 bytes of codes, a row of the swizzle
constexpr int kRowBytes = kDepth / 2;         // an instruction takes 64 elements, 32 bytes of them
constexpr int kProductThreads = 192;          // one warp loads, one issues, four read the sums out
constexpr uint32_t kWaitLimit = 1u << 22;     // polls of a barrier before giving up
constexpr uint32_t kStuck = 1u;               // status: a wait ran out

__device__ uint32_t g_product_status;

struct Product {
    const unsigned char *r_scales, *c_scales;
    void* y;
    unsigned long long pitch;
    uint32_t rows, cols;                      // of the output as this kernel sees it: rows go along the lanes
    uint32_t depth_blocks;                    // blocks of 32 along the contraction
    uint32_t row_tiles, col_tiles;
    int type;
    int across;                               // 1: y is stored the other way round, its rows along the kernel's columns
};

template <int BN>
struct ProductShape {
    static constexpr int kBands = BN > 128 ? 2 : 1;           // tiles of scales that a tile's columns lie in
    static constexpr int kRowCodes = kRows * kRowBytes, kColCodes = BN * kRowBytes;
    static constexpr int kColAt = kRowCodes, kRowScaleAt = kColAt + kColCodes, kColScaleAt = kRowScaleAt + 2 * kMxTileBytes;
    static constexpr int kStage = kColScaleAt + 2 * kMxTileBytes * kBands;
    static constexpr int kScaleColumns = 8 + 8 * kBands;      // of tensor memory, for one stage
};

struct Control {
    unsigned long long *full, *empty, *done, *free;
};

__device__ __forceinline__ bool wait_for(unsigned long long* bar, uint32_t parity)
{
    for (uint32_t i = 0; i < kWaitLimit; ++i)
        if (mbar_try_wait(bar, parity)) return true;
    atomicOr(&g_product_status, kStuck);
    return false;
}

// How much of the contraction is left from depth tile k on, in groups of 128 (0, 1 or 2) and instructions (up to 4).
__device__ __forceinline__ uint32_t groups_at(uint32_t k, uint32_t blocks) { return min(2u, (blocks - k * 8 + 3) / 4); }
__device__ __forceinline__ uint32_t steps_at(uint32_t k, uint32_t blocks) { return min(4u, (blocks - k * 8 + 1) / 2); }

template <class T>
__device__ __forceinline__ void store_row(T* y, uint32_t count, const uint32_t (&v)[32])
{
    if (count == 32 && ((uintptr_t)y & 15u) == 0) {
        constexpr int kPer = 16 / sizeof(T);
#pragma unroll
        for (int i = 0; i < 32 / kPer; ++i) {
            MxPack<T> p;
#pragma unroll
            for (int j = 0; j < kPer; ++j) p.v[j] = mx_round<T>(__uint_as_float(v[kPer * i + j]));
            reinterpret_cast<uint4*>(y)[i] = *reinterpret_cast<const uint4*>(&p);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 32; ++i)
            if (i < (int)count) y[i] = mx_round<T>(__uint_as_float(v[i]));
    }
}
// Up to 32 sums of a lane, columns c ... of row r.
template <class T>
__device__ __forceinline__ void store(const Product& k, uint32_t r, uint32_t c, uint32_t width, const uint32_t (&v)[32])
{
    if (r >= k.rows || c >= k.cols) return;
    const uint32_t count = min(width, k.cols - c);
    T* y = (T*)k.y;
    if (k.across) {
#pragma unroll
        for (int i = 0; i < 32; ++i)
            if (i < (int)count) y[(size_t)(c + i) * k.pitch + r] = mx_round<T>(__uint_as_float(v[i]));
    } else store_row(y + (size_t)r * k.pitch + c, count, v);
}
__device__ __forceinline__ void store_any(const Product& k, uint32_t r, uint32_t c, uint32_t width, const uint32_t (&v)[32])
{
    if (k.type == ZCCL_BF16) store<__nv_bfloat16>(k, r, c, width, v);
    else if (k.type == ZCCL_F16) store<__half>(k, r, c, width, v);
    else store<float>(k, r, c, width, v);
}

// Tile t of the output: eight tiles of rows share a walk along the columns, so what is in flight reads few rows and columns.
__device__ __forceinline__ void tile_of(const Product& k, uint32_t t, uint32_t& row_tile, uint32_t& col_tile)
{
    constexpr uint32_t kBand = 8;
    const uint32_t per = kBand * k.col_tiles, band = t / per, in = t - band * per;
    const uint32_t high = min(kBand, k.row_tiles - band * kBand);
    col_tile = in / high;
    row_tile = band * kBand + (in - col_tile * high);
}

// One CTA (SPLIT: one cluster) per tile of 128 x BN at a time.  SPLIT: the CTAs of a cluster take neighbouring pieces of the contraction
// of one tile; their sums are added in the order of the pieces out of each other's shared memory, each CTA some of the columns.
template <int BN, int STAGES, bool SPLIT>
__global__ void __launch_bounds__(kProductThreads, 1) mx4_product_kernel(const __grid_constant__ CUtensorMap r_map, const __grid_constant__ CUtensorMap c_map, const __grid_constant__ Product k)
{
    using S = ProductShape<BN>;
    constexpr int kSums = SPLIT ? 1 : 2;
    constexpr uint32_t kSumColumns = BN < 32 ? 32 : BN;
    constexpr uint32_t kNeed = kSums * kSumColumns + 2 * S::kScaleColumns;
    constexpr uint32_t kColumns = kNeed <= 64 ? 64 : kNeed <= 128 ? 128 : kNeed <= 256 ? 256 : 512;
    static_assert(kNeed <= 512, "tensor memory");
    extern __shared__ unsigned char raw[];
    __shared__ unsigned long long full[STAGES], empty[STAGES], done[2], free_[2], drained;
    __shared__ uint32_t tmem_at;
    unsigned char* const tiles = raw + (1024 - (smem_u32(raw) & 1023u)) % 1024;
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31u;

    if (warp == 0 && lane == 0) {
        prefetch_map(&r_map);
        prefetch_map(&c_map);
        for (int i = 0; i < STAGES; ++i) {
            mbar_init(&full[i], 1);
            mbar_init(&empty[i], 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&done[i], 1);
            mbar_init(&free_[i], 4);
        }
        mbar_init(&drained, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) tmem_alloc(&tmem_at, kColumns);
    tcgen05_fence_before();
    __syncthreads();
    tcgen05_fence_after();
    const uint32_t tmem = tmem_at;
    pdl_enter();

    const uint32_t depth_tiles = (k.depth_blocks + 7) / 8, total = k.row_tiles * k.col_tiles;
    uint32_t first_tile = blockIdx.x, stride = gridDim.x, k_begin = 0, k_end = depth_tiles, parts = 1, part = 0;
    if (SPLIT) {
        asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(parts));
        part = cluster_rank();
        first_tile = blockIdx.x / parts;
        stride = total;                        // one tile
        k_begin = (uint32_t)((unsigned long long)depth_tiles * part / parts);
        k_end = (uint32_t)((unsigned long long)depth_tiles * (part + 1) / parts);
    }

    if (warp == 0) {
        if (lane == 0) {
            const uint32_t groups = (k.depth_blocks + 3) / 4, col_bands = (k.cols + kMxBand - 1) / kMxBand;
            uint32_t n = 0;
            bool ok = true;
            for (uint32_t t = first_tile; t < total && ok; t += stride) {
                uint32_t rt, ct;
                tile_of(k, t, rt, ct);
                const uint32_t c0 = ct * BN, band = c0 / kMxBand, bands = min((uint32_t)S::kBands, col_bands - band);
                for (uint32_t d = k_begin; d < k_end; ++d, ++n) {
                    const uint32_t s = n % STAGES;
                    if (n >= STAGES && !(ok = wait_for(&empty[s], (n / STAGES - 1) & 1))) break;
                    unsigned char* const at = tiles + s * S::kStage;
                    const uint32_t scale_bytes = groups_at(d, k.depth_blocks) * kMxTileBytes;
                    mbar_expect_tx(&full[s], S::kRowCodes + S::kColCodes + scale_bytes * (1 + bands));
                    tile_load(at, &r_map, (int)(d * kRowBytes), (int)(rt * kRows), &full[s]);
                    tile_load(at + S::kColAt, &c_map, (int)(d * kRowBytes), (int)c0, &full[s]);
                    bytes_load(at + S::kRowScaleAt, k.r_scales + ((size_t)rt * groups + 2 * d) * kMxTileBytes, scale_bytes, &full[s]);
                    for (uint32_t b = 0; b < bands; ++b)
                        bytes_load(at + S::kColScaleAt + b * 2 * kMxTileBytes, k.c_scales + ((size_t)(band + b) * groups + 2 * d) * kMxTileBytes, scale_bytes, &full[s]);
                }
            }
            // what has been asked for lands before the memory is given up, whether it is used or not
            for (uint32_t i = n < STAGES ? 0 : n - STAGES; i < n; ++i) wait_for(&full[i % STAGES], (i / STAGES) & 1);
        }
    } else if (warp == 1) {
        if (elect_one()) {
            uint32_t n = 0, i = 0;
            bool ok = true;
            for (uint32_t t = first_tile; t < total && ok; t += stride, ++i) {
                uint32_t rt, ct;
                tile_of(k, t, rt, ct);
                const uint32_t sums = tmem + (SPLIT ? 0 : (i & 1) * kSumColumns);
                const uint32_t shift = (ct * BN % kMxBand) / 32;      // where the tile's columns begin in their first tile of scales
                if (i >= kSums) {
                    if (!(ok = wait_for(&free_[i & 1], (i / 2 - 1) & 1))) break;
                    tcgen05_fence_after();
                }
                for (uint32_t d = k_begin; d < k_end; ++d, ++n) {
                    const uint32_t s = n % STAGES;
                    if (!(ok = wait_for(&full[s], (n / STAGES) & 1))) break;
                    tcgen05_fence_after();
                    const uint32_t at = smem_u32(tiles) + s * S::kStage;
                    const uint32_t r_scale = tmem + kSums * kSumColumns + (n & 1) * S::kScaleColumns, c_scale = r_scale + 8;
                    for (uint32_t g = 0; g < groups_at(d, k.depth_blocks); ++g) {
                        tcgen05_copy_scales(r_scale + 4 * g, scales_descriptor(at + S::kRowScaleAt + g * kMxTileBytes));
                        for (int b = 0; b < S::kBands; ++b)
                            tcgen05_copy_scales(c_scale + 4 * (g * S::kBands + b), scales_descriptor(at + S::kColScaleAt + (b * 2 + g) * kMxTileBytes));
                    }
                    const unsigned long long r_codes = operand_descriptor(at), c_codes = operand_descriptor(at + S::kColAt);
                    const uint32_t steps = steps_at(d, k.depth_blocks);
                    for (uint32_t j = 0; j < steps; ++j)
                        tcgen05_mma_mx4(sums, r_codes + 2 * j, c_codes + 2 * j, mx4_instruction(kRows, BN, (j & 1) * 2), r_scale + 4 * (j / 2),
                                        c_scale + 4 * S::kBands * (j / 2) + shift, d > k_begin || j > 0);
                    tcgen05_commit(&empty[s]);
                }
                tcgen05_commit(&done[i & 1]);
            }
            tcgen05_commit(&drained);
            wait_for(&drained, 0);
        }
    } else {
        const uint32_t quarter = warp & 3u, row = quarter * 32 + lane;
        uint32_t i = 0;
        for (uint32_t t = first_tile; t < total; t += stride, ++i) {
            uint32_t rt, ct;
            tile_of(k, t, rt, ct);
            const uint32_t sums = tmem + (SPLIT ? 0 : (i & 1) * kSumColumns) + (quarter * 32 << 16);
            if (!wait_for(&done[i & 1], (i / 2) & 1)) break;
            tcgen05_fence_after();
            constexpr int kWide = BN < 32 ? BN : 32;
#pragma unroll 1
            for (int c = 0; c < BN; c += kWide) {
                uint32_t v[32];
                if (kWide == 32) tcgen05_load32(sums + c, v);
                else tcgen05_load16(sums + c, v);
                tcgen05_wait_loads();
                if (SPLIT) {
#pragma unroll
                    for (int j = 0; j < kWide; ++j) reinterpret_cast<float*>(tiles)[(c + j) * kRows + row] = __uint_as_float(v[j]);
                } else store_any(k, rt * kRows + row, ct * BN + c, kWide, v);
            }
            tcgen05_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&free_[i & 1]);
        }
    }
    if (SPLIT) {
        __syncwarp();
        cluster_sync();
        if (warp >= 2) {
            uint32_t rt, ct;
            tile_of(k, first_tile, rt, ct);
            const uint32_t row = threadIdx.x - 64;
            for (uint32_t c = part; c < (uint32_t)BN && ct * BN + c < k.cols; c += parts) {
                float sum = 0.0f;
                for (uint32_t p = 0; p < parts; ++p) sum += peer_load(smem_u32(tiles) + (c * kRows + row) * 4, p);
                const uint32_t r = rt * kRows + row, cc = ct * BN + c;
                if (r < k.rows) {
                    const size_t to = k.across ? (size_t)cc * k.pitch + r : (size_t)r * k.pitch + cc;
                    if (k.type == ZCCL_BF16) ((__nv_bfloat16*)k.y)[to] = mx_round<__nv_bfloat16>(sum);
                    else if (k.type == ZCCL_F16) ((__half*)k.y)[to] = mx_round<__half>(sum);
                    else ((float*)k.y)[to] = sum;
                }
            }
        }
        __syncwarp();
        cluster_sync();                        // nobody leaves while its sums are still read
    }
    tcgen05_fence_before();
    __syncthreads();
    __syncwarp();
    if (warp == 1) tmem_free(tmem, kColumns);
}

using EncodeFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*, const cuuint32_t*,
                              CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
constexpr int kMaxDevices = 64;
std::mutex g_product_mu;
EncodeFn g_product_encode = nullptr;
struct ProductDevice {
    bool ready = false;
    int sms = 0;
};
ProductDevice g_product_dev[kMaxDevices];

template <int BN, int STAGES, bool SPLIT>
constexpr size_t product_smem() { return (size_t)ProductShape<BN>::kStage * STAGES + 1024; }
template <int BN, int STAGES, bool SPLIT>
cudaError_t product_attr()
{
    return cudaFuncSetAttribute(mx4_product_kernel<BN, STAGES, SPLIT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)product_smem<BN, STAGES, SPLIT>());
}

cudaError_t product_device(const ProductDevice** out)
{
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= kMaxDevices) return cudaErrorInvalidDevice;
    std::lock_guard<std::mutex> lock(g_product_mu);
    if (!g_product_encode) {
        void* fn = nullptr;
        cudaDriverEntryPointQueryResult q;
        e = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &q);
        if (e != cudaSuccess) return e;
        if (q != cudaDriverEntryPointSuccess || !fn) return cudaErrorNotSupported;
        g_product_encode = reinterpret_cast<EncodeFn>(fn);
    }
    ProductDevice& d = g_product_dev[dev];
    if (!d.ready) {
        e = cudaDeviceGetAttribute(&d.sms, cudaDevAttrMultiProcessorCount, dev);
        if (e == cudaSuccess) e = product_attr<192, 5, false>();
        if (e == cudaSuccess) e = product_attr<128, 6, false>();
        if (e == cudaSuccess) e = product_attr<128, 3, true>();
        if (e == cudaSuccess) e = product_attr<64, 4, true>();
        if (e == cudaSuccess) e = product_attr<32, 4, true>();
        if (e == cudaSuccess) e = product_attr<16, 4, true>();
        if (e != cudaSuccess) return e;
        d.ready = true;
    }
    *out = &d;
    return cudaSuccess;
}

bool operand_map(CUtensorMap* map, const void* codes, size_t rows, size_t blocks, int box_rows)
{
    const cuuint64_t size[2] = {blocks * 16, rows}, stride[1] = {blocks * 16};
    const cuuint32_t box[2] = {kRowBytes, (cuuint32_t)box_rows}, step[2] = {1, 1};
    return g_product_encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(codes), size, stride, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

struct Sides {
    const void *r_codes, *c_codes;
    size_t rows, cols;
};

template <int BN, int STAGES, bool SPLIT>
int launch_product(const Sides& sides, Product k, unsigned parts, unsigned most_ctas, cudaStream_t st)
{
    CUtensorMap r_map, c_map;
    if (!operand_map(&r_map, sides.r_codes, sides.rows, k.depth_blocks, kRows) || !operand_map(&c_map, sides.c_codes, sides.cols, k.depth_blocks, BN)) return ZCCL_E_CUDA;
    k.row_tiles = (uint32_t)((sides.rows + kRows - 1) / kRows);
    k.col_tiles = (uint32_t)((sides.cols + BN - 1) / BN);
    const unsigned long long total = (unsigned long long)k.row_tiles * k.col_tiles;
    if (total * parts > 0x7FFFFFFFu) return ZCCL_E_ARG;
    const unsigned ctas = SPLIT ? (unsigned)total * parts : (unsigned)std::min<unsigned long long>(total, most_ctas);
    const cudaError_t e = launch_cluster(parts, mx4_product_kernel<BN, STAGES, SPLIT>, dim3(ctas), dim3(kProductThreads), product_smem<BN, STAGES, SPLIT>(), st, r_map, c_map, k);
    if (e == cudaSuccess) count_launches(1);
    return e == cudaSuccess ? ZCCL_OK : ZCCL_E_CUDA;
}

bool aligned16(const void* p) { return p && ((uintptr_t)p & 15u) == 0; }

}  // namespace
}  // namespace zccl

using namespace zccl;

extern "C" {

int zccl_mx4_matmul(const void* a_codes, const void* a_scales, size_t m, const void* b_codes, const void* b_scales, size_t n, size_t k, void* y, int type, size_t pitch, void* stream)
{
    if (type < ZCCL_F32 || type > ZCCL_F16) return ZCCL_E_ARG;
    const size_t element = type == ZCCL_F32 ? 4 : 2;
    constexpr size_t kMost = 0x7FFFFF00u;
    if (m == 0 || n == 0) return ZCCL_OK;
    if (m > kMost || n > kMost || k > kMost || pitch < n || !y || (uintptr_t)y % element) return ZCCL_E_ARG;
    cudaStream_t st = (cudaStream_t)stream;
    if (k == 0) return cudaMemset2DAsync(y, pitch * element, 0, n * element, m, st) == cudaSuccess ? ZCCL_OK : ZCCL_E_CUDA;
    if (!aligned16(a_codes) || !aligned16(a_scales) || !aligned16(b_codes) || !aligned16(b_scales)) return ZCCL_E_ARG;
    const ProductDevice* dev;
    if (product_device(&dev) != cudaSuccess) return ZCCL_E_CUDA;
    Product p{};
    p.y = y;
    p.pitch = pitch;
    p.type = type;
    p.depth_blocks = (uint32_t)mx_blocks(k);
    // the longer side goes along the lanes
    const bool across = m < n && m <= 128;
    Sides sides{a_codes, b_codes, m, n};
    p.r_scales = (const unsigned char*)a_scales;
    p.c_scales = (const unsigned char*)b_scales;
    if (across) {
        std::swap(sides.r_codes, sides.c_codes);
        std::swap(sides.rows, sides.cols);
        std::swap(p.r_scales, p.c_scales);
    }
    p.across = across;
    p.rows = (uint32_t)sides.rows;
    p.cols = (uint32_t)sides.cols;
    const unsigned sms = (unsigned)dev->sms;
    const uint32_t depth_tiles = (p.depth_blocks + 7) / 8;
    const size_t row_tiles = (sides.rows + kRows - 1) / kRows;
    if (sides.cols <= 128) {
        unsigned parts = 1;
        while (parts < 8 && parts * 2 <= depth_tiles && row_tiles * parts * 2 <= 2 * sms) parts *= 2;
        if (sides.cols <= 16) return launch_product<16, 4, true>(sides, p, parts, 0, st);
        if (sides.cols <= 32) return launch_product<32, 4, true>(sides, p, parts, 0, st);
        if (sides.cols <= 64) return launch_product<64, 4, true>(sides, p, parts, 0, st);
        return launch_product<128, 3, true>(sides, p, parts, 0, st);
    }
    const size_t tiles = row_tiles * ((sides.cols + 127) / 128);
    if (tiles * 2 <= sms) {
        unsigned parts = 1;
        while (parts < 8 && parts * 2 <= depth_tiles && tiles * parts * 2 <= 2 * sms) parts *= 2;
        if (parts > 1) return launch_product<128, 3, true>(sides, p, parts, 0, st);
    }
    if (row_tiles * ((sides.cols + 191) / 192) >= sms) return launch_product<192, 5, false>(sides, p, 1, sms, st);
    return launch_product<128, 6, false>(sides, p, 1, sms, st);
}

int zccl_mx4_status(void* stream)
{
    cudaStream_t st = (cudaStream_t)stream;
    uint32_t bits = 0;
    const uint32_t zero = 0;
    if (cudaMemcpyFromSymbolAsync(&bits, g_product_status, sizeof bits, 0, cudaMemcpyDeviceToHost, st) != cudaSuccess) return ZCCL_E_CUDA;
    if (cudaStreamSynchronize(st) != cudaSuccess) return ZCCL_E_CUDA;
    if (!bits) return ZCCL_OK;
    if (cudaMemcpyToSymbolAsync(g_product_status, &zero, sizeof zero, 0, cudaMemcpyHostToDevice, st) != cudaSuccess || cudaStreamSynchronize(st) != cudaSuccess) return ZCCL_E_CUDA;
    return ZCCL_E_TIMEOUT;
}

}  // extern "C"
