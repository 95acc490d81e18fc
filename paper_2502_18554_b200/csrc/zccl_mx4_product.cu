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
constexpr int kProductThreads = 192;          // one warp loads, one issues, four read the sums out (eight in pairs of CTAs)
constexpr uint32_t kWaitLimit = 1u << 19;     // polls of a barrier before giving up: two seconds (a poll that finds nothing takes 4 us; the deepest product that fits
                                              // the memory is through with a tile in half of one)
constexpr size_t kMostAcross = 64;            // rows of an output that is stored across
constexpr int kOutBytes = 64;                 // of a row of the output on its way through shared memory, and their pitch there
constexpr int kOutPitch = kOutBytes + 16;

struct Product {
    const unsigned char *r_scales, *c_scales;
    void* y;
    unsigned long long pitch;
    uint32_t rows, cols;                      // of the output as this kernel sees it: rows go along the lanes
    uint32_t depth_blocks;                    // blocks of 32 along the contraction
    uint32_t row_tiles, col_tiles;
    int type;
    int early;                                // the rows' operand is complete when the kernel starts (see mx4_split_kernel)
    int wide;                                 // every row of y begins on a 16-byte boundary
    int across;                               // 1: y is stored the other way round, its rows along the kernel's columns
    uint32_t* stuck;                          // the device's record of a wait that ran out, a word of the host's memory: the next call looks at it without a synchronisation
};

__device__ __noinline__ void record_stuck(uint32_t* stuck)
{
    *(volatile uint32_t*)stuck = 1u;
    __threadfence_system();
}
__device__ __forceinline__ bool wait_for(unsigned long long* bar, uint32_t parity, uint32_t* stuck)
{
    for (uint32_t i = 0; i < kWaitLimit; ++i)
        if (mbar_try_wait(bar, parity)) return true;
    record_stuck(stuck);
    return false;
}
__device__ __forceinline__ bool wait_for_cluster(unsigned long long* bar, uint32_t parity, uint32_t* stuck)
{
    for (uint32_t i = 0; i < kWaitLimit; ++i)
        if (mbar_try_wait_cluster(bar, parity)) return true;
    record_stuck(stuck);
    return false;
}
// The loading thread's last act: what it has asked for (n stages' worth, `loads`: at this CTA's barriers) lands, and what the tensor core still arrives for at
// `empty` has arrived, before the memory is given up, whether it is used or not.  `ok`: no wait has run out so far; after one the issuing thread may have given up.
template <int STAGES>
__device__ __forceinline__ void settle(unsigned long long* full, unsigned long long* empty, uint32_t n, bool loads, bool ok, uint32_t* stuck)
{
    for (uint32_t i = n < (uint32_t)STAGES ? 0 : n - STAGES; i < n; ++i) {
        if (loads) ok &= wait_for(&full[i % STAGES], (i / STAGES) & 1, stuck);
        ok = ok && wait_for(&empty[i % STAGES], (i / STAGES) & 1, stuck);
    }
}
__device__ __forceinline__ unsigned char* on_1024(unsigned char* raw) { return raw + (1024 - (smem_u32(raw) & 1023u)) % 1024; }

// How much of the contraction is left from depth tile k on, in groups of 128 (0, 1 or 2) and instructions (up to 4).
__device__ __forceinline__ uint32_t groups_at(uint32_t k, uint32_t blocks) { return min(2u, (blocks - k * 8 + 3) / 4); }
__device__ __forceinline__ uint32_t steps_at(uint32_t k, uint32_t blocks) { return min(4u, (blocks - k * 8 + 1) / 2); }

__device__ __forceinline__ void store_one(const Product& k, size_t to, float v)
{
    if (k.type == ZCCL_BF16) ((__nv_bfloat16*)k.y)[to] = mx_round<__nv_bfloat16>(v);
    else if (k.type == ZCCL_F16) ((__half*)k.y)[to] = mx_round<__half>(v);
    else ((float*)k.y)[to] = v;
}

// Up to four neighbouring elements of y, `left` of which are inside.
__device__ __forceinline__ void store_four(const Product& k, size_t to, uint32_t left, const float (&v)[4])
{
    if (k.wide && left >= 4) {
        if (k.type == ZCCL_F32) *reinterpret_cast<float4*>((float*)k.y + to) = make_float4(v[0], v[1], v[2], v[3]);
        else {
            ushort4 h;
            unsigned short* const e = &h.x;
#pragma unroll
            for (int i = 0; i < 4; ++i) e[i] = k.type == ZCCL_BF16 ? __bfloat16_as_ushort(mx_round<__nv_bfloat16>(v[i])) : __half_as_ushort(mx_round<__half>(v[i]));
            *reinterpret_cast<ushort4*>((unsigned short*)k.y + to) = h;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if ((uint32_t)i < left) store_one(k, to + i, v[i]);
    }
}

// Tile t of the output: `high` tiles of rows share a walk along the columns, so what is in flight reads few rows and columns.
__device__ __forceinline__ void tile_of(const Product& k, uint32_t t, uint32_t band_tiles, uint32_t& row_tile, uint32_t& col_tile)
{
    const uint32_t per = band_tiles * k.col_tiles, band = t / per, in = t - band * per;
    const uint32_t high = min(band_tiles, k.row_tiles - band * band_tiles);
    col_tile = in / high;
    row_tile = band * band_tiles + (in - col_tile * high);
}

// 64 bytes of each of the warp's 32 rows, from registers through shared memory: rows leave as whole sectors, or where they do not begin on 16 bytes as runs
// of neighbouring elements.  T is the type of the output, `v` has 64 / sizeof(T) columns of the lane's row from c on.
template <class T>
__device__ __forceinline__ void store_rows(const Product& k, unsigned char* out, uint32_t r, uint32_t c, const uint32_t* v)
{
    constexpr int kPer = 16 / sizeof(T), kWidth = kOutBytes / sizeof(T);
    const uint32_t lane = threadIdx.x & 31u;
    __syncwarp();
#pragma unroll
    for (int i = 0; i < kOutBytes / 16; ++i) {
        MxPack<T> p;
#pragma unroll
        for (int j = 0; j < kPer; ++j) p.v[j] = mx_round<T>(__uint_as_float(v[kPer * i + j]));
        *reinterpret_cast<uint4*>(out + lane * kOutPitch + 16 * i) = *reinterpret_cast<const uint4*>(&p);
    }
    __syncwarp();
    T* const y = (T*)k.y + (size_t)r * k.pitch + c;
    const uint32_t high = r < k.rows ? min(32u, k.rows - r) : 0u;
    if (k.wide && c + kWidth <= k.cols) {
#pragma unroll
        for (int i = 0; i < kOutBytes / 16; ++i) {
            const uint32_t row = 8 * i + (lane >> 2), piece = lane & 3u;
            if (row < high) reinterpret_cast<uint4*>(y + (size_t)row * k.pitch)[piece] = *reinterpret_cast<const uint4*>(out + row * kOutPitch + 16 * piece);
        }
    } else {
        constexpr uint32_t kAtOnce = 32 / kWidth;    // rows of a store
        const uint32_t at = lane % kWidth;
#pragma unroll 8
        for (uint32_t row = lane / kWidth; row < high; row += kAtOnce)
            if (c + at < k.cols) y[(size_t)row * k.pitch + at] = *reinterpret_cast<const T*>(out + row * kOutPitch + at * sizeof(T));
    }
}

// `COLS` columns of the warp's 32 rows out of tensor memory; `drained` is called when they are in registers.
template <class T, int COLS, class F>
__device__ __forceinline__ void store_columns(const Product& k, unsigned char* out, uint32_t sums, uint32_t r, uint32_t c, F&& drained)
{
    constexpr int kWidth = kOutBytes / sizeof(T);
    uint32_t v[COLS];
#pragma unroll
    for (int h = 0; h < COLS; h += 32) tcgen05_load32(sums + h, *reinterpret_cast<uint32_t(*)[32]>(&v[h]));
    tcgen05_wait_loads();
    tcgen05_fence_before();
    drained();
#pragma unroll
    for (int j = 0; j < COLS; j += kWidth) store_rows<T>(k, out, r, c + j, v + j);
}
template <int COLS, class F>
__device__ __forceinline__ void store_columns_any(const Product& k, unsigned char* out, uint32_t sums, uint32_t r, uint32_t c, F&& drained)
{
    if (k.type == ZCCL_BF16) store_columns<__nv_bfloat16, COLS>(k, out, sums, r, c, drained);
    else if (k.type == ZCCL_F16) store_columns<__half, COLS>(k, out, sums, r, c, drained);
    else store_columns<float, COLS>(k, out, sums, r, c, drained);
}

// ---------------------------------------------------------------- few rows, or few tiles

// A tile of 128 x BN to a cluster, whose CTAs take neighbouring pieces of the contraction.  Their sums are added in the order of the
// pieces out of each other's shared memory, each CTA some of the columns (or rows), so there is no workspace and no order that changes.
// Bound by latency, or for weights that do not stay in L2 by memory.  The few rows go along the instruction's columns (16 at least), the many along
// its 128 lanes: a stage is then little else than the weights.  More than one CTA to an SM: none allocates more tensor memory than its
// share by shared memory (SplitShape::kColumns), or clusters could wait for each other's.
template <int BN>
struct SplitShape {
    static constexpr int kStages = BN == 128 ? 3 : 4;
    static constexpr int kColAt = kRows * kRowBytes, kRowScaleAt = kColAt + BN * kRowBytes, kColScaleAt = kRowScaleAt + 2 * kMxTileBytes;
    static constexpr int kStage = kColScaleAt + 2 * kMxTileBytes;
    static constexpr int kScaleColumns = 16;                                     // of tensor memory, a set for each stage
    static constexpr int kSumColumns = BN < 32 ? 32 : BN;
    static constexpr int kColumns = BN <= 64 ? 128 : 256;
    static constexpr int kSumPitch = BN + 4;                                     // floats to a row of sums; across, sums are kept column by column instead
    static constexpr size_t kBytes = (size_t)kStage * kStages + 1024;
    static_assert(kSumColumns + kStages * kScaleColumns <= kColumns, "tensor memory");
    static_assert(kRows * kSumPitch * 4 <= kStage * kStages && 4 * 32 * kOutPitch <= kStage * kStages, "sums take the stages' place");
    static_assert((228 * 1024 / kBytes) * kColumns <= 512, "clusters must not wait for each other's tensor memory");
};

// N times four neighbouring sums, `step` bytes apart, added over the parts in their order.  All are asked for before the first is used: another SM's
// memory is far away.  And a warp's 32 lanes read 512 bytes in a row: what lies apart there comes at a fraction of the speed.
template <int PARTS, int N>
__device__ __forceinline__ void add_parts(uint32_t at, uint32_t step, float4 (&sum)[N])
{
    float4 v[PARTS][N];
#pragma unroll
    for (int p = 0; p < PARTS; ++p)
#pragma unroll
        for (int i = 0; i < N; ++i) v[p][i] = PARTS == 1 ? ld_shared4(at + i * step) : peer_load4(at + i * step, p);
#pragma unroll
    for (int i = 0; i < N; ++i) {
        sum[i] = v[0][i];
#pragma unroll
        for (int p = 1; p < PARTS; ++p) {
            sum[i].x += v[p][i].x;
            sum[i].y += v[p][i].y;
            sum[i].z += v[p][i].z;
            sum[i].w += v[p][i].w;
        }
    }
}
// The CTA's share of a tile's output; see mx4_split_kernel.
template <int BN, int PARTS>
__device__ __forceinline__ void store_share(const Product& k, uint32_t sums, uint32_t part, uint32_t r0, uint32_t c0)
{
    using S = SplitShape<BN>;
    const uint32_t thread = threadIdx.x - 64, warp = thread >> 5, lane = thread & 31u;
    if (BN <= (int)kMostAcross && k.across) {
        constexpr int kMine = BN / 4 / PARTS ? BN / 4 / PARTS : 1, N = kMine < 4 ? kMine : 4;     // columns of a warp, and at a time
        const uint32_t left = k.rows - min(k.rows, r0 + lane * 4);
        for (uint32_t j = 0; j < (uint32_t)kMine; j += N) {
            const uint32_t c = (part * kMine + j) * 4 + warp;                                     // and every fourth from here
            if (c >= (uint32_t)BN || c0 + c >= k.cols) break;
            float4 s[N];
            add_parts<PARTS, N>(sums + (c * kRows + lane * 4) * 4, 4 * kRows * 4, s);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float four[4] = {s[i].x, s[i].y, s[i].z, s[i].w};
                if (c0 + c + 4 * i < k.cols) store_four(k, (size_t)(c0 + c + 4 * i) * k.pitch + r0 + lane * 4, left, four);
            }
        }
    } else {
        constexpr uint32_t kQuads = BN / 4, kAtOnce = 128 / kQuads, kAll = kRows / kAtOnce, kSteps = kAll > PARTS ? kAll / PARTS : 1;   // rows that the four warps take at a time, and how often
        constexpr int N = kSteps < 4 ? kSteps : 4;
        const uint32_t c = thread % kQuads * 4, left = k.cols - min(k.cols, c0 + c);
        for (uint32_t j = 0; j < kSteps; j += N) {
            const uint32_t row = (part * kSteps + j) * kAtOnce + thread / kQuads;
            if (part * kSteps + j >= kAll || r0 + (part * kSteps + j) * kAtOnce >= k.rows) break;
            float4 s[N];
            add_parts<PARTS, N>(sums + (row * S::kSumPitch + c) * 4, kAtOnce * S::kSumPitch * 4, s);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float four[4] = {s[i].x, s[i].y, s[i].z, s[i].w};
                if (r0 + row + i * kAtOnce < k.rows) store_four(k, (size_t)(r0 + row + i * kAtOnce) * k.pitch + c0 + c, left, four);
            }
        }
    }
}

template <int BN>
__global__ void __launch_bounds__(kProductThreads, 1) mx4_split_kernel(const __grid_constant__ CUtensorMap r_map, const __grid_constant__ CUtensorMap c_map, const __grid_constant__ Product k)
{
    using S = SplitShape<BN>;
    constexpr int kStages = S::kStages;
    const bool across = BN <= (int)kMostAcross && k.across;
    extern __shared__ unsigned char raw[];
    __shared__ unsigned long long full[kStages], empty[kStages], done;
    __shared__ uint32_t tmem_at;
    unsigned char* const tiles = on_1024(raw);
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31u;

    if (warp == 0 && lane == 0) {
        prefetch_map(&r_map);
        prefetch_map(&c_map);
        for (int i = 0; i < kStages; ++i) {
            mbar_init(&full[i], 1);
            mbar_init(&empty[i], 1);
        }
        mbar_init(&done, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) tmem_alloc(&tmem_at, S::kColumns);
    tcgen05_fence_before();
    __syncthreads();
    tcgen05_fence_after();
    const uint32_t tmem = tmem_at;

    uint32_t parts;
    asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(parts));
    const uint32_t depth_tiles = (k.depth_blocks + 7) / 8, part = cluster_rank();
    const uint32_t k_begin = (uint32_t)((unsigned long long)depth_tiles * part / parts), k_end = (uint32_t)((unsigned long long)depth_tiles * (part + 1) / parts);
    uint32_t rt, ct;
    tile_of(k, blockIdx.x / parts, 8, rt, ct);
    const uint32_t c0 = ct * BN, groups = (k.depth_blocks + 3) / 4;
    const auto load_rows = [&](uint32_t s, uint32_t d) {
        unsigned char* const at = tiles + s * S::kStage;
        const uint32_t scale_bytes = groups_at(d, k.depth_blocks) * kMxTileBytes;
        mbar_expect_tx(&full[s], (kRows + BN) * kRowBytes + 2 * scale_bytes);
        tile_load(at, &r_map, (int)(d * kRowBytes), (int)(rt * kRows), &full[s]);
        bytes_load(at + S::kRowScaleAt, k.r_scales + ((size_t)rt * groups + 2 * d) * kMxTileBytes, scale_bytes, &full[s]);
    };
    // The kernel in front may still be at work on the columns' operand, so the rows' is asked for already: with `early` it was complete when that kernel
    // let this one start, since that one had waited for all before it.
    const bool loads = warp == 0 && lane == 0;
    uint32_t asked = 0;
    if (loads && k.early)
        for (; asked < (uint32_t)kStages && k_begin + asked < k_end; ++asked) load_rows(asked, k_begin + asked);
    __syncwarp();
    pdl_enter();

    if (warp == 0) {
        if (loads) {
            uint32_t n = 0;
            bool ok = true;
            for (uint32_t d = k_begin; d < k_end; ++d, ++n) {
                const uint32_t s = n % kStages;
                if (n >= kStages && !(ok = wait_for(&empty[s], (n / kStages - 1) & 1, k.stuck))) break;
                if (n >= asked) load_rows(s, d);
                unsigned char* const at = tiles + s * S::kStage;
                tile_load(at + S::kColAt, &c_map, (int)(d * kRowBytes), (int)c0, &full[s]);
                bytes_load(at + S::kColScaleAt, k.c_scales + ((size_t)(c0 / kMxBand) * groups + 2 * d) * kMxTileBytes, groups_at(d, k.depth_blocks) * kMxTileBytes, &full[s]);
            }
            settle<kStages>(full, empty, n, true, ok, k.stuck);
        }
    } else if (warp == 1) {
        if (elect_one()) {
            uint32_t n = 0;
            for (uint32_t d = k_begin; d < k_end; ++d, ++n) {
                const uint32_t s = n % kStages;
                if (!wait_for(&full[s], (n / kStages) & 1, k.stuck)) break;
                tcgen05_fence_after();
                const uint32_t at = smem_u32(tiles) + s * S::kStage;
                const uint32_t r_scale = tmem + S::kSumColumns + s * S::kScaleColumns, c_scale = r_scale + 8;
                for (uint32_t g = 0; g < groups_at(d, k.depth_blocks); ++g) {
                    tcgen05_copy_scales(r_scale + 4 * g, scales_descriptor(at + S::kRowScaleAt + g * kMxTileBytes));
                    tcgen05_copy_scales(c_scale + 4 * g, scales_descriptor(at + S::kColScaleAt + g * kMxTileBytes));
                }
                const unsigned long long r_codes = operand_descriptor(at), c_codes = operand_descriptor(at + S::kColAt);
                const uint32_t steps = steps_at(d, k.depth_blocks);
                for (uint32_t j = 0; j < steps; ++j)
                    tcgen05_mma_mx4(tmem, r_codes + 2 * j, c_codes + 2 * j, mx4_instruction(kRows, BN, (j & 1) * 2), r_scale + 4 * (j / 2), c_scale + 4 * (j / 2),
                                    n > 0 || j > 0);
                tcgen05_commit(&empty[s]);
            }
            tcgen05_commit(&done);
            wait_for(&done, 0, k.stuck);
        }
    } else if (wait_for(&done, 0, k.stuck)) {
        tcgen05_fence_after();
        const uint32_t quarter = warp & 3u, row = quarter * 32 + lane;
        if (BN == 128 && parts == 1) {
            unsigned char* const out = tiles + quarter * 32 * kOutPitch;
            const uint32_t sums = tmem + (quarter * 32 << 16), r = rt * kRows + quarter * 32;
            store_columns_any<128>(k, out, sums, r, c0, [] {});
        } else {
            constexpr int kWide = BN < 32 ? BN : 32;
            float* const to = reinterpret_cast<float*>(tiles) + (across ? row : row * S::kSumPitch);
#pragma unroll 1
            for (int c = 0; c < BN; c += kWide) {
                if (across && c0 + c >= k.cols) break;
                uint32_t v[32];
                if (kWide == 32) tcgen05_load32(tmem + (quarter * 32 << 16) + c, v);
                else tcgen05_load16(tmem + (quarter * 32 << 16) + c, v);
                tcgen05_wait_loads();
                if (across) {
#pragma unroll
                    for (int j = 0; j < kWide; ++j) to[(c + j) * kRows] = __uint_as_float(v[j]);
                } else {
#pragma unroll
                    for (int j = 0; j < kWide; j += 4) *reinterpret_cast<uint4*>(to + c + j) = make_uint4(v[j], v[j + 1], v[j + 2], v[j + 3]);
                }
            }
        }
        tcgen05_fence_before();
    }
    __syncwarp();
    cluster_sync();
    if (warp >= 2 && !(BN == 128 && parts == 1)) {
        const uint32_t sums = smem_u32(tiles), r0 = rt * kRows;
        if (parts == 8) store_share<BN, 8>(k, sums, part, r0, c0);
        else if (parts == 4) store_share<BN, 4>(k, sums, part, r0, c0);
        else if (parts == 2) store_share<BN, 2>(k, sums, part, r0, c0);
        else store_share<BN, 1>(k, sums, part, r0, c0);
    }
    __syncwarp();
    cluster_sync();                        // nobody leaves while its sums are still read
    tcgen05_fence_after();
    if (warp == 1) tmem_free(tmem, S::kColumns);
}

// ---------------------------------------------------------------- a few tokens

// The layer of a few rows in one launch: mx4_split_kernel<16> across, whose CTAs quantise their piece of x themselves, into the places in shared memory
// where a load would have put it, while the first weights are on their way.  A quantisation of its own takes 1.4 us and leaves the memory idle for
// longer: 1 x 8192 x 16384 with weights from memory 15.6 us, as two launches 17.2 us; 1 x 4096 x 4096 5.0 and 6.2 us.  Every CTA quantises all of its
// piece, so there may not be much of it (kMostUnits; 8 x 2048 x 30000, 128 runs to a CTA, took 12.5 us instead of 10.1 us).
struct TokenShape {
    using S = SplitShape<16>;
    static constexpr int kStages = S::kStages, kRowScaleAt = kRows * kRowBytes, kStage = kRowScaleAt + 2 * kMxTileBytes;
    // a depth tile of x: 16 rows of codes, and two tiles of scales of which 16 rows count; the rest of a tile is the next one's, or nothing
    static constexpr int kCodes = 16 * kRowBytes, kScales = 256;
    static constexpr uint32_t kMostUnits = 48;                                   // runs of 128 elements of a row: what 12 half-warps load at once
    static constexpr size_t kMostBytes = 112 * 1024;                             // two CTAs to an SM
    static size_t bytes(size_t depth_tiles) { return (size_t)kStage * kStages + depth_tiles * (kCodes + 2 * kScales) + kMxTileBytes + 1024; }
    static_assert(16 * kRows * 4 <= kStage * kStages, "sums take the stages' place");
    static_assert(((228 * 1024) / (kStage * kStages + 1024)) * S::kColumns <= 512, "clusters must not wait for each other's tensor memory");
};
struct Tokens {
    const void* x;
    size_t pitch;
    uint32_t cols;
    int vec;                                  // every row of x begins on a 16-byte boundary
};

template <class T>
__global__ void __launch_bounds__(kProductThreads, 1) mx4_token_kernel(const __grid_constant__ CUtensorMap r_map, const __grid_constant__ Product k, const __grid_constant__ Tokens x)
{
    using S = TokenShape;
    constexpr int kStages = S::kStages, BN = 16;
    extern __shared__ unsigned char raw[];
    __shared__ unsigned long long full[kStages], empty[kStages], done;
    __shared__ uint32_t tmem_at;
    unsigned char* const tiles = on_1024(raw);
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31u;

    if (warp == 0 && lane == 0) {
        prefetch_map(&r_map);
        for (int i = 0; i < kStages; ++i) {
            mbar_init(&full[i], 1);
            mbar_init(&empty[i], 1);
        }
        mbar_init(&done, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) tmem_alloc(&tmem_at, S::S::kColumns);
    tcgen05_fence_before();
    __syncthreads();
    tcgen05_fence_after();
    const uint32_t tmem = tmem_at;
    pdl_enter();

    uint32_t parts;
    asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(parts));
    const uint32_t depth_tiles = (k.depth_blocks + 7) / 8, part = cluster_rank(), rt = blockIdx.x / parts;
    const uint32_t k_begin = (uint32_t)((unsigned long long)depth_tiles * part / parts), k_end = (uint32_t)((unsigned long long)depth_tiles * (part + 1) / parts);
    const uint32_t groups = (k.depth_blocks + 3) / 4, mine = k_end - k_begin;
    unsigned char* const codes = tiles + S::kStage * kStages;
    unsigned char* const scales = codes + (size_t)mine * S::kCodes;
    const auto load = [&](uint32_t n) {
        const uint32_t s = n % kStages, d = k_begin + n, scale_bytes = groups_at(d, k.depth_blocks) * kMxTileBytes;
        unsigned char* const at = tiles + s * S::kStage;
        mbar_expect_tx(&full[s], kRows * kRowBytes + scale_bytes);
        tile_load(at, &r_map, (int)(d * kRowBytes), (int)(rt * kRows), &full[s]);
        bytes_load(at + S::kRowScaleAt, k.r_scales + ((size_t)rt * groups + 2 * d) * kMxTileBytes, scale_bytes, &full[s]);
    };
    uint32_t asked = 0;
    if (warp == 0 && lane == 0)
        for (; asked < (uint32_t)kStages && asked < mine; ++asked) load(asked);
    __syncwarp();

    // x: 16 lanes take a run of 128 elements of a row, as in quantising to memory; four runs are loaded at a time
    {
        const uint32_t sub = threadIdx.x & 15u, g_begin = 2 * k_begin, runs = min(2 * k_end, groups) - g_begin, units = k.cols * runs;
        constexpr uint32_t kHalves = kProductThreads / 16, kAtOnce = 4;
        for (uint32_t u0 = (threadIdx.x >> 4) & ~1u; u0 < units; u0 += kHalves * kAtOnce) {
            const uint32_t u = u0 + (lane >> 4);
            MxTwo<T> v[kAtOnce][4];
#pragma unroll
            for (uint32_t i = 0; i < kAtOnce; ++i) {
                const uint32_t at_u = u + i * kHalves, r = at_u / runs, at = (g_begin + at_u - r * runs) * kMxGroup + sub * 8;
                if (at_u < units && at < x.cols) {
                    const T* const row = (const T*)x.x + (size_t)r * x.pitch;
                    if (x.vec) load8<T, true>(row, at, x.cols, v[i]);
                    else load8<T, false>(row, at, x.cols, v[i]);
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[i][j] = MxTwo<T>{};
                }
            }
#pragma unroll
            for (uint32_t i = 0; i < kAtOnce; ++i) {
                uint32_t s;
                const uint32_t w = quantize_run(v[i], sub, s), at_u = u + i * kHalves;
                if (at_u < units) {
                    const uint32_t r = at_u / runs, g = at_u - r * runs, piece = (g & 1u) * 4 + (sub >> 2);
                    *reinterpret_cast<uint32_t*>(codes + (g >> 1) * S::kCodes + r * kRowBytes + ((piece ^ (r & 7u)) << 4) + (sub & 3u) * 4) = w;
                    if (sub == 0) *reinterpret_cast<uint32_t*>(scales + g * S::kScales + r * 16) = s;
                }
            }
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    __syncthreads();

    if (warp == 0) {
        if (lane == 0) {
            uint32_t n = asked;
            bool ok = true;
            for (; n < mine; ++n) {
                if (n >= (uint32_t)kStages && !(ok = wait_for(&empty[n % kStages], (n / kStages - 1) & 1, k.stuck))) break;
                load(n);
            }
            settle<kStages>(full, empty, n, true, ok, k.stuck);
        }
    } else if (warp == 1) {
        if (elect_one()) {
            for (uint32_t n = 0; n < mine; ++n) {
                const uint32_t s = n % kStages, d = k_begin + n;
                if (!wait_for(&full[s], (n / kStages) & 1, k.stuck)) break;
                tcgen05_fence_after();
                const uint32_t at = smem_u32(tiles) + s * S::kStage, r_scale = tmem + S::S::kSumColumns + s * S::S::kScaleColumns, c_scale = r_scale + 8;
                for (uint32_t g = 0; g < groups_at(d, k.depth_blocks); ++g) {
                    tcgen05_copy_scales(r_scale + 4 * g, scales_descriptor(at + S::kRowScaleAt + g * kMxTileBytes));
                    tcgen05_copy_scales(c_scale + 4 * g, scales_descriptor(smem_u32(scales) + (2 * n + g) * S::kScales));
                }
                const unsigned long long r_codes = operand_descriptor(at), c_codes = operand_descriptor(smem_u32(codes) + n * S::kCodes);
                const uint32_t steps = steps_at(d, k.depth_blocks);
                for (uint32_t j = 0; j < steps; ++j)
                    tcgen05_mma_mx4(tmem, r_codes + 2 * j, c_codes + 2 * j, mx4_instruction(kRows, BN, (j & 1) * 2), r_scale + 4 * (j / 2), c_scale + 4 * (j / 2), n > 0 || j > 0);
                tcgen05_commit(&empty[s]);
            }
            tcgen05_commit(&done);
            wait_for(&done, 0, k.stuck);
        }
    } else if (wait_for(&done, 0, k.stuck)) {
        tcgen05_fence_after();
        const uint32_t quarter = warp & 3u;
        float* const to = reinterpret_cast<float*>(tiles) + quarter * 32 + lane;
        uint32_t v[32];
        tcgen05_load16(tmem + (quarter * 32 << 16), v);
        tcgen05_wait_loads();
#pragma unroll
        for (int j = 0; j < BN; ++j) to[j * kRows] = __uint_as_float(v[j]);
        tcgen05_fence_before();
    }
    __syncwarp();
    cluster_sync();
    if (warp >= 2) {
        const uint32_t sums = smem_u32(tiles), r0 = rt * kRows;
        if (parts == 8) store_share<BN, 8>(k, sums, part, r0, 0);
        else if (parts == 4) store_share<BN, 4>(k, sums, part, r0, 0);
        else if (parts == 2) store_share<BN, 2>(k, sums, part, r0, 0);
        else store_share<BN, 1>(k, sums, part, r0, 0);
    }
    __syncwarp();
    cluster_sync();                        // nobody leaves while its sums are still read
    tcgen05_fence_after();
    if (warp == 1) tmem_free(tmem, S::S::kColumns);
}

// ---------------------------------------------------------------- many tiles

// A pair of CTAs (the two of a cluster) works on a tile of 256 x 256: the first issues instructions that use both tensor cores, each CTA brings and
// keeps its 128 rows of one operand and half of the other, so an SM reads 256 rows for 128 x 256 sums.  (Tiles of 128 x 192 to a single CTA were bound by
// the way from L2: 157 us for 4096 x 8192 x 8192, 12 TB/s; so are narrower tiles of a pair, whose stages take nearly as long.)  Now 100 us, 5.5 PFLOP/s, the
// tensor cores active for 70 % of the cycles: what is left goes by how fast the one thread issues and by the power that the clock is given.
// Eight warps read a tile's sums out, each half of the columns of a quarter of the rows, all into registers at once: 256 columns of sums do not fit tensor
// memory twice next to the scales, so the next tile's instructions wait for that.
struct PairShape {
    static constexpr int kCols = 256, kStages = 5;
    static constexpr int kBands = kCols / kMxBand;                               // tiles of scales that a tile's columns lie in
    static constexpr int kColAt = kRows * kRowBytes, kRowScaleAt = kColAt + kCols / 2 * kRowBytes, kColScaleAt = kRowScaleAt + 2 * kMxTileBytes;
    static constexpr int kStage = kColScaleAt + 2 * kMxTileBytes * kBands;
    static constexpr int kScaleColumns = 8 + 8 * kBands;                         // of tensor memory, a set for each stage
    static constexpr int kColumns = 512;
    static constexpr int kWarps = 8, kThreads = 64 + 32 * kWarps;                // that read sums out, and all
    static constexpr size_t kBytes = (size_t)kStage * kStages + kWarps * 32 * kOutPitch + 1024;
    static_assert(kCols + kStages * kScaleColumns <= kColumns, "tensor memory");
    static_assert(kBytes <= 227 * 1024 && kBytes > 114 * 1024, "one CTA to an SM");
};

__global__ void __launch_bounds__(PairShape::kThreads, 1) mx4_pair_kernel(const __grid_constant__ CUtensorMap r_map, const __grid_constant__ CUtensorMap c_map, const __grid_constant__ CUtensorMap r_scale_map,
                                                                      const __grid_constant__ CUtensorMap c_scale_map, const __grid_constant__ Product k)
{
    using S = PairShape;
    constexpr int kStages = S::kStages, BN = S::kCols;
    extern __shared__ unsigned char raw[];
    __shared__ unsigned long long full[kStages], empty[kStages], done, free_, drained;
    __shared__ uint32_t tmem_at;
    unsigned char* const tiles = on_1024(raw);
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31u, rank = cluster_rank();

    if (warp == 0 && lane == 0) {
        prefetch_map(&r_map);
        prefetch_map(&c_map);
        prefetch_map(&r_scale_map);
        prefetch_map(&c_scale_map);
        for (int i = 0; i < kStages; ++i) {
            mbar_init(&full[i], 1);
            mbar_init(&empty[i], 1);
        }
        mbar_init(&done, 1);
        mbar_init(&free_, 2 * S::kWarps);
        mbar_init(&drained, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) tmem_alloc_pair(&tmem_at, S::kColumns);
    tcgen05_fence_before();
    __syncthreads();
    cluster_sync();
    tcgen05_fence_after();
    const uint32_t tmem = tmem_at;
    pdl_enter();

    const uint32_t depth_tiles = (k.depth_blocks + 7) / 8, total = k.row_tiles * k.col_tiles, first = blockIdx.x / 2, stride = gridDim.x / 2;
    constexpr uint32_t kBand = 8;                   // tiles of rows that share a walk

    if (warp == 0) {
        if (lane == 0) {
            // what lands in either CTA counts at the first one's barrier
            constexpr uint32_t kBoth = 2 * ((kRows + BN / 2) * kRowBytes + 2 * kMxTileBytes * (1 + S::kBands));
            uint32_t n = 0;
            bool ok = true;
            for (uint32_t t = first; t < total && ok; t += stride) {
                uint32_t rt, ct;
                tile_of(k, t, kBand, rt, ct);
                const int row_band = (int)(rt * 2 + rank), c0 = (int)(ct * BN + rank * (BN / 2));
                for (uint32_t d = 0; d < depth_tiles; ++d, ++n) {
                    const uint32_t s = n % kStages;
                    if (n >= kStages && !(ok = wait_for(&empty[s], (n / kStages - 1) & 1, k.stuck))) break;
                    unsigned char* const at = tiles + s * S::kStage;
                    const uint32_t bar = address_at(&full[s], 0);
                    if (rank == 0) mbar_expect_tx(&full[s], kBoth);
                    tile_load_pair(at, &r_map, (int)(d * kRowBytes), row_band * kRows, bar);
                    tile_load_pair(at + S::kColAt, &c_map, (int)(d * kRowBytes), c0, bar);
                    scales_load_pair(at + S::kRowScaleAt, &r_scale_map, (int)(2 * d), row_band, bar);
                    scales_load_pair(at + S::kColScaleAt, &c_scale_map, (int)(2 * d), (int)(ct * S::kBands), bar);
                }
            }
            settle<kStages>(full, empty, n, rank == 0, ok, k.stuck);   // the first CTA sees both's loads; each sees the arrivals at its own `empty`
        }
    } else if (warp == 1) {
        if (rank == 0 && elect_one()) {
            // What bounds a large product is how fast this thread issues: a stage's instructions run for 512 cycles, and with one wait more to a stage (or the
            // next stage's scales in front of this one's instructions) 4096 x 8192 x 8192 took 20 to 30 us longer.
            const uint32_t base = smem_u32(tiles);
            const auto issue = [&](uint32_t s, bool add, uint32_t groups, uint32_t steps) {
                const uint32_t at = base + s * S::kStage, r_scale = tmem + BN + s * S::kScaleColumns, c_scale = r_scale + 8;
                const unsigned long long r_codes = operand_descriptor(at), c_codes = operand_descriptor(at + S::kColAt), r_in = scales_descriptor(at + S::kRowScaleAt),
                                         c_in = scales_descriptor(at + S::kColScaleAt);
#pragma unroll
                for (uint32_t g = 0; g < 2; ++g)
                    if (g < groups) {
                        tcgen05_copy_scales_pair(r_scale + 4 * g, r_in + g * (kMxTileBytes >> 4));
#pragma unroll
                        for (uint32_t b = 0; b < S::kBands; ++b) tcgen05_copy_scales_pair(c_scale + 4 * (g * S::kBands + b), c_in + (b * 2 + g) * (kMxTileBytes >> 4));
                    }
#pragma unroll
                for (uint32_t j = 0; j < 4; ++j)
                    if (j < steps)
                        tcgen05_mma_mx4_pair(tmem, r_codes + 2 * j, c_codes + 2 * j, mx4_instruction(2 * kRows, BN, (j & 1) * 2), r_scale + 4 * (j / 2),
                                             c_scale + 4 * S::kBands * (j / 2), add || j > 0);
            };
            uint32_t s = 0, parity = 0, i = 0;
            bool ok = true;
            for (uint32_t t = first; t < total && ok; t += stride, ++i) {
                if (i >= 1) {
                    if (!(ok = wait_for_cluster(&free_, (i - 1) & 1, k.stuck))) break;
                    tcgen05_fence_after();
                }
                for (uint32_t d = 0; d < depth_tiles; ++d) {
                    if (!(ok = wait_for(&full[s], parity, k.stuck))) break;
                    tcgen05_fence_after();
                    if (d + 1 < depth_tiles) issue(s, d > 0, 2, 4);
                    else issue(s, d > 0, groups_at(d, k.depth_blocks), steps_at(d, k.depth_blocks));
                    tcgen05_commit_pair(&empty[s]);
                    if (++s == kStages) {
                        s = 0;
                        parity ^= 1;
                    }
                }
                tcgen05_commit_pair(&done);
            }
            tcgen05_commit_own(&drained);
            wait_for(&drained, 0, k.stuck);
        }
    } else {
        const uint32_t quarter = warp & 3u, half = (warp - 2) >> 2;
        unsigned char* const out = tiles + S::kStage * kStages + (warp - 2) * 32 * kOutPitch;
        uint32_t i = 0;
        for (uint32_t t = first; t < total; t += stride, ++i) {
            uint32_t rt, ct;
            tile_of(k, t, kBand, rt, ct);
            const uint32_t c = half * (BN / 2);
            if (!wait_for(&done, i & 1, k.stuck)) break;
            tcgen05_fence_after();
            store_columns_any<BN / 2>(k, out, tmem + c + (quarter * 32 << 16), (rt * 2 + rank) * kRows + quarter * 32, ct * BN + c, [&] {
                __syncwarp();
                if (lane == 0) mbar_arrive_at(&free_, 0);
            });
        }
    }
    __syncwarp();
    tcgen05_fence_before();
    // Neither leaves while the other still reaches its barriers or its tensor memory.  The tensor core's arrivals at the second CTA's barriers are no thread's
    // doing and not ordered by this: that CTA has waited for each of them itself (`done` where sums are read out, `empty` in settle).
    cluster_sync();
    tcgen05_fence_after();
    if (warp == 1) tmem_free_pair(tmem, S::kColumns);
}

// A test's: waits, as the products do, for a barrier that nothing arrives at.
__global__ void mx4_waiting_kernel(uint32_t* stuck)
{
    __shared__ unsigned long long bar;
    pdl_enter();
    mbar_init(&bar, 1);
    wait_for(&bar, 0, stuck);
}

using EncodeFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*, const cuuint32_t*,
                              CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
constexpr int kMaxDevices = 64;
std::mutex g_product_mu;
EncodeFn g_product_encode = nullptr;
struct ProductDevice {
    bool ready = false;
    int sms = 0, pairs = 0;       // pairs of CTAs that are resident together
    uint32_t* stuck = nullptr;    // see Product
};
bool is_stuck(const ProductDevice& d) { return *(volatile const uint32_t*)d.stuck != 0; }
ProductDevice g_product_dev[kMaxDevices];

template <int BN>
cudaError_t split_attr() { return cudaFuncSetAttribute(mx4_split_kernel<BN>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)SplitShape<BN>::kBytes); }

template <class T>
cudaError_t token_attr() { return cudaFuncSetAttribute(mx4_token_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)TokenShape::kMostBytes); }

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
        if (e == cudaSuccess) e = split_attr<16>();
        if (e == cudaSuccess) e = split_attr<32>();
        if (e == cudaSuccess) e = split_attr<64>();
        if (e == cudaSuccess) e = split_attr<128>();
        if (e == cudaSuccess) e = token_attr<float>();
        if (e == cudaSuccess) e = token_attr<__nv_bfloat16>();
        if (e == cudaSuccess) e = token_attr<__half>();
        if (e == cudaSuccess) e = cudaFuncSetAttribute(mx4_pair_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)PairShape::kBytes);
        if (e != cudaSuccess) return e;
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)d.sms / 2 * 2);
        cfg.blockDim = dim3(PairShape::kThreads);
        cfg.dynamicSmemBytes = PairShape::kBytes;
        cudaLaunchAttribute attr;
        attr.id = cudaLaunchAttributeClusterDimension;
        attr.val.clusterDim.x = 2; attr.val.clusterDim.y = 1; attr.val.clusterDim.z = 1;
        cfg.attrs = &attr;
        cfg.numAttrs = 1;
        e = cudaOccupancyMaxActiveClusters(&d.pairs, mx4_pair_kernel, &cfg);
        if (e != cudaSuccess) return e;
        if (d.pairs < 1) return cudaErrorNotSupported;
        if (!d.stuck) {
            // also where the first call is one that is captured
            cudaStreamCaptureMode mode = cudaStreamCaptureModeRelaxed;
            if ((e = cudaThreadExchangeStreamCaptureMode(&mode)) != cudaSuccess) return e;
            void* word = nullptr;
            e = cudaHostAlloc(&word, sizeof(uint32_t), cudaHostAllocPortable | cudaHostAllocMapped);
            cudaThreadExchangeStreamCaptureMode(&mode);
            if (e != cudaSuccess) return e;
            d.stuck = (uint32_t*)word;
            *d.stuck = 0;
        }
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

// Tiles of scales as [bands][groups][512 bytes]; a box is two groups of `bands` bands.
bool scales_map(CUtensorMap* map, const void* scales, size_t rows, size_t blocks, int bands)
{
    const size_t groups = (blocks + 3) / 4;
    const cuuint64_t size[3] = {kMxTileBytes / 4, groups, mx_bands(rows)}, stride[2] = {kMxTileBytes, groups * kMxTileBytes};
    const cuuint32_t box[3] = {kMxTileBytes / 4, 2, (cuuint32_t)bands}, step[3] = {1, 1, 1};
    return g_product_encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT32, 3, const_cast<void*>(scales), size, stride, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                            CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

struct Sides {
    const void *r_codes, *c_codes;
    size_t rows, cols;
};
constexpr size_t up(size_t n, size_t per) { return (n + per - 1) / per; }

bool set_tiles(Product& k, const Sides& s, int row_tile, int col_tile)
{
    k.row_tiles = (uint32_t)up(s.rows, row_tile);
    k.col_tiles = (uint32_t)up(s.cols, col_tile);
    return (size_t)k.row_tiles * k.col_tiles <= 0x7FFFFFFFu / 16;
}
int launched(cudaError_t e)
{
    if (e == cudaSuccess) count_launches(1);
    return e == cudaSuccess ? ZCCL_OK : ZCCL_E_CUDA;
}
// Tiles narrower than a tile of scales (128) are for outputs that one of them is wide enough for: their scales begin where the tile of scales does.
template <int BN>
int launch_split(const Sides& s, Product k, unsigned parts, cudaStream_t st)
{
    CUtensorMap r, c;
    if (!set_tiles(k, s, kRows, BN) || (BN < kMxBand && k.col_tiles > 1)) return ZCCL_E_ARG;
    if (!operand_map(&r, s.r_codes, s.rows, k.depth_blocks, kRows) || !operand_map(&c, s.c_codes, s.cols, k.depth_blocks, BN)) return ZCCL_E_CUDA;
    return launched(launch_cluster(parts, mx4_split_kernel<BN>, dim3(k.row_tiles * k.col_tiles * parts), dim3(kProductThreads), SplitShape<BN>::kBytes, st, r, c, k));
}
int launch_pair(const Sides& s, Product k, int pairs, cudaStream_t st)
{
    CUtensorMap r, c, rs, cs;
    if (!set_tiles(k, s, 2 * kRows, PairShape::kCols)) return ZCCL_E_ARG;
    if (!operand_map(&r, s.r_codes, s.rows, k.depth_blocks, kRows) || !operand_map(&c, s.c_codes, s.cols, k.depth_blocks, PairShape::kCols / 2) ||
        !scales_map(&rs, k.r_scales, s.rows, k.depth_blocks, 1) || !scales_map(&cs, k.c_scales, s.cols, k.depth_blocks, PairShape::kBands)) return ZCCL_E_CUDA;
    const unsigned clusters = std::min(k.row_tiles * k.col_tiles, (unsigned)pairs);
    return launched(launch_cluster(2, mx4_pair_kernel, dim3(2 * clusters), dim3(PairShape::kThreads), PairShape::kBytes, st, r, c, rs, cs, k));
}

bool aligned16(const void* p) { return p && ((uintptr_t)p & 15u) == 0; }

// In how many pieces, a power of two up to 8, the contraction goes.  Narrow tiles: as many as there is room for at two CTAs to an SM.  Tiles of 128 x 128: at
// one to an SM, and not at all where that saves fewer than seven stages, since joining their sums takes 2.6 us and a stage 0.4 us (measured, in
// a graph: 512^3 4.0 us in one piece and 6.1 us in two; 300 x 300 x 16384 28.7 us in one, 9.5 us in eight; 128 x 4096 x 4096 11.8 us in one,
// 7.5 us in four and 10.6 us in eight at two to an SM).
unsigned parts_of(size_t tiles, size_t depth_tiles, size_t sms, bool wide)
{
    unsigned parts = 1;
    while (parts < 8 && parts * 2 <= depth_tiles && tiles * parts * 2 <= (wide ? 1 : 2) * sms) parts *= 2;
    return wide && depth_tiles - up(depth_tiles, parts) < 7 ? 1 : parts;
}

// The layer of a few tokens in one launch; false where that would not pay (see mx4_token_kernel) or the arguments are wrong.
template <class T>
bool tokens(const T* x, int type, size_t m, size_t k, size_t x_pitch, const void* w_codes, const void* w_scales, size_t n, void* y, size_t pitch, cudaStream_t st, int& rc)
{
    const ProductDevice* dev;
    const size_t depth_tiles = up(k, kDepth), row_tiles = up(n, kRows);
    if (m > 16 || m >= n || n > 0x7FFFFF00u || k > 0x7FFFFF00u || product_device(&dev) != cudaSuccess) return false;
    const unsigned parts = parts_of(row_tiles, depth_tiles, (size_t)dev->sms, false);
    const size_t mine = up(depth_tiles, parts), bytes = TokenShape::bytes(mine);
    if (m * std::min(2 * mine, mx_groups(k)) > TokenShape::kMostUnits || bytes > TokenShape::kMostBytes || row_tiles * parts > 0x7FFFFFFFu) return false;
    Product p{};
    p.r_scales = (const unsigned char*)w_scales;
    p.y = y;
    p.pitch = pitch;
    p.type = type;
    p.wide = (uintptr_t)y % 16 == 0 && pitch * sizeof(T) % 16 == 0;
    p.across = 1;
    p.stuck = dev->stuck;
    p.depth_blocks = (uint32_t)mx_blocks(k);
    p.rows = (uint32_t)n;
    p.cols = (uint32_t)m;
    const Tokens in{x, x_pitch, (uint32_t)k, (uintptr_t)x % 16 == 0 && x_pitch * sizeof(T) % 16 == 0};
    CUtensorMap map;
    if (!operand_map(&map, w_codes, n, p.depth_blocks, kRows)) rc = ZCCL_E_CUDA;
    else rc = launched(launch_cluster(parts, mx4_token_kernel<T>, dim3((unsigned)row_tiles * parts), dim3(kProductThreads), bytes, st, map, p, in));
    return true;
}

// `weights_ready`: B was complete before the kernel in front on the stream started.
int multiply(const void* a_codes, const void* a_scales, size_t m, const void* b_codes, const void* b_scales, size_t n, size_t k, void* y, int type, size_t pitch, bool weights_ready, void* stream)
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
    if (is_stuck(*dev)) return ZCCL_E_TIMEOUT;
    Product p{};
    p.stuck = dev->stuck;
    p.y = y;
    p.pitch = pitch;
    p.type = type;
    p.wide = (uintptr_t)y % 16 == 0 && pitch * element % 16 == 0;
    p.depth_blocks = (uint32_t)mx_blocks(k);
    // few rows of the output go along the instruction's columns, the weights along its lanes (from 65 rows on they fill the lanes well enough, and their sums are
    // stored along the rows: 100 x 500 x 300 4.3 us, across 6.4 us)
    Sides sides{a_codes, b_codes, m, n};
    p.r_scales = (const unsigned char*)a_scales;
    p.c_scales = (const unsigned char*)b_scales;
    p.across = m < n && m <= kMostAcross;
    p.early = weights_ready && p.across;
    if (p.across) {
        std::swap(sides.r_codes, sides.c_codes);
        std::swap(sides.rows, sides.cols);
        std::swap(p.r_scales, p.c_scales);
    }
    p.rows = (uint32_t)sides.rows;
    p.cols = (uint32_t)sides.cols;
    const size_t sms = (size_t)dev->sms, depth_tiles = up(p.depth_blocks, 8), tiles = up(sides.rows, kRows) * up(sides.cols, 128);
    if (tiles <= sms || sides.cols <= 128) {
        const unsigned parts = parts_of(tiles, depth_tiles, sms, sides.cols > 64);
        if (sides.cols <= 16) return launch_split<16>(sides, p, parts, st);
        if (sides.cols <= 32) return launch_split<32>(sides, p, parts, st);
        if (sides.cols <= 64) return launch_split<64>(sides, p, parts, st);
        return launch_split<128>(sides, p, parts, st);
    }
    return launch_pair(sides, p, dev->pairs, st);
}

}  // namespace
}  // namespace zccl

using namespace zccl;

extern "C" {

int zccl_mx4_matmul(const void* a_codes, const void* a_scales, size_t m, const void* b_codes, const void* b_scales, size_t n, size_t k, void* y, int type, size_t pitch, void* stream)
{
    return multiply(a_codes, a_scales, m, b_codes, b_scales, n, k, y, type, pitch, false, stream);
}

int zccl_mx4_linear(const void* x, int type, size_t m, size_t k, size_t x_pitch, const void* w_codes, const void* w_scales, size_t n, void* x_codes, void* x_scales, void* y, size_t pitch, void* stream)
{
    if (m == 0 || n == 0 || k == 0) return multiply(x_codes, x_scales, m, w_codes, w_scales, n, k, y, type, pitch, false, stream);
    if (type < ZCCL_F32 || type > ZCCL_F16 || !aligned16(w_codes) || !aligned16(w_scales) || !aligned16(x_codes) || !aligned16(x_scales) || pitch < n || x_pitch < k) return ZCCL_E_ARG;
    const size_t element = type == ZCCL_F32 ? 4 : 2;
    if (!x || !y || (uintptr_t)x % element || (uintptr_t)y % element) return ZCCL_E_ARG;
    const ProductDevice* dev;
    if (product_device(&dev) != cudaSuccess) return ZCCL_E_CUDA;
    if (is_stuck(*dev)) return ZCCL_E_TIMEOUT;
    cudaStream_t st = (cudaStream_t)stream;
    int rc = ZCCL_OK;
    if (type == ZCCL_F32 ? tokens((const float*)x, type, m, k, x_pitch, w_codes, w_scales, n, y, pitch, st, rc)
        : type == ZCCL_BF16 ? tokens((const __nv_bfloat16*)x, type, m, k, x_pitch, w_codes, w_scales, n, y, pitch, st, rc)
                            : tokens((const __half*)x, type, m, k, x_pitch, w_codes, w_scales, n, y, pitch, st, rc)) return rc;
    rc = zccl_mx4_quantize(x, type, m, k, x_pitch, 0, x_codes, x_scales, stream);
    return rc == ZCCL_OK ? multiply(x_codes, x_scales, m, w_codes, w_scales, n, k, y, type, pitch, true, stream) : rc;
}

int zccl_mx4_status(void* stream)
{
    const ProductDevice* dev;
    if (product_device(&dev) != cudaSuccess || cudaStreamSynchronize((cudaStream_t)stream) != cudaSuccess) return ZCCL_E_CUDA;
    if (!is_stuck(*dev)) return ZCCL_OK;
    *(volatile uint32_t*)dev->stuck = 0;
    return ZCCL_E_TIMEOUT;
}

int zccl_debug_mx4_wait(void* stream)
{
    const ProductDevice* dev;
    if (product_device(&dev) != cudaSuccess) return ZCCL_E_CUDA;
    return launched(launch_k(mx4_waiting_kernel, dim3(1), dim3(1), 0, (cudaStream_t)stream, dev->stuck));
}

}  // extern "C"
