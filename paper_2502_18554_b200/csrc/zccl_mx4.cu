// Quantisation to microscaled 4-bit floating point, along the rows or along the columns, and back.
#include "../../include/zccl.h"
#include "zccl_mx4.cuh"

#include <algorithm>

namespace zccl {
namespace {

constexpr int kMxThreads = 256;

// One matrix to quantise: its sizes, how its kernel goes round it (rows), and the launch's CTA that it begins at.
enum MxKind : uint32_t { kMxRowsStrips, kMxRows, kMxRowsPlain, kMxColumns, kMxColumnsPlain };
struct MxJob {
    const void* x;
    void* codes;
    unsigned char* scales;
    size_t pitch;
    uint32_t rows, cols, blocks, groups;
    uint32_t strips, total, work, step_row, step_strip;   // rows: see Rounds; `work`: CTAs that quantise, those behind fill scales up
    uint32_t across;                                      // columns: CTAs to a band of eight blocks
    uint32_t first;
    MxKind kind;
};
constexpr int kMxJobs = 8;
struct MxJobs {
    MxJob job[kMxJobs];
    int count;
};

// Inputs are not __restrict__ anywhere here: the kernel in front may still be writing them, and loads of what never changes could be moved in front of the wait.

// Rows: 16 lanes take STRIP groups of 128 neighbouring elements of a row (a group: four blocks, one word of scales), a lane
// eight elements of each, so loads are 16 bytes a lane and codes leave as whole lines.  Blocks behind the last are quantised as zeros. CTAs from
// `work` on write the scales of the rows that fill the last band up, a word a thread.
// Bound by memory where it is large (8192 x 8192 bf16: 25.8 us, 6.6 TB/s); with one group at a time the indexes cost more instructions than the elements
// (23 to an element, 52.5 us).  The lane that has a block's scale stores it: putting four together for one lane to store took 3 % longer.  Rows that do not begin on
// 16-byte boundaries are loaded element by element and take twice as long (16384 x 4097: 56 us; cutting them out of aligned pieces took as long).
template <class T, bool VEC, int STRIP>
__device__ __forceinline__ void quantize_rows(const MxJob& job, uint32_t cta)
{
    const T* const x = (const T*)job.x;
    const uint32_t rows = job.rows, cols = job.cols, blocks = job.blocks, groups = job.groups, strips = job.strips, total = job.total, work = job.work;
    const uint32_t step_row = job.step_row, step_strip = job.step_strip;
    const size_t pitch = job.pitch;
    uint32_t* __restrict__ const codes = (uint32_t*)job.codes;
    unsigned char* __restrict__ const scales = job.scales;
    if (cta >= work) {
        const uint32_t i = (cta - work) * kMxThreads + threadIdx.x, r = rows + i / groups;
        if ((rows - 1) / kMxBand == r / kMxBand) *reinterpret_cast<uint32_t*>(scales + mx_scale_at(r, i % groups, groups)) = 0u;
        return;
    }
    const uint32_t sub = threadIdx.x & 15u;
    uint32_t u = cta * (kMxThreads / 16) + (threadIdx.x >> 4);
    uint32_t r = u / strips, strip = u - r * strips;
    const uint32_t stride = work * (kMxThreads / 16);
    // whole warps go round together: the last round's idle half takes part in the exchanges with zeros
    for (uint32_t first = u & ~1u; first < total; first += stride, u += stride) {
        MxTwo<T> v[STRIP][4];
        const uint32_t g0 = strip * STRIP, at = g0 * kMxGroup + sub * 8;
        const T* const row = x + (size_t)r * pitch;
        const bool there = u < total;
#pragma unroll
        for (int j = 0; j < STRIP; ++j) {
            const uint32_t here = at + j * kMxGroup;
            if (there && here < cols) load8<T, VEC>(row, here, cols, v[j]);
            else {
#pragma unroll
                for (int i = 0; i < 4; ++i) v[j][i] = MxTwo<T>{};
            }
        }
        uint32_t* const out = codes + ((size_t)r * blocks + (at >> 5)) * 4 + (sub & 3u);
        unsigned char* const scale = scales + mx_scale_at(r, g0, groups);
#pragma unroll
        for (int j = 0; j < STRIP; ++j) {
            uint32_t s;
            const uint32_t w = quantize_block(v[j], s);
            if (there && (at >> 5) + 4 * j < blocks) out[16 * j] = w;
            if ((sub & 3u) == 0 && there && g0 + j < groups) scale[j * kMxTileBytes + (sub >> 2)] = (unsigned char)s;
        }
        r += step_row;
        strip += step_strip;
        if (strip >= strips) { strip -= strips; ++r; }
    }
}

// Columns: the form of the transpose.  A warp takes a block of 32 rows x 64 columns (a lane two columns, so a row's load is one line
// of 16-bit elements): a lane holds whole blocks and needs no exchange.  A CTA's eight blocks go through shared memory, so that they leave as lines of
// 128 bytes and words of scales.
constexpr int kColumnWarps = 8, kColumnWidth = 64;
constexpr int kColumnPad = kColumnWarps + 1;   // sixteen-byte pieces of a column in shared memory: an odd number keeps the writes of eight lanes apart
struct ColumnsShared {
    uint4 codes[kColumnWidth][kColumnPad];
    __align__(8) unsigned char scales[kColumnWidth][kColumnWarps];
};
template <class T, bool VEC>
__device__ __forceinline__ void quantize_columns(const MxJob& job, uint32_t cta, ColumnsShared& sh)
{
    const T* const x = (const T*)job.x;
    const uint32_t rows = job.rows, cols = job.cols, blocks = job.blocks, groups = job.groups, across = job.across;
    const size_t pitch = job.pitch;
    uint4* __restrict__ const codes = (uint4*)job.codes;
    unsigned char* __restrict__ const scales = job.scales;
    auto& sh_codes = sh.codes;
    auto& sh_scales = sh.scales;
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31u;
    const uint32_t band = cta / across, c0 = (cta - band * across) * kColumnWidth;
    const uint32_t c = c0 + lane * 2, b = band * kColumnWarps + warp, r0 = b * kMxBlock;
    MxTwo<T> v[kMxBlock];
    if (VEC && c0 + kColumnWidth <= cols && r0 + kMxBlock <= rows) {
        const T* p = x + (size_t)r0 * pitch + c;
#pragma unroll
        for (int i = 0; i < kMxBlock; ++i, p += pitch) v[i] = *reinterpret_cast<const MxTwo<T>*>(p);
    } else {
#pragma unroll
        for (int i = 0; i < kMxBlock; ++i) {
            const T* p = x + (size_t)(r0 + i) * pitch + c;
            T e[2] = {mx_round<T>(0.0f), mx_round<T>(0.0f)};
            if (r0 + i < rows) {
                if (c < cols) e[0] = p[0];
                if (c + 1 < cols) e[1] = p[1];
            }
            v[i] = *reinterpret_cast<const MxTwo<T>*>(e);
        }
    }
    MxTop<T> top;
#pragma unroll
    for (int i = 0; i < kMxBlock; ++i) mx_top(top, v[i]);
    const uint32_t s0 = mx_exponent(mx_first(top)), s1 = mx_exponent(mx_second(top));
    const float i0 = mx_inverse(s0), i1 = mx_inverse(s1);
    const uint32_t both = mx_pair(i0, i1);
    uint32_t w0[4], w1[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        float f0[8], f1[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) mx_scaled(v[8 * q + i], i0, i1, both, f0[i], f1[i]);
        w0[q] = s0 == 255u ? 0u : mx_encode8(f0);
        w1[q] = s1 == 255u ? 0u : mx_encode8(f1);
    }
    sh_codes[lane * 2][warp] = make_uint4(w0[0], w0[1], w0[2], w0[3]);
    sh_codes[lane * 2 + 1][warp] = make_uint4(w1[0], w1[1], w1[2], w1[3]);
    sh_scales[lane * 2][warp] = (unsigned char)s0;
    sh_scales[lane * 2 + 1][warp] = (unsigned char)s1;
    __syncthreads();
    const uint32_t b0 = band * kColumnWarps;
#pragma unroll
    for (int i = 0; i < kColumnWidth / 32; ++i) {
        const uint32_t column = (threadIdx.x >> 3) + 32 * i, piece = threadIdx.x & 7u;
        if (c0 + column < cols && b0 + piece < blocks) codes[(size_t)(c0 + column) * blocks + b0 + piece] = sh_codes[column][piece];
    }
    if (threadIdx.x < 2 * kColumnWidth) {
        const uint32_t column = threadIdx.x >> 1, half = threadIdx.x & 1u, g = band * 2 + half;
        if (g < groups) *reinterpret_cast<uint32_t*>(scales + mx_scale_at(c0 + column, g, groups)) = *reinterpret_cast<const uint32_t*>(&sh_scales[column][4 * half]);
    }
}

template <class T, MxKind KIND>
__device__ __forceinline__ void quantize_one(const MxJob& job, uint32_t cta, ColumnsShared& sh)
{
    if constexpr (KIND == kMxRowsStrips) quantize_rows<T, true, 4>(job, cta);
    else if constexpr (KIND == kMxRows) quantize_rows<T, true, 1>(job, cta);
    else if constexpr (KIND == kMxRowsPlain) quantize_rows<T, false, 4>(job, cta);
    else if constexpr (KIND == kMxColumns) quantize_columns<T, true>(job, cta, sh);
    else quantize_columns<T, false>(job, cta, sh);
}
// CTAs that an SM is to hold, which is what registers a kernel may have.  Columns wait for memory, so where there are many CTAs as many are resident as a
// few spilled registers buy: with whole pairs of 16-bit elements four (8192 x 8192 bf16: 26.4 us; three 28.1, two 34.1), otherwise three (16384 x 4097 bf16: 42.9 us;
// four 63.3, two 55.5).  Where all are resident at two to an SM anyhow nothing is spilled (777 x 1000: 3.0 us, with four 5.8).  Rows need half the registers.
template <class T, MxKind KIND>
constexpr int ctas_of(bool many) { return KIND < kMxColumns ? (sizeof(T) == 2 ? 6 : 4) : !many ? 2 : KIND == kMxColumns && sizeof(T) == 2 ? 4 : 3; }

// One matrix: a kernel for each way.
template <class T, MxKind KIND, bool MANY>
__global__ void __launch_bounds__(kMxThreads, ctas_of<T, KIND>(MANY)) mx_quantize_kernel(const __grid_constant__ MxJob job)
{
    __shared__ ColumnsShared sh;
    pdl_enter();
    quantize_one<T, KIND>(job, blockIdx.x, sh);
}
// Several: the small ones of a layer would each take as long as a launch.  With rows alone a kernel that knows no columns, since two CTAs' worth of
// registers would be too few warps for them (two of 4096 x 4096 bf16: 29 us at two CTAs to an SM, 19 at four).
enum MxMix { kMxRowsAlone, kMxFewColumns, kMxManyColumns };
template <class T, MxMix MIX>
__global__ void __launch_bounds__(kMxThreads, MIX == kMxRowsAlone ? ctas_of<T, kMxRows>(true) : ctas_of<T, kMxColumns>(MIX == kMxManyColumns))
mx_quantize_all_kernel(const __grid_constant__ MxJobs jobs)
{
    __shared__ ColumnsShared sh;
    pdl_enter();
    int i = 0;
    while (i + 1 < jobs.count && jobs.job[i + 1].first <= blockIdx.x) ++i;
    const MxJob& job = jobs.job[i];
    const uint32_t cta = blockIdx.x - job.first;
    switch (job.kind) {
        case kMxRowsStrips: quantize_one<T, kMxRowsStrips>(job, cta, sh); break;
        case kMxRows: quantize_one<T, kMxRows>(job, cta, sh); break;
        case kMxRowsPlain: quantize_one<T, kMxRowsPlain>(job, cta, sh); break;
        default:
            if constexpr (MIX != kMxRowsAlone) {
                if (job.kind == kMxColumns) quantize_one<T, kMxColumns>(job, cta, sh);
                else quantize_one<T, kMxColumnsPlain>(job, cta, sh);
            }
    }
}

// Back: 16 lanes take STRIP runs of 128 neighbouring elements of a row, a lane as many as make 16 bytes of the output at a time, so a store of the
// 16 lanes is one run of whole sectors.  Rows that begin on 16 bytes (WIDE) have their runs begin there; elsewhere runs begin at the row's first 16-byte
// boundary, `head` elements in, and a lane's elements are cut out of two words of codes and may lie in two blocks; the head and the end are stored one by one
// (16384 x 4097 bf16: 52 us against 73.6 us one by one; 8192 x 8192, on boundaries: 27.5 us, 6.2 TB/s).
template <class T, bool WIDE, int STRIP>
__global__ void __launch_bounds__(kMxThreads) mx_dequantize_kernel(const uint32_t* codes, const unsigned char* scales, uint32_t rows,
                                                                    uint32_t cols, uint32_t blocks, uint32_t groups, uint32_t strips, uint32_t total, uint32_t step_row,
                                                                    uint32_t step_strip, T* __restrict__ y, size_t pitch)
{
    pdl_enter();
    constexpr uint32_t kPer = 16 / sizeof(T), kTurns = kMxGroup / 16 / kPer;     // elements of a lane at a time, and how often to a run
    const uint32_t sub = threadIdx.x & 15u;
    uint32_t u = blockIdx.x * (kMxThreads / 16) + (threadIdx.x >> 4);
    uint32_t r = u / strips, strip = u - r * strips;
    const uint32_t stride = gridDim.x * (kMxThreads / 16);
    for (; u < total; u += stride) {
        T* const row = y + (size_t)r * pitch;
        const uint32_t* const in = codes + (size_t)r * blocks * 4;
        const auto scale_at = [&](uint32_t block) { return scales[mx_scale_at(r, block >> 2, groups) + (block & 3u)]; };
        const uint32_t head = WIDE ? 0u : (16u - (uint32_t)((uintptr_t)row & 15u)) % 16u / (uint32_t)sizeof(T);
        const uint32_t from = head + strip * STRIP * kMxGroup + sub * kPer;
        uint32_t w[STRIP * kTurns], s[STRIP * kTurns], s2[WIDE ? 1 : STRIP * kTurns];
#pragma unroll
        for (int j = 0; j < STRIP * (int)kTurns; ++j) {
            const uint32_t at = from + j * 16 * kPer;
            if (at < cols) {
                w[j] = __ldcs(in + (at >> 3));
                s[j] = scale_at(at >> 5);
                if (!WIDE) {
                    const uint32_t next = (at >> 3) + 1, last = min(at + kPer - 1, cols - 1);
                    w[j] = __funnelshift_r(w[j], next < blocks * 4 ? in[next] : 0u, 4 * (at & 7u));
                    s2[j] = last >> 5 == at >> 5 ? s[j] : scale_at(last >> 5);
                } else if (kPer == 4) w[j] >>= 4 * (at & 7u);
            }
        }
#pragma unroll
        for (int j = 0; j < STRIP * (int)kTurns; ++j) {
            const uint32_t at = from + j * 16 * kPer;
            if (at >= cols) break;
            float v[8];
            if constexpr (kPer == 8) mx_decode8(w[j], v);
            else {
                // with half of its results unused, mx_decode8's unpacking came out wrong (the other half's) from this compiler
#pragma unroll
                for (int q = 0; q < 4; ++q) v[q] = mx_decode1(w[j] >> (4 * q) & 15u);
            }
            const float first = mx_scale(s[j]), second = WIDE ? first : mx_scale(s2[j]);
            MxPack<T> p;
#pragma unroll
            for (int q = 0; q < (int)kPer; ++q) p.v[q] = mx_round<T>(v[q] * (WIDE || (at & 31u) + q < 32u ? first : second));
            if (at + kPer <= cols) *reinterpret_cast<uint4*>(row + at) = *reinterpret_cast<const uint4*>(&p);
            else {
#pragma unroll
                for (int q = 0; q < (int)kPer; ++q)
                    if (at + q < cols) row[at + q] = p.v[q];
            }
        }
        if (!WIDE && strip == 0 && sub < min(head, cols)) row[sub] = mx_round<T>(mx_decode1(in[0] >> (4 * sub) & 15u) * mx_scale(scale_at(0)));
        r += step_row;
        strip += step_strip;
        if (strip >= strips) { strip -= strips; ++r; }
    }
}

struct Rounds {
    uint32_t strips, total;
    unsigned ctas;
    uint32_t step_row, step_strip;
};
// Strips of a row, as many CTAs as there is work for (at most 2^16), and how far (row, strip) moves from round to round.
Rounds rounds_of(size_t rows, size_t groups, int strip)
{
    const size_t per = kMxThreads / 16, strips = (groups + strip - 1) / strip, total = rows * strips;
    const unsigned ctas = (unsigned)std::min((total + per - 1) / per, (size_t)1 << 16);
    const uint32_t stride = ctas * (uint32_t)per;
    return {(uint32_t)strips, (uint32_t)total, ctas, stride / (uint32_t)strips, stride % (uint32_t)strips};
}
// Strips of four groups where a row has that many and there are enough of them for all SMs; else of one.
constexpr size_t kStripWork = 1 << 15;
bool strips_pay(size_t rows, size_t groups) { return groups >= 4 && rows * groups >= kStripWork; }

int launched(cudaError_t e)
{
    if (e == cudaSuccess) count_launches(1);
    return e == cudaSuccess ? ZCCL_OK : ZCCL_E_CUDA;
}
// How a matrix is gone about; returns its CTAs (0: more than can be counted).
unsigned plan(const zccl_mx4_job& j, size_t element, MxJob& to)
{
    const uintptr_t at = (uintptr_t)j.x;
    to = MxJob{};
    to.x = j.x;
    to.codes = j.codes;
    to.scales = (unsigned char*)j.scales;
    to.pitch = j.pitch;
    to.rows = (uint32_t)j.rows;
    to.cols = (uint32_t)j.cols;
    const size_t along = j.transpose ? j.rows : j.cols, groups = mx_groups(along);
    to.blocks = (uint32_t)mx_blocks(along);
    to.groups = (uint32_t)groups;
    if (j.transpose) {
        const size_t across = mx_bands(j.cols) * (kMxBand / kColumnWidth), ctas = (to.blocks + kColumnWarps - 1) / kColumnWarps * across;
        to.across = (uint32_t)across;
        to.kind = at % (2 * element) == 0 && j.pitch % 2 == 0 ? kMxColumns : kMxColumnsPlain;
        return ctas > kMxMaxGroups ? 0u : (unsigned)ctas;
    }
    if (mx_bands(j.rows) * kMxBand * groups > kMxMaxGroups) return 0u;
    to.kind = at % 16 || j.pitch * element % 16 ? kMxRowsPlain : strips_pay(j.rows, groups) ? kMxRowsStrips : kMxRows;
    const Rounds k = rounds_of(j.rows, groups, to.kind == kMxRows ? 1 : 4);
    to.strips = k.strips;
    to.total = k.total;
    to.work = k.ctas;
    to.step_row = k.step_row;
    to.step_strip = k.step_strip;
    return k.ctas + (unsigned)(((mx_bands(j.rows) * kMxBand - j.rows) * groups + kMxThreads - 1) / kMxThreads);
}
template <class T>
int quantize_all(const zccl_mx4_job* jobs, int count, cudaStream_t st)
{
    MxJobs list;
    for (int i = 0; i < count; ++i)     // before anything runs
        if (jobs[i].rows && jobs[i].cols && plan(jobs[i], sizeof(T), list.job[0]) == 0) return ZCCL_E_ARG;
    for (int at = 0; at < count;) {
        unsigned ctas = 0, columns = 0;
        list.count = 0;
        for (; at < count && list.count < kMxJobs; ++at) {
            if (jobs[at].rows == 0 || jobs[at].cols == 0) continue;
            MxJob& job = list.job[list.count];
            const unsigned mine = plan(jobs[at], sizeof(T), job);
            if (ctas > kMxMaxGroups - mine) break;
            job.first = ctas;
            ctas += mine;
            if (job.kind >= kMxColumns) columns += mine;
            ++list.count;
        }
        if (list.count == 0) continue;
        int dev = 0, sms = 0;
        if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return ZCCL_E_CUDA;
        int rc;
        const bool many = columns > (list.count > 1 ? 1u : 2u) * (unsigned)sms;   // several: rows' CTAs want room too
        if (list.count > 1)
            rc = launched(launch_k(columns == 0 ? mx_quantize_all_kernel<T, kMxRowsAlone> : many ? mx_quantize_all_kernel<T, kMxManyColumns> : mx_quantize_all_kernel<T, kMxFewColumns>,
                                   dim3(ctas), dim3(kMxThreads), 0, st, list));
        else {
            const MxKind kind = list.job[0].kind;
            const auto kernel = kind == kMxRowsStrips ? mx_quantize_kernel<T, kMxRowsStrips, true> : kind == kMxRows ? mx_quantize_kernel<T, kMxRows, true>
                                : kind == kMxRowsPlain ? mx_quantize_kernel<T, kMxRowsPlain, true>
                                : kind == kMxColumns ? (many ? mx_quantize_kernel<T, kMxColumns, true> : mx_quantize_kernel<T, kMxColumns, false>)
                                                     : (many ? mx_quantize_kernel<T, kMxColumnsPlain, true> : mx_quantize_kernel<T, kMxColumnsPlain, false>);
            rc = launched(launch_k(kernel, dim3(ctas), dim3(kMxThreads), 0, st, list.job[0]));
        }
        if (rc != ZCCL_OK) return rc;
    }
    return ZCCL_OK;
}

template <class T, bool VEC>
cudaError_t launch_back(const void* codes, const void* scales, size_t rows, size_t cols, T* y, size_t pitch, cudaStream_t st)
{
    const size_t blocks = mx_blocks(cols), groups = mx_groups(cols);
    constexpr int kStrip = VEC && sizeof(T) == 2 ? 4 : 2;   // the others hold more for each run (8192 x 8192 to f32: 50.6 us, with four 55.2)
    const bool many = strips_pay(rows, groups);
    const Rounds k = rounds_of(rows, groups, many ? kStrip : 1);
    return launch_k(many ? mx_dequantize_kernel<T, VEC, kStrip> : mx_dequantize_kernel<T, VEC, 1>, dim3(k.ctas), dim3(kMxThreads), 0, st, (const uint32_t*)codes,
                    (const unsigned char*)scales, (uint32_t)rows, (uint32_t)cols, (uint32_t)blocks, (uint32_t)groups, k.strips, k.total, k.step_row, k.step_strip, y, pitch);
}

template <class T>
int dequantize(const void* codes, const void* scales, size_t rows, size_t cols, T* y, size_t pitch, cudaStream_t st)
{
    if (rows * mx_groups(cols) > kMxMaxGroups) return ZCCL_E_ARG;
    const bool vec = (uintptr_t)y % 16 == 0 && pitch * sizeof(T) % 16 == 0;
    const cudaError_t e = vec ? launch_back<T, true>(codes, scales, rows, cols, y, pitch, st) : launch_back<T, false>(codes, scales, rows, cols, y, pitch, st);
    return launched(e);
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

int zccl_mx4_quantize_all(const zccl_mx4_job* jobs, int count, int type, void* stream)
{
    if (count < 0 || (count && !jobs) || type < ZCCL_F32 || type > ZCCL_F16) return ZCCL_E_ARG;
    for (int i = 0; i < count; ++i)
        if (jobs[i].rows && jobs[i].cols && (!matrix_ok(jobs[i].x, type, jobs[i].rows, jobs[i].cols, jobs[i].pitch) || !aligned(jobs[i].codes, 16) || !aligned(jobs[i].scales, 16)))
            return ZCCL_E_ARG;
    cudaStream_t st = (cudaStream_t)stream;
    return type == ZCCL_F32 ? quantize_all<float>(jobs, count, st) : type == ZCCL_BF16 ? quantize_all<__nv_bfloat16>(jobs, count, st) : quantize_all<__half>(jobs, count, st);
}

int zccl_mx4_quantize(const void* x, int type, size_t rows, size_t cols, size_t pitch, int transpose, void* codes, void* scales, void* stream)
{
    const zccl_mx4_job job{x, rows, cols, pitch, transpose, codes, scales};
    return zccl_mx4_quantize_all(&job, 1, type, stream);
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
