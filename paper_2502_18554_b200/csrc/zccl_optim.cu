// The norm of all gradients and the AdamW step over many tensors at once, states in 32 or in 8 bits.
#include "../../include/zccl.h"
#include "zccl_mx4.cuh"

#include <algorithm>
#include <cfloat>
#include <cmath>

namespace zccl {
namespace {

constexpr int kOptThreads = 256;
constexpr int kPerThread = 8;                       // neighbouring elements of a thread: four threads hold a block of 32
constexpr int kPass = kOptThreads * kPerThread;
constexpr int kChunk = 4 * kPass;                   // elements of a gradient that a CTA takes the norm of at a time
constexpr int kChunksWanted = 1024;                 // of a step, before they get longer
// Tensors travel as kernel arguments, so a call copies nothing, needs no memory and can be captured.  Arguments above 4 KB cost
// the launch a few microseconds, hence three sizes of the list (a step of 41 tensors 6.5 us on the host, with two sizes 11.4; of 100 12.6 and 14.5).
constexpr int kFewTensors = 40, kMoreTensors = 128, kManyTensors = 360;

// Which tensor chunk `c` belongs to: the last one that begins at or in front of it (tensors without elements have no chunks).
template <class L>
__device__ __forceinline__ int tensor_of(const L& list, uint32_t c)
{
    int lo = 0, hi = list.count;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (list.first[mid] <= c) lo = mid; else hi = mid;
    }
    return lo;
}

template <class T>
__device__ __forceinline__ bool wide(const T* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// Eight neighbouring elements as they are in memory.
template <class T> struct Eight { uint4 w[sizeof(T) / 2]; };

template <class T>
__device__ __forceinline__ Eight<T> load_wide(const T* p)
{
    Eight<T> e;
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) e.w[i] = __ldcs(reinterpret_cast<const uint4*>(p) + i);
    return e;
}
__device__ __forceinline__ void values_of(const Eight<float>& e, float (&v)[8])
{
    const uint32_t w[8] = {e.w[0].x, e.w[0].y, e.w[0].z, e.w[0].w, e.w[1].x, e.w[1].y, e.w[1].z, e.w[1].w};
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(w[i]);
}
__device__ __forceinline__ void values_of(const Eight<__nv_bfloat16>& e, float (&v)[8])
{
    const uint32_t w[4] = {e.w[0].x, e.w[0].y, e.w[0].z, e.w[0].w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
}
__device__ __forceinline__ void two_halves(uint32_t w, float& a, float& b)
{
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w));
    a = f.x;
    b = f.y;
}
__device__ __forceinline__ void values_of(const Eight<__half>& e, float (&v)[8])
{
    const uint32_t w[4] = {e.w[0].x, e.w[0].y, e.w[0].z, e.w[0].w};
#pragma unroll
    for (int i = 0; i < 4; ++i) two_halves(w[i], v[2 * i], v[2 * i + 1]);
}
__device__ __forceinline__ uint32_t two_of(float a, float b, __nv_bfloat16)
{
    const __nv_bfloat162 p = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&p);
}
__device__ __forceinline__ uint32_t two_of(float a, float b, __half)
{
    const __half2 p = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&p);
}
template <class T>
__device__ __forceinline__ void store_wide(T* p, const float (&v)[8])
{
    uint4* const out = reinterpret_cast<uint4*>(p);
    if constexpr (sizeof(T) == 4) {
        __stcs(out, make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])));
        __stcs(out + 1, make_uint4(__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7])));
    } else __stcs(out, make_uint4(two_of(v[0], v[1], T()), two_of(v[2], v[3], T()), two_of(v[4], v[5], T()), two_of(v[6], v[7], T())));
}
// `full`: all eight are there and the array begins on a 16-byte boundary; else the first `left` ones are read.
template <class T>
__device__ __forceinline__ void read8(const T* p, bool full, int left, float (&v)[8])
{
    if (full) values_of(load_wide(p), v);
    else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < left ? mx_float(p[i]) : 0.0f;
    }
}
template <class T>
__device__ __forceinline__ void write8(T* p, bool full, int left, const float (&v)[8])
{
    if (full) store_wide(p, v);
    else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < left) p[i] = mx_round<T>(v[i]);
    }
}

// ------------------------------------------------------------------------------------------------ norm

constexpr int kNormCtas = 1024;   // partial sums of a launch

template <int CAP>
struct NormList {
    const void* g[CAP];
    unsigned long long n[CAP];
    uint32_t first[CAP];
    uint32_t chunks;
    int count;
};

__device__ __forceinline__ double block_sum(double s)
{
    __shared__ double part[kOptThreads / 32];
#pragma unroll
    for (int d = 16; d; d >>= 1) s += __shfl_xor_sync(kFull, s, d);
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = s;
    __syncthreads();
    s = 0.0;
    for (int i = 0; i < kOptThreads / 32; ++i) s += part[i];
    __syncthreads();
    return s;
}

// A thread squares and adds the eight elements that it holds in binary32 and all that follows in binary64: converting every element
// would cost the double-precision units more than the memory has time for.  Where the eight's sum may have left the range
// of binary32 it is taken again in binary64.
__device__ __forceinline__ double squares_of(const float (&v)[8])
{
    float s = 0.0f;
#pragma unroll
    for (int j = 0; j < 8; ++j) s = __fmaf_rn(v[j], v[j], s);
    if (s > 1e-24f && s < 1e37f) return (double)s;
    double d = 0.0;
    for (int j = 0; j < 8; ++j) d += (double)v[j] * (double)v[j];
    return d;
}
// `norm`: given to a launch of one CTA that has everything; else the sums of all CTAs are left to norm_join_kernel.
template <class G, int CAP>
__global__ void __launch_bounds__(kOptThreads) norm_parts_kernel(const __grid_constant__ NormList<CAP> list, double* __restrict__ parts, float* __restrict__ norm)
{
    pdl_enter();
    double sum = 0.0;
    for (uint32_t c = blockIdx.x; c < list.chunks; c += gridDim.x) {
        const int t = tensor_of(list, c);
        const unsigned long long n = list.n[t], begin = (unsigned long long)(c - list.first[t]) * kChunk;
        const G* g = (const G*)list.g[t] + begin;
        const bool aligned = wide((const G*)list.g[t]);
        const int left_all = (int)min((unsigned long long)kChunk, n - begin);
        if (aligned && left_all == kChunk) {
            Eight<G> e[kChunk / kPass];
#pragma unroll
            for (int i = 0; i < kChunk / kPass; ++i) e[i] = load_wide(g + i * kPass + threadIdx.x * kPerThread);
#pragma unroll
            for (int i = 0; i < kChunk / kPass; ++i) {
                float v[8];
                values_of(e[i], v);
                sum += squares_of(v);
            }
        } else {
            for (int at = threadIdx.x * kPerThread; at < left_all; at += kPass) {
                float v[8];
                read8(g + at, aligned && left_all - at >= 8, left_all - at, v);
                sum += squares_of(v);
            }
        }
    }
    sum = block_sum(sum);
    if (threadIdx.x == 0) {
        if (norm) *norm = (float)sqrt(sum);
        else parts[blockIdx.x] = sum;
    }
}

__global__ void __launch_bounds__(kOptThreads) norm_join_kernel(const double* parts, uint32_t count, float* norm)
{
    pdl_enter();
    double sum = 0.0;
    for (uint32_t i = threadIdx.x; i < count; i += kOptThreads) sum += parts[i];
    sum = block_sum(sum);
    if (threadIdx.x == 0) *norm = (float)sqrt(sum);
}

// ------------------------------------------------------------------------------------------------ AdamW

struct AdamTensor {
    void* p;
    const void* g;
    void *m, *v;
    unsigned char *m_scale, *v_scale;
    void* copy;
    unsigned long long n, place;   // `place`: its first element in the order that the random bits go by
    bool wide;                     // all arrays begin on 16-byte boundaries
};
template <int CAP>
struct AdamList {
    AdamTensor t[CAP];
    uint32_t first[CAP];
    int count;
};

struct AdamCall {
    float beta1, rest1, beta2, eps;
    // Square roots of beta2 and of 1 - beta2: a square of a product for two products.  Each is rounded to binary32 and squared, up to 2^-23 of beta2 and of 1 - beta2.
    float root_beta2, root_rest2;
    float keep, rate, root;        // 1 - lr weight_decay; lr / (1 - beta1^step); 1 / sqrt(1 - beta2^step)
    double lr, weight_decay, log_beta1, log_beta2;   // where step or lr is on the device
    const long long* step;
    const float* lr_device;
    long long step_host;
    unsigned long long seed;
    const float* norm;
    float max_norm;
    int copy_type;
    uint32_t passes;               // of 2048 elements to a chunk
};

__host__ __device__ inline unsigned long long random_key(unsigned long long seed, long long step)
{
    return seed + (unsigned long long)step * 0x9E3779B97F4A7C15ull;
}
// 32 random bits h for the element at `place`: three rounds of multiplying and folding the upper bits down, the last fold left to noise_of.  The shape, and the first two multipliers,
// are those of the 32-bit integer hash that Wellons published as the least biased of a search (Prospecting for hash functions, 2018); random_key steps by
// 2^64 over the golden ratio, as Weyl sequences do (Steele, Lea and Flood, 2014).
// `low` is the lower half of place ^ key, `high` the upper half of place ^ key.
__device__ __forceinline__ uint32_t random_bits(uint32_t low, uint32_t high)
{
    uint32_t h = low * 0x7FEB352Du;
    h = ((h ^ (h >> 15)) ^ high) * 0x846CA68Bu;
    return (h ^ (h >> 13)) * 0x6C8E9CF5u;
}
// The upper 16 of the bits h ^ (h >> 16), and the lower 16, each in bits 8 ... 23.
__device__ __forceinline__ void noise_of(uint32_t h, uint32_t& first, uint32_t& second)
{
    first = prmt(h, 0, 0x4324);
    second = prmt(h, 0, 0x4104) ^ first;
}

// Two neighbours as one operand: the multiplications and additions of two elements are one instruction, each rounded as it would be alone.
struct Two { unsigned long long w; };
__device__ __forceinline__ Two two(float a, float b)
{
    Two t;
    asm("mov.b64 %0, {%1, %2};" : "=l"(t.w) : "f"(a), "f"(b));
    return t;
}
__device__ __forceinline__ void both(Two t, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(t.w)); }
__device__ __forceinline__ Two times(Two a, Two b)
{
    Two t;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(t.w) : "l"(a.w), "l"(b.w));
    return t;
}
__device__ __forceinline__ Two times_plus(Two a, Two b, Two c)
{
    Two t;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(t.w) : "l"(a.w), "l"(b.w), "l"(c.w));
    return t;
}
// The largest of three, NaN where one of them is.
__device__ __forceinline__ float largest(float a, float b, float c)
{
    float d;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}

// The largest magnitude of a block, as bits, of which four neighbouring lanes hold eight each.
__device__ __forceinline__ uint32_t top8(const float (&v)[8])
{
    const float t = largest(fabsf(v[0]), fabsf(v[1]), fabsf(v[2]));
    const float u = largest(fabsf(v[3]), fabsf(v[4]), fabsf(v[5]));
    uint32_t top = __float_as_uint(largest(t, u, largest(fabsf(v[6]), fabsf(v[7]), 0.0f)));
    top = max(top, __shfl_xor_sync(kFull, top, 1));
    return max(top, __shfl_xor_sync(kFull, top, 2));
}
// The biased exponent at which the block's largest magnitude is at most 448 = 1.75 * 2^8; 255 where it is not finite.
__device__ __forceinline__ uint32_t exponent8(uint32_t top)
{
    const int field = (int)(top >> 23);
    return field == 255 ? 255u : (uint32_t)max(field - 8 + ((top & 0x7FFFFFu) > 0x600000u ? 1 : 0), 0);
}
// Eight codes as the numbers that E4M3 gives them (without the block's scale).
__device__ __forceinline__ void decode8(uint2 w, float (&v)[8])
{
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        uint32_t a, b;
        asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, l;\n\tcvt.rn.f16x2.e4m3x2 %1, h;\n\t}" : "=r"(a), "=r"(b) : "r"(i ? w.y : w.x));
        two_halves(a, v[4 * i], v[4 * i + 1]);
        two_halves(b, v[4 * i + 2], v[4 * i + 3]);
    }
}
__device__ __forceinline__ uint2 read_codes(const unsigned char* p, bool full, int left)
{
    if (full) return __ldcs(reinterpret_cast<const uint2*>(p));
    uint32_t w[2] = {0, 0};
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < left) w[i >> 2] |= (uint32_t)p[i] << (8 * (i & 3));
    return make_uint2(w[0], w[1]);
}
__device__ __forceinline__ void write_codes(unsigned char* p, bool full, int left, uint2 w)
{
    if (full) __stcs(reinterpret_cast<uint2*>(p), w);
    else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < left) p[i] = (unsigned char)((i & 4 ? w.y : w.x) >> (8 * (i & 3)));
    }
}
// Eight elements of a block to codes with the block's biased exponent s.  Times 2^-120 a magnitude's bits in binary32 are E4M3's, 20 places further
// up, subnormal numbers of the one among those of the other, so rounding is one addition below the last bit that is kept: `noise` has its
// 16 random bits in bits 8 ... 23, the magnitude is moved up by four to meet them, and the code is the top byte.
template <bool ROOT>
__device__ __forceinline__ uint2 pack8(float (&v)[8], const uint32_t (&noise)[8], uint32_t s)
{
    if (s > 133u) {                                  // 2^-e 2^-120 would be no normal number: in two steps
        const float down = __uint_as_float((254u - min(s, 253u)) << 23);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] *= down;
        if (s == 255u) return make_uint2(0x7F7F7F7Fu, 0x7F7F7F7Fu);
        s = 127u;
    }
    const float inverse = __uint_as_float((134u - s) << 23);
    uint32_t z[8], least = 0xFFFFFFFFu;
    float scaled[8];
#pragma unroll
    for (int i = 0; i < 8; i += 2) both(times(two(v[i], v[i + 1]), two(inverse, inverse)), scaled[i], scaled[i + 1]);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t bits = __float_as_uint(scaled[i]);
        z[i] = (bits << 4) + noise[i];
        if (ROOT) least = min(least, z[i]);
        else z[i] |= bits & 0x80000000u;
    }
    if (ROOT && least < 0x01000000u) {
#pragma unroll
        for (int i = 0; i < 8; ++i) z[i] = max(z[i], v[i] > 0.0f ? 0x01000000u : 0u);
    }
    return make_uint2(prmt(prmt(z[0], z[1], 0x0073), prmt(z[2], z[3], 0x0073), 0x5410), prmt(prmt(z[4], z[5], 0x0073), prmt(z[6], z[7], 0x0073), 0x5410));
}

// Both to within 2^-22.  A root of a subnormal number is taken of it as it is (gradients of 1e-19 square to these); no root is subnormal itself and zccl_adamw takes no eps that is, so
// no quotient is by one: its reciprocal would be infinite, and 0 times that NaN.
__device__ __forceinline__ float root_of(float v)
{
    float r;
    asm("sqrt.approx.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}
__device__ __forceinline__ float reciprocal_of(float v)
{
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}

// What a step does to an element, with everything that does not depend on it worked out before.
struct AdamRates {
    float keep, rate, root;        // see AdamCall
    float gain1, gain2;            // what a gradient enters m with, and the root of what its square enters v with (clipping included)
    unsigned long long key;
};

template <bool EIGHT>
__device__ __forceinline__ void update8(const AdamCall& call, const AdamRates& k, float m_unit, float v_unit, const float (&g)[8], float (&p)[8], float (&m)[8], float (&v)[8], float (&r)[8])
{
    const Two gain1 = two(k.gain1, k.gain1), gain2 = two(k.gain2, k.gain2), m_units = two(m_unit, m_unit), v_units = two(v_unit, v_unit);
    const Two root = two(k.root, k.root), eps = two(call.eps, call.eps), keep = two(k.keep, k.keep), rate = two(-k.rate, -k.rate);
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
        const Two gi = two(g[i], g[i + 1]), u = times(gain2, gi), w = times(v_units, two(v[i], v[i + 1]));
        const Two mi = times_plus(gain1, gi, times(m_units, two(m[i], m[i + 1])));
        both(mi, m[i], m[i + 1]);
        both(times_plus(u, u, EIGHT ? times(w, w) : w), v[i], v[i + 1]);
        r[i] = root_of(v[i]);
        r[i + 1] = root_of(v[i + 1]);
        float d0, d1;
        both(times_plus(two(r[i], r[i + 1]), root, eps), d0, d1);
        both(times_plus(rate, times(mi, two(reciprocal_of(d0), reciprocal_of(d1))), times(two(p[i], p[i + 1]), keep)), p[i], p[i + 1]);
    }
}
// New states of eight elements to codes; `place` counts the first one.
__device__ __forceinline__ void encode_states(const AdamRates& k, unsigned long long place, float (&m)[8], float (&r)[8], uint2& mc, uint2& vc, uint32_t& ms, uint32_t& vs)
{
    const unsigned long long from = place ^ k.key;   // `place` is a multiple of 8: element i changes the lowest bits alone
    uint32_t first[8], second[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) noise_of(random_bits((uint32_t)from ^ i, (uint32_t)(from >> 32)), first[i], second[i]);
    ms = exponent8(top8(m));
    vs = exponent8(top8(r));
    mc = pack8<false>(m, first, ms);
    vc = pack8<true>(r, second, vs);
}

// A CTA takes a chunk of `passes` times 2048 elements of one tensor, a thread eight neighbours at a time.  Passes that are whole, of arrays on
// 16-byte boundaries, go the short way, where the next eight are loaded while these are worked on.  States in 32 bits: bound by memory, two CTAs to an SM
// have enough loads in flight.  In 8 bits: about 50 instructions to an element against 10 bytes, so issue and memory take about as long and warps have
// to cover each other's waits: four CTAs, though for binary32 a few registers are spilled for it (128 Mi bf16 parameters as one tensor: 241 us; 261 us with every
// multiplication an instruction of its own, and of those 335 with two or three CTAs.  As 290 tensors 261 us, and 272 us in seconds of them on end, at the 1.79 GHz that power leaves).
// Sums fused and roots of the instruction's: of the 2^28 new codes of such a step 387 are off those of the definition in 64 bits (a value off by its last bit carries over, or does
// not, or is the block's largest next to a border of its scale); with every operation rounded by itself and IEEE roots 337, and the step takes 298 us instead of 279 us.
template <class P, class G, bool EIGHT, int CAP>
__global__ void __launch_bounds__(kOptThreads, EIGHT ? 4 : 2) adamw_kernel(const __grid_constant__ AdamList<CAP> list, const __grid_constant__ AdamCall call)
{
    pdl_enter();
    float clip = 1.0f;
    if (call.norm) {
        const float norm = *call.norm;
        if (!(norm >= 0.0f && norm < __int_as_float(0x7F800000))) return;   // no norm of finite gradients: no step
        clip = fminf(1.0f, __fdiv_rn(call.max_norm, norm + 1e-6f));
    }
    AdamRates k{call.keep, call.rate, call.root, call.rest1 * clip, call.root_rest2 * clip, random_key(call.seed, call.step_host)};
    if (call.step || call.lr_device) {
        __shared__ float sh[3];
        const long long step = call.step ? *call.step : call.step_host;
        k.key = random_key(call.seed, step);
        if (threadIdx.x == 0) {
            const double lr = call.lr_device ? (double)*call.lr_device : call.lr;
            sh[0] = (float)(1.0 - lr * call.weight_decay);
            sh[1] = (float)(lr / -expm1((double)step * call.log_beta1));
            sh[2] = (float)(1.0 / sqrt(-expm1((double)step * call.log_beta2)));
        }
        __syncthreads();
        k.keep = sh[0];
        k.rate = sh[1];
        k.root = sh[2];
    }
    const int t = tensor_of(list, blockIdx.x);
    const AdamTensor& a = list.t[t];
    const uint32_t chunk = call.passes * kPass;
    const unsigned long long begin = (unsigned long long)(blockIdx.x - list.first[t]) * chunk;
    const uint32_t mine = threadIdx.x * kPerThread;
    const int left_all = (int)min((unsigned long long)chunk, a.n - begin), whole = a.wide ? left_all / kPass : 0;   // passes that go the short way
    if (whole) {
        P* p = (P*)a.p + begin + mine;
        const G* g = (const G*)a.g + begin + mine;
        unsigned char* copy = a.copy ? (unsigned char*)a.copy + 2 * (begin + mine) : nullptr;
        unsigned long long place = a.place + begin + mine;
        Eight<P> pe = load_wide(p);
        Eight<G> ge = load_wide(g);
        if (EIGHT) {
            unsigned char *mc = (unsigned char*)a.m + begin + mine, *vc = (unsigned char*)a.v + begin + mine;
            unsigned char *ms = a.m_scale + (begin + mine) / kMxBlock, *vs = a.v_scale + (begin + mine) / kMxBlock;
            uint2 me = __ldcs(reinterpret_cast<const uint2*>(mc)), ve = __ldcs(reinterpret_cast<const uint2*>(vc));
            uint32_t mu = *ms, vu = *vs;
            for (int i = 1; i <= whole; ++i) {
                float pv[8], gv[8], mv[8], vv[8], rv[8];
                values_of(pe, pv);
                values_of(ge, gv);
                decode8(me, mv);
                decode8(ve, vv);
                const float m_unit = call.beta1 * mx_scale(mu), v_unit = call.root_beta2 * mx_scale(vu);
                if (i < whole) {
                    pe = load_wide(p + kPass);
                    ge = load_wide(g + kPass);
                    me = __ldcs(reinterpret_cast<const uint2*>(mc + kPass));
                    ve = __ldcs(reinterpret_cast<const uint2*>(vc + kPass));
                    mu = ms[kPass / kMxBlock];
                    vu = vs[kPass / kMxBlock];
                }
                update8<true>(call, k, m_unit, v_unit, gv, pv, mv, vv, rv);
                store_wide(p, pv);
                if (copy) {
                    if (call.copy_type == ZCCL_BF16) store_wide((__nv_bfloat16*)copy, pv);
                    else store_wide((__half*)copy, pv);
                    copy += 2 * kPass;
                }
                uint2 mw, vw;
                uint32_t se, re;
                encode_states(k, place, mv, rv, mw, vw, se, re);
                __stcs(reinterpret_cast<uint2*>(mc), mw);
                __stcs(reinterpret_cast<uint2*>(vc), vw);
                if ((threadIdx.x & 3) == 0) {
                    *ms = (unsigned char)se;
                    *vs = (unsigned char)re;
                }
                p += kPass; g += kPass; mc += kPass; vc += kPass; ms += kPass / kMxBlock; vs += kPass / kMxBlock; place += kPass;
            }
        } else {
            float *m = (float*)a.m + begin + mine, *v = (float*)a.v + begin + mine;
            Eight<float> me = load_wide(m), ve = load_wide(v);
            for (int i = 1; i <= whole; ++i) {
                float pv[8], gv[8], mv[8], vv[8], rv[8];
                values_of(pe, pv);
                values_of(ge, gv);
                values_of(me, mv);
                values_of(ve, vv);
                update8<false>(call, k, call.beta1, call.beta2, gv, pv, mv, vv, rv);
                if (i < whole) {
                    pe = load_wide(p + kPass);
                    ge = load_wide(g + kPass);
                    me = load_wide((const float*)m + kPass);
                    ve = load_wide((const float*)v + kPass);
                }
                store_wide(p, pv);
                if (copy) {
                    if (call.copy_type == ZCCL_BF16) store_wide((__nv_bfloat16*)copy, pv);
                    else store_wide((__half*)copy, pv);
                    copy += 2 * kPass;
                }
                store_wide(m, mv);
                store_wide(v, vv);
                p += kPass; g += kPass; m += kPass; v += kPass;
            }
        }
    }
    P* const p = (P*)a.p + begin;
    const G* const g = (const G*)a.g + begin;
    const bool p_wide = wide(p), g_wide = wide(g), copies = a.copy != nullptr, copy_wide = wide((const __half*)a.copy);
    for (int at = whole * kPass + (int)mine; at - (int)(threadIdx.x & 31) * kPerThread < left_all; at += kPass) {   // whole warps
        const int left = left_all - at;
        const bool all = left >= 8;
        float pv[8], gv[8], mv[8], vv[8], rv[8];
        read8(p + at, all && p_wide, left, pv);
        read8(g + at, all && g_wide, left, gv);
        unsigned char *mc = nullptr, *vc = nullptr, *ms = nullptr, *vs = nullptr;
        bool m_wide, v_wide;
        float m_unit = call.beta1, v_unit = call.beta2;
        if (EIGHT) {
            mc = (unsigned char*)a.m + begin + at;
            vc = (unsigned char*)a.v + begin + at;
            ms = a.m_scale + (begin + at) / kMxBlock;
            vs = a.v_scale + (begin + at) / kMxBlock;
            m_wide = all && ((uintptr_t)mc & 7u) == 0;
            v_wide = all && ((uintptr_t)vc & 7u) == 0;
            m_unit = call.beta1 * mx_scale(left > 0 ? *ms : 0u);
            v_unit = call.root_beta2 * mx_scale(left > 0 ? *vs : 0u);
            decode8(read_codes(mc, m_wide, left), mv);
            decode8(read_codes(vc, v_wide, left), vv);
        } else {
            m_wide = all && wide((float*)a.m);
            v_wide = all && wide((float*)a.v);
            read8((const float*)a.m + begin + at, m_wide, left, mv);
            read8((const float*)a.v + begin + at, v_wide, left, vv);
        }
        update8<EIGHT>(call, k, m_unit, v_unit, gv, pv, mv, vv, rv);
        write8(p + at, all && p_wide, left, pv);
        if (copies) {
            if (call.copy_type == ZCCL_BF16) write8((__nv_bfloat16*)a.copy + begin + at, all && copy_wide, left, pv);
            else write8((__half*)a.copy + begin + at, all && copy_wide, left, pv);
        }
        if (EIGHT) {
            if (!all) {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (i >= left) mv[i] = rv[i] = 0.0f;
            }
            uint2 mw, vw;
            uint32_t se, re;
            encode_states(k, a.place + begin + at, mv, rv, mw, vw, se, re);
            write_codes(mc, m_wide, left, mw);
            write_codes(vc, v_wide, left, vw);
            if ((threadIdx.x & 3) == 0 && left > 0) {
                *ms = (unsigned char)se;
                *vs = (unsigned char)re;
            }
        } else {
            write8((float*)a.m + begin + at, m_wide, left, mv);
            write8((float*)a.v + begin + at, v_wide, left, vv);
        }
    }
}

template <class P, class G, bool EIGHT, int CAP>
cudaError_t launch_adamw(const AdamList<CAP>& list, uint32_t chunks, const AdamCall& call, cudaStream_t st)
{
    return launch_k(adamw_kernel<P, G, EIGHT, CAP>, dim3(chunks), dim3(kOptThreads), 0, st, list, call);
}
template <class P, class G, int CAP>
cudaError_t launch_adamw_bits(int bits, const AdamList<CAP>& list, uint32_t chunks, const AdamCall& call, cudaStream_t st)
{
    return bits == 8 ? launch_adamw<P, G, true>(list, chunks, call, st) : launch_adamw<P, G, false>(list, chunks, call, st);
}
template <class P, int CAP>
cudaError_t launch_adamw_grad(const zccl_adamw_config& k, const AdamList<CAP>& list, uint32_t chunks, const AdamCall& call, cudaStream_t st)
{
    if (k.grad_type == ZCCL_F32) return launch_adamw_bits<P, float>(k.state_bits, list, chunks, call, st);
    if (k.grad_type == ZCCL_BF16) return launch_adamw_bits<P, __nv_bfloat16>(k.state_bits, list, chunks, call, st);
    return launch_adamw_bits<P, __half>(k.state_bits, list, chunks, call, st);
}
template <int CAP>
cudaError_t launch_adamw_param(const zccl_adamw_config& k, const AdamList<CAP>& list, uint32_t chunks, const AdamCall& call, cudaStream_t st)
{
    if (k.param_type == ZCCL_F32) return launch_adamw_grad<float>(k, list, chunks, call, st);
    if (k.param_type == ZCCL_BF16) return launch_adamw_grad<__nv_bfloat16>(k, list, chunks, call, st);
    return launch_adamw_grad<__half>(k, list, chunks, call, st);
}

constexpr size_t kMostElems = (size_t)1 << 42;   // of a tensor: chunks of a launch are counted in 31 bits
constexpr uint32_t kMostChunks = 0x7FFFFFFFu;

// The list of tensors from `at` on that one launch takes; returns how many entries of `tensors` that covers.
template <int CAP>
size_t fill_list(AdamList<CAP>& list, uint32_t& chunks, const zccl_adamw_tensor* tensors, size_t count, size_t at, unsigned long long& place, size_t chunk)
{
    list.count = 0;
    chunks = 0;
    size_t i = at;
    for (; i < count && list.count < CAP; ++i) {
        const zccl_adamw_tensor& s = tensors[i];
        if (s.n == 0) continue;
        const size_t mine = (s.n + chunk - 1) / chunk;
        if (mine > kMostChunks - chunks) break;
        AdamTensor& to = list.t[list.count];
        to = {s.p, s.g, s.m, s.v, (unsigned char*)s.m_scale, (unsigned char*)s.v_scale, s.copy, s.n, place, false};
        to.wide = (((uintptr_t)s.p | (uintptr_t)s.g | (uintptr_t)s.m | (uintptr_t)s.v | (uintptr_t)s.copy) % 16) == 0;
        list.first[list.count++] = chunks;
        chunks += (uint32_t)mine;
        place += (s.n + kMxBlock - 1) / kMxBlock * kMxBlock;
    }
    return i - at;
}
// (Lists are up to 32 KB, as arguments of a kernel may be, and stand on the stack: there is no allocation to fail.)
template <int CAP>
int run_list(const zccl_adamw_tensor* tensors, size_t count, const zccl_adamw_config& k, const AdamCall& call, cudaStream_t st)
{
    AdamList<CAP> list;
    unsigned long long place = 0;
    int rc = ZCCL_OK;
    for (size_t at = 0; at < count && rc == ZCCL_OK;) {
        uint32_t chunks;
        at += fill_list(list, chunks, tensors, count, at, place, (size_t)call.passes * kPass);
        if (chunks == 0) continue;
        if (launch_adamw_param(k, list, chunks, call, st) == cudaSuccess) count_launches(1);
        else rc = ZCCL_E_CUDA;
    }
    return rc;
}

// Up to this many chunks are one CTA's work in less time than a second launch takes.
constexpr size_t kNormAlone = 4;

template <int CAP>
int run_norm(const void* const* g, const size_t* n, size_t count, size_t chunks, int type, float* norm, double* parts, cudaStream_t st)
{
    NormList<CAP> list;
    uint32_t written = 0;
    cudaError_t e = cudaSuccess;
    bool joined = false;
    for (size_t at = 0; at < count && e == cudaSuccess;) {
        list.count = 0;
        list.chunks = 0;
        const size_t from = at;
        for (; at < count && list.count < CAP; ++at) {
            if (n[at] == 0) continue;
            const size_t mine = (n[at] + kChunk - 1) / kChunk;
            if (mine > kMostChunks - list.chunks) break;
            list.g[list.count] = g[at];
            list.n[list.count] = n[at];
            list.first[list.count++] = list.chunks;
            list.chunks += (uint32_t)mine;
        }
        if (list.chunks == 0) continue;
        joined = chunks <= kNormAlone && from == 0 && list.chunks == chunks;
        const uint32_t ctas = joined ? 1u : std::min<uint32_t>(list.chunks, kNormCtas);
        const auto kernel = type == ZCCL_F32 ? norm_parts_kernel<float, CAP> : type == ZCCL_BF16 ? norm_parts_kernel<__nv_bfloat16, CAP> : norm_parts_kernel<__half, CAP>;
        e = launch_k(kernel, dim3(ctas), dim3(kOptThreads), 0, st, list, parts + written, joined ? norm : nullptr);
        if (e == cudaSuccess) count_launches(1);
        written += ctas;
    }
    if (!joined && e == cudaSuccess) {
        e = launch_k(norm_join_kernel, dim3(1), dim3(kOptThreads), 0, st, parts, written, norm);
        if (e == cudaSuccess) count_launches(1);
    }
    return e == cudaSuccess ? ZCCL_OK : ZCCL_E_CUDA;
}

bool type_ok(int t) { return t >= ZCCL_F32 && t <= ZCCL_F16; }
uintptr_t mask_of(int t) { return t == ZCCL_F32 ? 3u : 1u; }
bool at_element(const void* p, uintptr_t mask) { return p && ((uintptr_t)p & mask) == 0; }

}  // namespace
}  // namespace zccl

using namespace zccl;

extern "C" {

int zccl_adamw(const zccl_adamw_tensor* tensors, size_t count, const zccl_adamw_config* config, void* stream)
{
    if (!config || (!tensors && count)) return ZCCL_E_ARG;
    const zccl_adamw_config& k = *config;
    if (!type_ok(k.param_type) || !type_ok(k.grad_type) || (k.state_bits != 32 && k.state_bits != 8)) return ZCCL_E_ARG;
    const auto rate_ok = [](double b) { return b >= 0.0 && b < 1.0; };
    if (!rate_ok(k.beta1) || !rate_ok(k.beta2) || !(k.eps >= 0.0) || !std::isfinite(k.eps) || !std::isfinite(k.weight_decay)) return ZCCL_E_ARG;
    if (k.eps > 0.0 && (float)k.eps < FLT_MIN) return ZCCL_E_ARG;   // see reciprocal_of
    if ((!k.lr_device && !std::isfinite(k.lr)) || (!k.step_device && k.step < 1) || (k.norm && !(k.max_norm > 0.0))) return ZCCL_E_ARG;
    if (((uintptr_t)k.step_device & 7u) || ((uintptr_t)k.lr_device & 3u) || ((uintptr_t)k.norm & 3u)) return ZCCL_E_ARG;
    size_t used = 0, total = 0;
    for (size_t i = 0; i < count; ++i) {
        const zccl_adamw_tensor& t = tensors[i];
        if (t.n == 0) continue;
        ++used;
        total += t.n;
        const uintptr_t state = k.state_bits == 8 ? 0u : 3u;
        if (t.n > kMostElems || !at_element(t.p, mask_of(k.param_type)) || !at_element(t.g, mask_of(k.grad_type)) || !at_element(t.m, state) || !at_element(t.v, state))
            return ZCCL_E_ARG;
        if (k.state_bits == 8 && (!t.m_scale || !t.v_scale)) return ZCCL_E_ARG;
        if (t.copy && (k.param_type != ZCCL_F32 || (k.copy_type != ZCCL_BF16 && k.copy_type != ZCCL_F16) || ((uintptr_t)t.copy & 1u))) return ZCCL_E_ARG;
    }
    if (used == 0) return ZCCL_OK;
    AdamCall call{};
    call.beta1 = (float)k.beta1;
    call.rest1 = (float)(1.0 - k.beta1);
    call.beta2 = (float)k.beta2;
    call.root_beta2 = (float)std::sqrt(k.beta2);
    call.root_rest2 = (float)std::sqrt(1.0 - k.beta2);
    call.eps = (float)k.eps;
    call.lr = k.lr;
    call.weight_decay = k.weight_decay;
    call.log_beta1 = std::log(k.beta1);
    call.log_beta2 = std::log(k.beta2);
    call.step = k.step_device;
    call.lr_device = k.lr_device;
    call.step_host = k.step_device ? 1 : k.step;
    if (!k.step_device && !k.lr_device) {
        call.keep = (float)(1.0 - k.lr * k.weight_decay);
        call.rate = (float)(k.lr / -std::expm1((double)k.step * call.log_beta1));
        call.root = (float)(1.0 / std::sqrt(-std::expm1((double)k.step * call.log_beta2)));
    }
    call.seed = k.seed;
    call.norm = k.norm;
    call.max_norm = (float)k.max_norm;
    call.copy_type = k.copy_type;
    // Small models are spread over the SMs; large ones have chunks of several passes, whose first loads alone are not covered by work.  Of two, four and eight
    // passes 64 Mi parameters with states in 32 bits took 326, 317 and 328 us (more is left at the end).  With states in 8 bits and 16-bit parameters four and eight
    // took (290 tensors) 77.8 and 77.8 us for 32 Mi, 143.4 and 139.3 for 64 Mi, 270 and 260 for 128 Mi, 1078 and 1032 for 512 Mi, one tensor 1 to 2 % less with eight; with
    // binary32 parameters eight took 1 to 3 % longer from 16 to 512 Mi (128 Mi: 336 and 340 us).
    call.passes = 1;
    while (call.passes < 4 && total / kPass > (size_t)kChunksWanted * call.passes) call.passes *= 2;
    if (k.state_bits == 8 && k.param_type != ZCCL_F32 && total / kPass >= (size_t)32 * kChunksWanted) call.passes = 8;
    if (used <= (size_t)kFewTensors) return run_list<kFewTensors>(tensors, count, k, call, (cudaStream_t)stream);
    if (used <= (size_t)kMoreTensors) return run_list<kMoreTensors>(tensors, count, k, call, (cudaStream_t)stream);
    return run_list<kManyTensors>(tensors, count, k, call, (cudaStream_t)stream);
}

size_t zccl_grad_norm_work(size_t count) { return (count / kFewTensors + 2) * kNormCtas * sizeof(double); }

int zccl_grad_norm(const void* const* g, const size_t* n, size_t count, int grad_type, float* norm, void* work, void* stream)
{
    if (!type_ok(grad_type) || (count && (!g || !n)) || !at_element(norm, 3u) || !at_element(work, 7u)) return ZCCL_E_ARG;
    for (size_t i = 0; i < count; ++i)
        if (n[i] && (n[i] > kMostElems || !at_element(g[i], mask_of(grad_type)))) return ZCCL_E_ARG;
    size_t used = 0, chunks = 0;
    for (size_t i = 0; i < count; ++i) {
        used += n[i] != 0;
        chunks += (n[i] + kChunk - 1) / kChunk;
    }
    cudaStream_t st = (cudaStream_t)stream;
    return used <= (size_t)kFewTensors ? run_norm<kFewTensors>(g, n, count, chunks, grad_type, norm, (double*)work, st)
                                       : run_norm<kManyTensors>(g, n, count, chunks, grad_type, norm, (double*)work, st);
}

}  // extern "C"
