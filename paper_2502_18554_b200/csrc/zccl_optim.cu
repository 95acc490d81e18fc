// The norm of all gradients and the AdamW step over many tensors at once, states in 32 or in 8 bits.
#include "../../include/zccl.h"
#include "zccl_mx4.cuh"

#include <cuda_fp8.h>

#include <algorithm>
#include <cmath>
#include <new>
#include <vector>

namespace zccl {
namespace {

constexpr int kOptThreads = 256;
constexpr int kPerThread = 8;                       // neighbouring elements of a thread: four threads hold a block of 32
constexpr int kPass = kOptThreads * kPerThread;
constexpr int kChunk = 4 * kPass;                   // elements of a tensor that a CTA takes
// Tensors travel as kernel arguments, so a call copies nothing, needs no memory and can be captured.  Arguments above 4 KB cost
// the launch a few microseconds, hence two sizes of the list.
constexpr int kFewTensors = 40, kManyTensors = 380;

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

// `full`: all eight are there and the array begins on a 16-byte boundary; else the first `left` ones are read.
template <class T>
__device__ __forceinline__ void read8(const T* p, bool full, int left, float (&v)[8])
{
    constexpr int kPer = 16 / sizeof(T);
    if (full) {
#pragma unroll
        for (int i = 0; i < 8 / kPer; ++i) {
            const uint4 raw = __ldcs(reinterpret_cast<const uint4*>(p) + i);
            const MxPack<T> pack = *reinterpret_cast<const MxPack<T>*>(&raw);
#pragma unroll
            for (int j = 0; j < kPer; ++j) v[kPer * i + j] = mx_float(pack.v[j]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < left ? mx_float(p[i]) : 0.0f;
    }
}
template <class T>
__device__ __forceinline__ void write8(T* p, bool full, int left, const float (&v)[8])
{
    constexpr int kPer = 16 / sizeof(T);
    if (full) {
#pragma unroll
        for (int i = 0; i < 8 / kPer; ++i) {
            MxPack<T> pack;
#pragma unroll
            for (int j = 0; j < kPer; ++j) pack.v[j] = mx_round<T>(v[kPer * i + j]);
            __stcs(reinterpret_cast<uint4*>(p) + i, *reinterpret_cast<const uint4*>(&pack));
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < left) p[i] = mx_round<T>(v[i]);
    }
}

// ------------------------------------------------------------------------------------------------ norm

constexpr int kNormCtas = 1024;   // partial sums of a launch

struct NormList {
    static constexpr int kMost = kManyTensors;
    const void* g[kMost];
    unsigned long long n[kMost];
    uint32_t first[kMost];
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
template <class G>
__global__ void __launch_bounds__(kOptThreads) norm_parts_kernel(const __grid_constant__ NormList list, double* __restrict__ parts)
{
    pdl_enter();
    double sum = 0.0;
    for (uint32_t c = blockIdx.x; c < list.chunks; c += gridDim.x) {
        const int t = tensor_of(list, c);
        const unsigned long long n = list.n[t], begin = (unsigned long long)(c - list.first[t]) * kChunk;
        const G* g = (const G*)list.g[t] + begin;
        const bool aligned = wide((const G*)list.g[t]);
        const int left_all = (int)min((unsigned long long)kChunk, n - begin);
#pragma unroll
        for (int i = 0; i < kChunk / kPass; ++i) {
            const int at = i * kPass + threadIdx.x * kPerThread, left = left_all - at;
            if (left > 0) {
                float v[8];
                read8(g + at, aligned && left >= 8, left, v);
                float s = 0.0f;
#pragma unroll
                for (int j = 0; j < 8; ++j) s = __fmaf_rn(v[j], v[j], s);
                if (s > 1e-24f && s < 1e37f) sum += (double)s;
                else
                    for (int j = 0; j < 8; ++j) sum += (double)v[j] * (double)v[j];
            }
        }
    }
    sum = block_sum(sum);
    if (threadIdx.x == 0) parts[blockIdx.x] = sum;
}

__global__ void __launch_bounds__(kOptThreads) norm_join_kernel(const double* __restrict__ parts, uint32_t count, float* __restrict__ norm)
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
};
template <int CAP>
struct AdamList {
    AdamTensor t[CAP];
    uint32_t first[CAP];
    int count;
};

struct AdamCall {
    float beta1, rest1, beta2, rest2, eps;
    float keep, rate, root;        // 1 - lr weight_decay; lr / (1 - beta1^step); 1 / sqrt(1 - beta2^step)
    double lr, weight_decay, log_beta1, log_beta2;   // where step or lr is on the device
    const long long* step;
    const float* lr_device;
    long long step_host;
    unsigned long long seed;
    const float* norm;
    float max_norm;
    int copy_type;
};

__host__ __device__ inline unsigned long long random_key(unsigned long long seed, long long step)
{
    return seed + (unsigned long long)step * 0x9E3779B97F4A7C15ull;
}
// 32 random bits for the element at `place`: three rounds of multiplying and folding the upper bits down.
__device__ __forceinline__ uint32_t random_bits(unsigned long long key, unsigned long long place)
{
    uint32_t h = ((uint32_t)place ^ (uint32_t)key) * 0x7FEB352Du;
    h = ((h ^ (h >> 15)) ^ (uint32_t)(key >> 32) ^ (uint32_t)(place >> 32)) * 0x846CA68Bu;
    h = (h ^ (h >> 13)) * 0x6C8E9CF5u;
    return h ^ (h >> 16);
}

__device__ __forceinline__ uint32_t top8(const float (&v)[8])
{
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(v[i]) & 0x7FFFFFFFu);
    top = max(top, __shfl_xor_sync(kFull, top, 1));
    return max(top, __shfl_xor_sync(kFull, top, 2));
}
// The biased exponent at which the block's largest magnitude is at most 448 = 1.75 * 2^8; 255 where it is not finite.
__device__ __forceinline__ uint32_t exponent8(uint32_t top)
{
    const int field = (int)(top >> 23);
    return field == 255 ? 255u : (uint32_t)max(field - 8 + ((top & 0x7FFFFFu) > 0x600000u ? 1 : 0), 0);
}
// One value, already times 2^-e, to E4M3: `noise` (20 bits) is added below the last bit that is kept.  Magnitudes below 2^-6 have the
// step of 2^-9: with 2^-6 added their step is where a normal number's is.
__device__ __forceinline__ uint32_t encode8(float y, uint32_t noise)
{
    const float a = fabsf(y);
    const bool small = a < 0.015625f;
    const float b = small ? __fadd_rz(a, 0.015625f) : a;
    return ((__float_as_uint(b) + noise) >> 20) - (small ? 968u : 960u);
}
__device__ __forceinline__ void decode8(uint2 w, float scale, float (&v)[8])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t two = (i & 2 ? w.y : w.x) >> (16 * (i & 1));
        const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(two & 0xFFFFu), __NV_E4M3);
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
        v[2 * i] = f.x * scale;
        v[2 * i + 1] = f.y * scale;
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
// Eight elements of a block to codes; `shift` says which half of the random bits they take.
template <bool ROOT>
__device__ __forceinline__ uint2 pack8(const float (&v)[8], const uint32_t (&random)[8], uint32_t s)
{
    const float inverse = __uint_as_float((254u - s) << 23);
    uint32_t w[2] = {0, 0};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t noise = ROOT ? (random[i] & 0xFFFFu) << 4 : random[i] >> 16 << 4;
        uint32_t c = encode8(v[i] * inverse, noise);
        if (ROOT) c = max(c, v[i] > 0.0f ? 1u : 0u);
        else c |= __float_as_uint(v[i]) >> 31 << 7;
        w[i >> 2] |= c << (8 * (i & 3));
    }
    return s == 255u ? make_uint2(0x7F7F7F7Fu, 0x7F7F7F7Fu) : make_uint2(w[0], w[1]);
}

__device__ __forceinline__ float root_of(float v)
{
    float r;
    asm("sqrt.approx.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}

template <class P, class G, bool EIGHT, int CAP>
__global__ void __launch_bounds__(kOptThreads) adamw_kernel(const __grid_constant__ AdamList<CAP> list, const __grid_constant__ AdamCall call)
{
    pdl_enter();
    float clip = 1.0f;
    if (call.norm) {
        const float norm = *call.norm;
        if (!(norm >= 0.0f && norm < __int_as_float(0x7F800000))) return;   // no norm of finite gradients: no step
        clip = fminf(1.0f, __fdiv_rn(call.max_norm, norm + 1e-6f));
    }
    float keep = call.keep, rate = call.rate, root = call.root;
    unsigned long long key = random_key(call.seed, call.step_host);
    if (call.step || call.lr_device) {
        __shared__ float sh[3];
        const long long step = call.step ? *call.step : call.step_host;
        key = random_key(call.seed, step);
        if (threadIdx.x == 0) {
            const double lr = call.lr_device ? (double)*call.lr_device : call.lr;
            sh[0] = (float)(1.0 - lr * call.weight_decay);
            sh[1] = (float)(lr / -expm1((double)step * call.log_beta1));
            sh[2] = (float)(1.0 / sqrt(-expm1((double)step * call.log_beta2)));
        }
        __syncthreads();
        keep = sh[0];
        rate = sh[1];
        root = sh[2];
    }
    const int t = tensor_of(list, blockIdx.x);
    const AdamTensor& a = list.t[t];
    const unsigned long long begin = (unsigned long long)(blockIdx.x - list.first[t]) * kChunk;
    const int left_all = (int)min((unsigned long long)kChunk, a.n - begin);
    P* const p = (P*)a.p + begin;
    const G* const g = (const G*)a.g + begin;
    const bool p_wide = wide(p), g_wide = wide(g), copies = a.copy != nullptr, copy_wide = wide((const __half*)a.copy);
    for (int at = threadIdx.x * kPerThread; at - (int)(threadIdx.x & 31) * kPerThread < left_all; at += kPass) {   // whole warps
        const int left = left_all - at;
        const bool all = left >= 8;
        float pv[8], gv[8], mv[8], vv[8], rv[8];
        read8(p + at, all && p_wide, left, pv);
        read8(g + at, all && g_wide, left, gv);
        unsigned char *mc = nullptr, *vc = nullptr, *ms = nullptr, *vs = nullptr;
        bool m_wide, v_wide;
        if (EIGHT) {
            mc = (unsigned char*)a.m + begin + at;
            vc = (unsigned char*)a.v + begin + at;
            ms = a.m_scale + (begin + at) / kMxBlock;
            vs = a.v_scale + (begin + at) / kMxBlock;
            m_wide = all && ((uintptr_t)mc & 7u) == 0;
            v_wide = all && ((uintptr_t)vc & 7u) == 0;
            decode8(read_codes(mc, m_wide, left), mx_scale(left > 0 ? *ms : 0u), mv);
            decode8(read_codes(vc, v_wide, left), mx_scale(left > 0 ? *vs : 0u), vv);
#pragma unroll
            for (int i = 0; i < 8; ++i) vv[i] *= vv[i];
        } else {
            m_wide = all && wide((float*)a.m);
            v_wide = all && wide((float*)a.v);
            read8((const float*)a.m + begin + at, m_wide, left, mv);
            read8((const float*)a.v + begin + at, v_wide, left, vv);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float gc = gv[i] * clip;
            mv[i] = __fmaf_rn(call.rest1, gc, call.beta1 * mv[i]);
            vv[i] = __fmaf_rn(call.rest2 * gc, gc, call.beta2 * vv[i]);
            rv[i] = root_of(vv[i]);
            pv[i] = __fmaf_rn(pv[i], keep, -(rate * __fdividef(mv[i], __fmaf_rn(rv[i], root, call.eps))));
        }
        write8(p + at, all && p_wide, left, pv);
        if (copies) {
            if (call.copy_type == ZCCL_BF16) write8((__nv_bfloat16*)a.copy + begin + at, all && copy_wide, left, pv);
            else write8((__half*)a.copy + begin + at, all && copy_wide, left, pv);
        }
        if (EIGHT) {
            uint32_t random[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                random[i] = random_bits(key, a.place + begin + at + i);
                if (i >= left) mv[i] = rv[i] = 0.0f;
            }
            const uint32_t se = exponent8(top8(mv)), re = exponent8(top8(rv));
            write_codes(mc, m_wide, left, pack8<false>(mv, random, se));
            write_codes(vc, v_wide, left, pack8<true>(rv, random, re));
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
size_t fill_list(AdamList<CAP>& list, uint32_t& chunks, const zccl_adamw_tensor* tensors, size_t count, size_t at, unsigned long long& place)
{
    list.count = 0;
    chunks = 0;
    size_t i = at;
    for (; i < count && list.count < CAP; ++i) {
        const zccl_adamw_tensor& s = tensors[i];
        if (s.n == 0) continue;
        const size_t mine = (s.n + kChunk - 1) / kChunk;
        if (mine > kMostChunks - chunks) break;
        list.t[list.count] = {s.p, s.g, s.m, s.v, (unsigned char*)s.m_scale, (unsigned char*)s.v_scale, s.copy, s.n, place};
        list.first[list.count++] = chunks;
        chunks += (uint32_t)mine;
        place += (s.n + kMxBlock - 1) / kMxBlock * kMxBlock;
    }
    return i - at;
}
template <int CAP>
int run_list(const zccl_adamw_tensor* tensors, size_t count, const zccl_adamw_config& k, const AdamCall& call, cudaStream_t st)
{
    AdamList<CAP>* list = new (std::nothrow) AdamList<CAP>;
    if (!list) return ZCCL_E_ARG;
    unsigned long long place = 0;
    int rc = ZCCL_OK;
    for (size_t at = 0; at < count && rc == ZCCL_OK;) {
        uint32_t chunks;
        at += fill_list(*list, chunks, tensors, count, at, place);
        if (chunks == 0) continue;
        if (launch_adamw_param(k, *list, chunks, call, st) == cudaSuccess) count_launches(1);
        else rc = ZCCL_E_CUDA;
    }
    delete list;
    return rc;
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
    if ((!k.lr_device && !std::isfinite(k.lr)) || (!k.step_device && k.step < 1) || (k.norm && !(k.max_norm > 0.0))) return ZCCL_E_ARG;
    if (((uintptr_t)k.step_device & 7u) || ((uintptr_t)k.lr_device & 3u) || ((uintptr_t)k.norm & 3u)) return ZCCL_E_ARG;
    size_t used = 0;
    for (size_t i = 0; i < count; ++i) {
        const zccl_adamw_tensor& t = tensors[i];
        if (t.n == 0) continue;
        ++used;
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
    call.rest2 = (float)(1.0 - k.beta2);
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
    return used <= (size_t)kFewTensors ? run_list<kFewTensors>(tensors, count, k, call, (cudaStream_t)stream)
                                       : run_list<kManyTensors>(tensors, count, k, call, (cudaStream_t)stream);
}

size_t zccl_grad_norm_work(size_t count) { return (count / kManyTensors + 2) * kNormCtas * sizeof(double); }

int zccl_grad_norm(const void* const* g, const size_t* n, size_t count, int grad_type, float* norm, void* work, void* stream)
{
    if (!type_ok(grad_type) || (count && (!g || !n)) || !at_element(norm, 3u) || !at_element(work, 7u)) return ZCCL_E_ARG;
    for (size_t i = 0; i < count; ++i)
        if (n[i] && (n[i] > kMostElems || !at_element(g[i], mask_of(grad_type)))) return ZCCL_E_ARG;
    NormList* list = new (std::nothrow) NormList;
    if (!list) return ZCCL_E_ARG;
    cudaStream_t st = (cudaStream_t)stream;
    double* parts = (double*)work;
    uint32_t written = 0;
    cudaError_t e = cudaSuccess;
    for (size_t at = 0; at < count && e == cudaSuccess;) {
        list->count = 0;
        list->chunks = 0;
        for (; at < count && list->count < NormList::kMost; ++at) {
            if (n[at] == 0) continue;
            const size_t mine = (n[at] + kChunk - 1) / kChunk;
            if (mine > kMostChunks - list->chunks) break;
            list->g[list->count] = g[at];
            list->n[list->count] = n[at];
            list->first[list->count++] = list->chunks;
            list->chunks += (uint32_t)mine;
        }
        if (list->chunks == 0) continue;
        const uint32_t ctas = std::min<uint32_t>(list->chunks, kNormCtas);
        const auto kernel = grad_type == ZCCL_F32 ? norm_parts_kernel<float> : grad_type == ZCCL_BF16 ? norm_parts_kernel<__nv_bfloat16> : norm_parts_kernel<__half>;
        e = launch_k(kernel, dim3(ctas), dim3(kOptThreads), 0, st, *list, parts + written);
        if (e == cudaSuccess) count_launches(1);
        written += ctas;
    }
    delete list;
    if (e == cudaSuccess) e = launch_k(norm_join_kernel, dim3(1), dim3(kOptThreads), 0, st, parts, written, norm);
    if (e == cudaSuccess) count_launches(1);
    return e == cudaSuccess ? ZCCL_OK : ZCCL_E_CUDA;
}

}  // extern "C"
