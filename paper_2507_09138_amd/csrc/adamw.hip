// The step of AdamW over many tensors, moments in 32 or in 8 bits (hr_layers.h).
#include <cmath>

#include "entry.h"
#include "hr_layers.h"
#include "wave.h"

namespace hr {

constexpr int kBlock = HR_ADAMW_BLOCK;                   // one wave's: four numbers a lane
constexpr int kBlocks = 4;                               // that a wave asks for at once
constexpr int kChunk = 4 * kBlocks * kBlock;             // of a workgroup of four waves
constexpr int kTensors = 48;                             // of a launch: what its arguments have room for

struct AdamwTensor {
    void* param; const void* grad; float* master; void* m; void* v; uint8_t* exponents;
    int64_t n;
    float decay;                                         // 1 - lr weight_decay
    int32_t kind;                                        // Kind of its numbers, and the 16-bit types among them
};
enum { kParam16 = 1, kGrad16 = 2, kMaster = 4, kEight = 8, kParamHalf = 16, kGradHalf = 32 };
struct AdamwArgs {
    AdamwTensor t[kTensors];
    uint32_t first[kTensors + 1];                        // chunk at which each tensor begins, and how many there are
    int count;
    float beta1, left1, beta2, left2, eps;               // left: 1 - beta
    float rate, spread;                                  // lr / (1 - beta1^step), 1 / sqrt(1 - beta2^step)
    double lr, b1, b2;                                   // for device_step
    const int64_t* device_step;
    const float* grad_scale;
};

__device__ __forceinline__ float power(uint32_t biased) { return __builtin_bit_cast(float, biased << 23); }

// four numbers from i on, zeros from n on
template <typename T>
__device__ __forceinline__ void load_four(const T* at, int64_t i, int64_t n, T* x)
{
    if (i + 4 <= n) {
        __builtin_memcpy(x, at + i, 4 * sizeof(T));      // (tensors may begin at any element)
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = i + e < n ? at[i + e] : T{};
    }
}
template <typename T>
__device__ __forceinline__ void store_four(T* at, int64_t i, int64_t n, const T* x)
{
    if (i + 4 <= n) {
        __builtin_memcpy(at + i, x, 4 * sizeof(T));
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (i + e < n) at[i + e] = x[e];
    }
}
// 16-bit numbers, which of the two types they are known when it runs
__device__ __forceinline__ float from16(uint16_t b, bool half)
{
    return half ? (float)__builtin_bit_cast(_Float16, b) : __builtin_bit_cast(float, (uint32_t)b << 16);
}
__device__ __forceinline__ uint16_t to16(float x, bool half)
{
    return half ? __builtin_bit_cast(uint16_t, (_Float16)x) : __builtin_bit_cast(uint16_t, (__bf16)x);
}

__device__ __forceinline__ void decode_m(uint32_t codes, uint32_t em, float* m)
{
    const float unit = em == 255 ? NAN : power(max(em, 8u) - 7);
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(codes, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(codes, true);
    m[0] = lo[0] * unit;
    m[1] = lo[1] * unit;
    m[2] = hi[0] * unit;
    m[3] = hi[1] * unit;
}
__device__ __forceinline__ void decode_v(uint32_t codes, uint32_t ev, float* v)
{
    const uint32_t base = 8 * (max(ev, 31u) - 31);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const uint32_t c = codes >> (8 * e) & 0xffu;
        v[e] = ev == 255 ? NAN : (c ? __builtin_bit_cast(float, (c + base) << 20) : 0.0f);
    }
}
__device__ __forceinline__ uint32_t most(uint32_t v)
{
    return wave_fold(v, [](uint32_t x, uint32_t y) { return x > y ? x : y; });
}
// The codes of a block: the lanes' four numbers each, and the block's exponent.
__device__ __forceinline__ uint32_t encode_m(const float* m, uint32_t& em)
{
    uint32_t largest = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) largest = max(largest, __builtin_bit_cast(uint32_t, m[e]) & 0x7fffffffu);
    em = max(most(largest) >> 23, 8u);
    const float up = power(261 - em);
    uint32_t w = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(m[0] * up, m[1] * up, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(m[2] * up, m[3] * up, (int)w, true);
}
__device__ __forceinline__ uint32_t encode_v(const float* v, uint32_t& ev)
{
    uint32_t upper[4], largest = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const uint32_t b = __builtin_bit_cast(uint32_t, v[e]) & 0x7fffffffu;
        upper[e] = (b + 0x7ffffu + (b >> 20 & 1)) >> 20;
        largest = max(largest, upper[e]);
    }
    ev = max(min(most(largest) >> 3, 255u), 31u);
    const int base = 8 * ((int)ev - 31);
    uint32_t w = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) w |= (v[e] > 0.0f ? (uint32_t)max((int)upper[e] - base, 1) & 0xffu : 0u) << (8 * e);
    return w;
}

struct Rates { float rate, spread, scale; };

// A chunk of a tensor: all of a wave's blocks are asked for before the first is worked on.  Bound by memory, about half of it written; 10^8 numbers: float32
// 515 us (28 bytes each, 5.4 TB/s), bfloat16 with a master 523 (28 bytes), moments in 8 bits 290 (16 bytes, 5.5 TB/s).
template <bool P16, bool G16, bool MASTER, bool EIGHT>
__device__ __forceinline__ void adamw_chunk(const AdamwArgs& a, const AdamwTensor& t, const Rates& r, int64_t begin)
{
    using P = std::conditional_t<P16, uint16_t, float>;
    using G = std::conditional_t<G16, uint16_t, float>;
    using M = std::conditional_t<EIGHT, uint8_t, float>;
    const bool phalf = t.kind & kParamHalf, ghalf = t.kind & kGradHalf;
    const int64_t n = t.n, base = begin + (int64_t)(threadIdx.x / 64) * kBlocks * kBlock;
    const int lane = lane_id();
    P p[kBlocks][4];
    G g[kBlocks][4];
    float w[kBlocks][4];
    M m8[kBlocks][4], v8[kBlocks][4];
    uint32_t ex[kBlocks];
#pragma unroll
    for (int u = 0; u < kBlocks; ++u) {
        const int64_t at = base + u * kBlock, i = at + lane * 4;
        if (at >= n) continue;
        if constexpr (MASTER) load_four(t.master, i, n, w[u]);
        else load_four((const P*)t.param, i, n, p[u]);
        load_four((const G*)t.grad, i, n, g[u]);
        load_four((const M*)t.m, i, n, m8[u]);
        load_four((const M*)t.v, i, n, v8[u]);
        if constexpr (EIGHT) {
            const uint8_t* e = t.exponents + at / kBlock * 2;
            ex[u] = e[0] | (uint32_t)e[1] << 8;
        }
    }
#pragma unroll
    for (int u = 0; u < kBlocks; ++u) {
        const int64_t at = base + u * kBlock, i = at + lane * 4;
        if (at >= n) continue;
        float m[4], v[4];
        if constexpr (EIGHT) {
            uint32_t mw, vw;
            __builtin_memcpy(&mw, m8[u], 4);
            __builtin_memcpy(&vw, v8[u], 4);
            decode_m(mw, ex[u] & 0xffu, m);
            decode_v(vw, ex[u] >> 8, v);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) m[e] = m8[u][e], v[e] = v8[u][e];
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
#pragma clang fp contract(off)
            float grad, value;
            if constexpr (G16) grad = from16(g[u][e], ghalf);
            else grad = g[u][e];
            grad = grad * r.scale;
            m[e] = m[e] * a.beta1 + grad * a.left1;
            v[e] = v[e] * a.beta2 + grad * grad * a.left2;
            if constexpr (MASTER) value = w[u][e];
            else if constexpr (P16) value = from16(p[u][e], phalf);
            else value = p[u][e];
            value = value * t.decay - m[e] * r.rate / (sqrtf(v[e]) * r.spread + a.eps);
            if constexpr (MASTER) w[u][e] = value;
            if constexpr (P16) p[u][e] = to16(value, phalf);
            else p[u][e] = value;
        }
        store_four((P*)t.param, i, n, p[u]);
        if constexpr (MASTER) store_four(t.master, i, n, w[u]);
        if constexpr (EIGHT) {
            // (behind the tensor's end the lanes hold zeros: gradient and moments)
            uint32_t em, ev;
            const uint32_t mw = encode_m(m, em), vw = encode_v(v, ev);
            __builtin_memcpy(m8[u], &mw, 4);
            __builtin_memcpy(v8[u], &vw, 4);
            uint8_t* e = t.exponents + at / kBlock * 2;
            if (lane < 2) e[lane] = (uint8_t)(lane ? ev : em);
            store_four((M*)t.m, i, n, m8[u]);
            store_four((M*)t.v, i, n, v8[u]);
        } else {
            store_four((M*)t.m, i, n, (const M*)m);
            store_four((M*)t.v, i, n, (const M*)v);
        }
    }
}

// What is updated, and where its chunks begin, are arguments of the launch: a step of an encoder's hundred tensors is a few launches and no copy.
__global__ __launch_bounds__(256) void k_adamw(AdamwArgs a)
{
    Rates r{a.rate, a.spread, a.grad_scale ? *a.grad_scale : 1.0f};
    if (a.device_step) {
        const double t = (double)max(*a.device_step, (int64_t)1);
        r.rate = (float)(a.lr / (1.0 - pow(a.b1, t)));
        r.spread = (float)(1.0 / sqrt(1.0 - pow(a.b2, t)));
    }
    const uint32_t chunks = a.first[a.count];
    for (uint32_t c = blockIdx.x; c < chunks; c += gridDim.x) {
        int lo = 0, hi = a.count;                        // the last tensor that begins at c or before (one without numbers begins where the next does)
        while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            if (a.first[mid] <= c) lo = mid;
            else hi = mid;
        }
        const AdamwTensor& t = a.t[lo];
        const int64_t begin = (int64_t)(c - a.first[lo]) * kChunk;
        switch (t.kind & 15) {
        case 0: adamw_chunk<false, false, false, false>(a, t, r, begin); break;
        case kParam16: adamw_chunk<true, false, false, false>(a, t, r, begin); break;
        case kGrad16: adamw_chunk<false, true, false, false>(a, t, r, begin); break;
        case kParam16 | kGrad16: adamw_chunk<true, true, false, false>(a, t, r, begin); break;
        case kParam16 | kMaster: adamw_chunk<true, false, true, false>(a, t, r, begin); break;
        case kParam16 | kGrad16 | kMaster: adamw_chunk<true, true, true, false>(a, t, r, begin); break;
        case kEight: adamw_chunk<false, false, false, true>(a, t, r, begin); break;
        case kEight | kParam16: adamw_chunk<true, false, false, true>(a, t, r, begin); break;
        case kEight | kGrad16: adamw_chunk<false, true, false, true>(a, t, r, begin); break;
        case kEight | kParam16 | kGrad16: adamw_chunk<true, true, false, true>(a, t, r, begin); break;
        case kEight | kParam16 | kMaster: adamw_chunk<true, false, true, true>(a, t, r, begin); break;
        case kEight | kParam16 | kGrad16 | kMaster: adamw_chunk<true, true, true, true>(a, t, r, begin); break;
        }
    }
}

// (memory too: 528 million numbers of both 1060 us, 5.0 TB/s)
__global__ __launch_bounds__(256) void k_adamw_moments(const uint8_t* m, const uint8_t* v, const uint8_t* exponents, int64_t n, float* out_m, float* out_v)
{
    const int64_t fours = (n + 3) / 4;
    for (int64_t j = (int64_t)blockIdx.x * 256 + threadIdx.x; j < fours; j += (int64_t)gridDim.x * 256) {
        const int64_t i = j * 4;
        const uint8_t* e = exponents + i / kBlock * 2;
        uint8_t codes[4];
        uint32_t w;
        float x[4];
        if (out_m) {
            load_four(m, i, n, codes);
            __builtin_memcpy(&w, codes, 4);
            decode_m(w, e[0], x);
            store_four(out_m, i, n, x);
        }
        if (out_v) {
            load_four(v, i, n, codes);
            __builtin_memcpy(&w, codes, 4);
            decode_v(w, e[1], x);
            store_four(out_v, i, n, x);
        }
    }
}

static int check_tensor(int32_t i, const hr_adamw_tensor& t)
{
    if (!known_type(t.param_dtype) || !known_type(t.grad_dtype)) return fail(HR_ERR_ARG, "tensor %d: unknown dtype", i);
    if (t.n < 0 || t.n > (1LL << 36)) return fail(HR_ERR_ARG, "tensor %d: n=%lld out of range", i, (long long)t.n);
    if (!std::isfinite(t.weight_decay)) return fail(HR_ERR_ARG, "tensor %d: weight_decay=%g", i, (double)t.weight_decay);
    if (t.master && t.param_dtype == HR_F32) return fail(HR_ERR_ARG, "tensor %d: a master beside a parameter in 32 bits", i);
    if (t.n == 0) return HR_OK;
    if (!t.param || !t.grad || !t.m || !t.v) return fail(HR_ERR_ARG, "tensor %d: param, grad, m or v is null", i);
    if ((uintptr_t)t.param % element_bytes(t.param_dtype) || (uintptr_t)t.grad % element_bytes(t.grad_dtype) || (uintptr_t)t.master % 4 ||
        (!t.exponents && ((uintptr_t)t.m % 4 || (uintptr_t)t.v % 4)))
        return fail(HR_ERR_ARG, "tensor %d is not aligned to its elements", i);
    return HR_OK;
}

}  // namespace hr

// ---- C entry points
using namespace hr;

extern "C" {

int hr_adamw(const hr_adamw_tensor* tensors, int32_t count, double lr, double beta1, double beta2, double eps, int64_t step,
             const int64_t* device_step, const float* grad_scale, void* stream)
{
    if (count < 0) return fail(HR_ERR_ARG, "count=%d", count);
    if (count > 0 && !tensors) return fail(HR_ERR_ARG, "tensors is null");
    if (!std::isfinite(lr)) return fail(HR_ERR_ARG, "lr=%g", lr);
    if (!(beta1 >= 0 && beta1 < 1) || !(beta2 >= 0 && beta2 < 1)) return fail(HR_ERR_ARG, "beta1=%g, beta2=%g: want 0 <= beta < 1", beta1, beta2);
    if (!(eps >= 0) || !std::isfinite(eps)) return fail(HR_ERR_ARG, "eps=%g", eps);
    if (!device_step && step < 1) return fail(HR_ERR_ARG, "step=%lld: want 1 or more", (long long)step);
    if ((uintptr_t)device_step % 8 || (uintptr_t)grad_scale % 4) return fail(HR_ERR_ARG, "device_step or grad_scale is not aligned");
    for (int32_t i = 0; i < count; ++i)
        if (int rc = check_tensor(i, tensors[i])) return rc;
    const double t = (double)(step < 1 ? 1 : step);
    AdamwArgs a;
    a.beta1 = (float)beta1;
    a.left1 = (float)(1 - beta1);
    a.beta2 = (float)beta2;
    a.left2 = (float)(1 - beta2);
    a.eps = (float)eps;
    a.rate = (float)(lr / (1 - std::pow(beta1, t)));
    a.spread = (float)(1 / std::sqrt(1 - std::pow(beta2, t)));
    a.lr = lr;
    a.b1 = beta1;
    a.b2 = beta2;
    a.device_step = device_step;
    a.grad_scale = grad_scale;
    for (int32_t i = 0; i < count;) {
        a.count = 0;
        a.first[0] = 0;
        for (; i < count && a.count < kTensors; ++i) {
            const hr_adamw_tensor& x = tensors[i];
            if (x.n == 0) continue;
            AdamwTensor& y = a.t[a.count];
            y = {x.param, x.grad, x.master, x.m, x.v, x.exponents, x.n, (float)(1 - lr * (double)x.weight_decay), 0};
            y.kind = (x.param_dtype != HR_F32 ? kParam16 : 0) | (x.grad_dtype != HR_F32 ? kGrad16 : 0) | (x.master ? kMaster : 0) | (x.exponents ? kEight : 0) |
                     (x.param_dtype == HR_F16 ? kParamHalf : 0) | (x.grad_dtype == HR_F16 ? kGradHalf : 0);
            a.first[a.count + 1] = a.first[a.count] + (uint32_t)((x.n + kChunk - 1) / kChunk);
            ++a.count;
        }
        if (a.count == 0) break;
        const uint32_t chunks = a.first[a.count];
        hipLaunchKernelGGL(k_adamw, dim3(chunks < (1u << 20) ? chunks : 1u << 20), dim3(256), 0, (hipStream_t)stream, a);
        HR_HIP(hipGetLastError());
    }
    return HR_OK;
}

int hr_adamw_moments(const uint8_t* m, const uint8_t* v, const uint8_t* exponents, int64_t n, float* out_m, float* out_v, void* stream)
{
    if (n < 0 || n > (1LL << 36)) return fail(HR_ERR_ARG, "n=%lld out of range", (long long)n);
    if (n == 0 || (!out_m && !out_v)) return HR_OK;
    if ((out_m && !m) || (out_v && !v) || !exponents) return fail(HR_ERR_ARG, "m, v or exponents is null");
    if ((uintptr_t)out_m % 4 || (uintptr_t)out_v % 4) return fail(HR_ERR_ARG, "out_m or out_v is not aligned to its elements");
    const int64_t want = ((n + 3) / 4 + 255) / 256;
    hipLaunchKernelGGL(k_adamw_moments, dim3((unsigned)(want < (1 << 20) ? want : 1 << 20)), dim3(256), 0, (hipStream_t)stream, m, v, exponents, n, out_m, out_v);
    HR_HIP(hipGetLastError());
    return HR_OK;
}

}  // extern "C"
