// The gated half of a feed-forward block, act(x w_gate') * (x w_up'), and its gradients (hr_layers.h).
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "entry.h"
#include "hr_layers.h"
#include "wave.h"

namespace hr {

// ---- activations: the value and the slope
constexpr float kSqrtHalf = 0.7071067811865476f, kSqrt2OverPi = 0.7978845608028654f, kOverSqrt2Pi = 0.3989422804014327f;

__device__ __forceinline__ float act_value(float z, int act, float& slope)
{
    if (act == HR_SILU) {
        const float p = 1.0f / (1.0f + expf(-z));
        slope = p * (1.0f + z * (1.0f - p));
        return z * p;
    }
    if (act == HR_GELU) {
        const float p = 0.5f * (1.0f + erff(z * kSqrtHalf));
        slope = p + z * expf(-0.5f * z * z) * kOverSqrt2Pi;
        return z * p;
    }
    const float t = tanhf(kSqrt2OverPi * (z + 0.044715f * z * z * z));
    slope = 0.5f * (1.0f + t) + 0.5f * z * (1.0f - t * t) * (kSqrt2OverPi * (1.0f + 3 * 0.044715f * z * z));
    return 0.5f * z * (1.0f + t);
}

// 16 bytes of k a lane: one matrix instruction of 16 bits, four of 32 bits (k in another order, the same for both operands).
// The first operand's rows are the result's rows, four of them in the registers of a lane, 4 (lane / 16) .. + 3, in column lane % 16.
template <typename T> using Frag = T __attribute__((ext_vector_type(16 / sizeof(T))));
__device__ __forceinline__ floatx4 multiply(Frag<_Float16> a, Frag<_Float16> b, floatx4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ floatx4 multiply(Frag<__bf16> a, Frag<__bf16> b, floatx4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ floatx4 multiply(Frag<float> a, Frag<float> b, floatx4 c)
{
#pragma unroll
    for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], c, 0, 0, 0);
    return c;
}

// out[i, j] = sum_t a[i, t] b[j, t] over one or two stretches of t, any strides
struct Operand { const void* at; int64_t row, step; };
struct ProductArgs {
    Operand a[2], b[2];
    int stretches;
    int64_t m, n, k;
    void *out, *out2; int64_t ldo, ldo2, split;          // rows from `split` on go to out2
    float* pre; int act;                                 // GATED: b[0] is the gate's matrix, b[1] up's
};
template <typename T, bool GATED>
__global__ __launch_bounds__(256) void k_product(ProductArgs p)
{
    constexpr int E = 16 / sizeof(T), K = 4 * E, S = K + E;
    __shared__ __align__(16) T ta[64 * S], tb[64 * S];
    constexpr int COLS = GATED ? 32 : 64;
    const int64_t m0 = (int64_t)blockIdx.x * 64, n0 = (int64_t)blockIdx.y * COLS;
    const int lane = lane_id(), wave = threadIdx.x / 64;
    floatx4 acc[4] = {};
    for (int s = 0; s < (GATED ? 1 : p.stretches); ++s)
        for (int64_t t0 = 0; t0 < p.k; t0 += K) {
            __syncthreads();
            for (int i = threadIdx.x; i < 64 * K; i += 256) {
                const int r = i / K, t = i % K;
                const Operand &oa = p.a[s], &ob = p.b[GATED ? r / 32 : s];
                const int64_t row = m0 + r, col = n0 + (GATED ? r % 32 : r);
                ta[r * S + t] = row < p.m && t0 + t < p.k ? ((const T*)oa.at)[row * oa.row + (t0 + t) * oa.step] : (T)0.0f;
                tb[r * S + t] = col < p.n && t0 + t < p.k ? ((const T*)ob.at)[col * ob.row + (t0 + t) * ob.step] : (T)0.0f;
            }
            __syncthreads();
            const Frag<T> fa = *(const Frag<T>*)(ta + (wave * 16 + lane % 16) * S + lane / 16 * E);
            for (int j = 0; j < 4; ++j) acc[j] = multiply(*(const Frag<T>*)(tb + (j * 16 + lane % 16) * S + lane / 16 * E), fa, acc[j]);
        }
    const int64_t row = m0 + wave * 16 + lane % 16;
    if (row >= p.m) return;
    for (int j = 0; j < (GATED ? 2 : 4); ++j)
        for (int e = 0; e < 4; ++e) {
            const int64_t col = n0 + j * 16 + lane / 16 * 4 + e;
            if (col >= p.n) continue;
            if (GATED) {
                float slope;
                const float g = acc[j][e], u = acc[j + 2][e];
                ((T*)p.out)[row * p.ldo + col] = (T)(act_value(g, p.act, slope) * u);
                if (p.pre) {
                    p.pre[row * 2 * p.n + col] = g;
                    p.pre[(row * 2 + 1) * p.n + col] = u;
                }
            } else if (row < p.split) {
                ((T*)p.out)[row * p.ldo + col] = (T)acc[j][e];
            } else {
                ((T*)p.out2)[(row - p.split) * p.ldo2 + col] = (T)acc[j][e];
            }
        }
}

// gradients of gate and up, [m][2][f] in T
template <typename T>
__global__ __launch_bounds__(256) void k_gated_slopes(const float* pre, const void* dh, int64_t ldh, int64_t m, int64_t f, int act, void* out)
{
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < m * f; i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / f, j = i - r * f;
        const float g = pre[r * 2 * f + j], u = pre[(r * 2 + 1) * f + j], d = (float)((const T*)dh)[r * ldh + j];
        float slope;
        const float a = act_value(g, act, slope);
        ((T*)out)[r * 2 * f + j] = (T)(d * u * slope);
        ((T*)out)[(r * 2 + 1) * f + j] = (T)(d * a);
    }
}

static int check_gated(int64_t m, int64_t k, int64_t f, int32_t dtype, int32_t activation)
{
    if (!known_type(dtype)) return fail(HR_ERR_ARG, "unknown dtype %d", dtype);
    if (m < 0 || m > HR_GATED_MAX) return fail(HR_ERR_ARG, "m=%lld must be in 0..%d", (long long)m, HR_GATED_MAX);
    if (k < 1 || k > HR_GATED_MAX) return fail(HR_ERR_ARG, "k=%lld must be in 1..%d", (long long)k, HR_GATED_MAX);
    if (f < 1 || f > HR_GATED_MAX) return fail(HR_ERR_ARG, "f=%lld must be in 1..%d", (long long)f, HR_GATED_MAX);
    if (activation < HR_SILU || activation > HR_GELU_TANH) return fail(HR_ERR_ARG, "unknown activation %d", activation);
    return HR_OK;
}

template <typename T, bool GATED>
static void launch(const ProductArgs& p, hipStream_t s)
{
    hipLaunchKernelGGL((k_product<T, GATED>), dim3((unsigned)((p.m + 63) / 64), (unsigned)((p.n + (GATED ? 31 : 63)) / (GATED ? 32 : 64))), dim3(256), 0, s, p);
}

}  // namespace hr

// ---- C entry points
using namespace hr;

extern "C" {

size_t hr_gated_workspace_bytes(int64_t m, int64_t k, int64_t f, int32_t dtype)
{
    if (check_gated(m, k, f, dtype, HR_SILU)) return 0;
    return HR_WORKSPACE_ALIGN;
}

int hr_gated(const void* x, int64_t ldx, const void* w_gate, int64_t ldwg, const void* w_up, int64_t ldwu, int32_t dtype, int64_t m, int64_t k,
             int64_t f, int32_t activation, void* out, int64_t ldo, float* out_pre, void* workspace, size_t workspace_bytes, void* stream)
{
    if (int rc = check_gated(m, k, f, dtype, activation)) return rc;
    const size_t es = element_bytes(dtype);
    if (int rc = check_matrix("x", x, m, k, ldx, es)) return rc;
    if (int rc = check_matrix("w_gate", w_gate, f, k, ldwg, es)) return rc;
    if (int rc = check_matrix("w_up", w_up, f, k, ldwu, es)) return rc;
    if (int rc = check_matrix("out", out, m, f, ldo, es)) return rc;
    if ((uintptr_t)out_pre % 4) return fail(HR_ERR_ARG, "out_pre is not aligned to its elements");
    if (m == 0) return HR_OK;
    if (int rc = check_workspace(workspace, workspace_bytes, hr_gated_workspace_bytes(m, k, f, dtype))) return rc;
    ProductArgs p{};
    p.a[0] = {x, ldx, 1};
    p.b[0] = {w_gate, ldwg, 1};
    p.b[1] = {w_up, ldwu, 1};
    p.m = m;
    p.n = f;
    p.k = k;
    p.out = out;
    p.ldo = ldo;
    p.pre = out_pre;
    p.act = activation;
    with_type(dtype, [&](auto t) { launch<decltype(t), true>(p, (hipStream_t)stream); });
    HR_HIP(hipGetLastError());
    return HR_OK;
}

size_t hr_gated_backward_workspace_bytes(int64_t m, int64_t k, int64_t f, int32_t dtype)
{
    if (check_gated(m, k, f, dtype, HR_SILU)) return 0;
    return aligned((size_t)(m * 2 * f) * element_bytes(dtype)) + HR_WORKSPACE_ALIGN;
}

int hr_gated_backward(const void* x, int64_t ldx, const void* w_gate, int64_t ldwg, const void* w_up, int64_t ldwu, int32_t dtype, int64_t m,
                      int64_t k, int64_t f, int32_t activation, const float* pre, const void* grad_out, int64_t ldgo, void* grad_x,
                      int64_t ldgx, void* grad_w_gate, int64_t ldgg, void* grad_w_up, int64_t ldgu, void* workspace, size_t workspace_bytes,
                      void* stream)
{
    if (int rc = check_gated(m, k, f, dtype, activation)) return rc;
    const size_t es = element_bytes(dtype);
    if (int rc = check_matrix("x", x, m, k, ldx, es)) return rc;
    if (int rc = check_matrix("w_gate", w_gate, f, k, ldwg, es)) return rc;
    if (int rc = check_matrix("w_up", w_up, f, k, ldwu, es)) return rc;
    if (int rc = check_matrix("grad_out", grad_out, m, f, ldgo, es)) return rc;
    if (m > 0 && !pre) return fail(HR_ERR_ARG, "pre is null");
    if ((uintptr_t)pre % 4) return fail(HR_ERR_ARG, "pre is not aligned to its elements");
    if (grad_x)
        if (int rc = check_matrix("grad_x", grad_x, m, k, ldgx, es)) return rc;
    if (!grad_w_gate != !grad_w_up) return fail(HR_ERR_ARG, "one of grad_w_gate and grad_w_up is null: want both or neither");
    if (grad_w_gate) {
        if (int rc = check_matrix("grad_w_gate", grad_w_gate, f, k, ldgg, es)) return rc;
        if (int rc = check_matrix("grad_w_up", grad_w_up, f, k, ldgu, es)) return rc;
    }
    if (int rc = check_workspace(workspace, workspace_bytes, hr_gated_backward_workspace_bytes(m, k, f, dtype))) return rc;
    hipStream_t s = (hipStream_t)stream;
    char* d = (char*)workspace;
    with_type(dtype, [&](auto t) {
        using T = decltype(t);
        if (m > 0) hipLaunchKernelGGL(k_gated_slopes<T>, dim3((unsigned)std::min<int64_t>((m * f + 255) / 256, 1 << 20)), dim3(256), 0, s, pre, grad_out, ldgo, m, f, activation, d);
        if (grad_x && m > 0) {
            ProductArgs p{};
            p.a[0] = {d, 2 * f, 1};
            p.a[1] = {d + f * es, 2 * f, 1};
            p.b[0] = {w_gate, 1, ldwg};
            p.b[1] = {w_up, 1, ldwu};
            p.stretches = 2;
            p.m = m;
            p.n = k;
            p.k = f;
            p.out = grad_x;
            p.ldo = ldgx;
            p.split = m;
            launch<T, false>(p, s);
        }
        if (grad_w_gate) {
            ProductArgs p{};
            p.a[0] = {d, 1, 2 * f};
            p.b[0] = {x, 1, ldx};
            p.stretches = 1;
            p.m = 2 * f;
            p.n = k;
            p.k = m;
            p.out = grad_w_gate;
            p.out2 = grad_w_up;
            p.ldo = ldgg;
            p.ldo2 = ldgu;
            p.split = f;
            launch<T, false>(p, s);
        }
    });
    HR_HIP(hipGetLastError());
    return HR_OK;
}

}  // extern "C"
