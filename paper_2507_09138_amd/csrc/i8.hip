// Products in 8-bit integers with a scale for each row of both matrices, and the quantisation of rows (hr_scores.h).
#include "entry.h"
#include "row_math.h"

namespace hr {

typedef int intx4 __attribute__((ext_vector_type(4)));

struct QuantizeArgs {
    const void* x; int64_t ldx, m; int k;
    int8_t* q; int64_t ldq; float* scale;
};

// A row's scale, from the largest magnitude in it and whether it holds a NaN or an infinity.
__device__ __forceinline__ float quant_scale(float top, bool bad) { return bad ? NAN : top / 127.0f; }
__device__ __forceinline__ int quant(float v, float scale) { return scale > 0.0f ? (int)rintf(v / scale) : 0; }

template <typename T, int THREADS>
__global__ __launch_bounds__(THREADS) void k_quantize(QuantizeArgs a)
{
    constexpr int E = Row<T>::E;
    __shared__ RowShared<THREADS> sh;
    for (int64_t r = blockIdx.x; r < a.m; r += gridDim.x) {
        const Row<T> row(a.x, r * a.ldx, a.k);
        float top = 0.0f;
        bool bad = false;
        for (int c = threadIdx.x; c < row.nchunks; c += THREADS) {
            float v[E];
            const int first = row.load(c, v);
            for (int e = 0; e < E; ++e) {
                const bool in = first + e >= 0 && first + e < a.k;
                top = fmaxf(top, in ? fabsf(v[e]) : 0.0f);
                bad |= in && !(fabsf(v[e]) <= FLT_MAX);
            }
        }
        top = group_max<THREADS>(top, sh);
        bad = __syncthreads_or(bad);
        const float scale = quant_scale(top, bad);
        if (threadIdx.x == 0) a.scale[r] = scale;
        int8_t* q = a.q + r * a.ldq;
        for (int c = threadIdx.x; c < row.nchunks; c += THREADS) {
            float v[E];
            const int first = row.load(c, v);
            for (int e = 0; e < E; ++e)
                if (first + e >= 0 && first + e < a.k) q[first + e] = (int8_t)quant(v[e], scale);
        }
        const int64_t padded = (a.k + 63LL) / 64 * 64, end = padded < a.ldq ? padded : a.ldq;
        for (int64_t i = a.k + threadIdx.x; i < end; i += THREADS) q[i] = 0;
    }
}

struct ProductArgs {
    const int8_t* a; int64_t lda; const float* a_scale;
    const int8_t* b; int64_t ldb; const float* b_scale;
    const float* bias;
    int64_t m, n; int k;
    void* out; int64_t ldo;
};

// The value of an output: the exact sum, scaled and rounded once.
__device__ __forceinline__ float scaled_sum(int sum, float sa, float sb, bool has_bias, float bias)
{
    const float v = (float)sum * sa;
    return has_bias ? fmaf(v, sb, bias) : v * sb;
}

// 16 bytes of a row from byte t on, zeros from byte k on; rows may start anywhere
__device__ __forceinline__ u32x4 load16(const int8_t* row, int t, int k)
{
    u32x4 v = {0, 0, 0, 0};
    if (t + 16 <= k) {
        __builtin_memcpy(&v, row + t, 16);
    } else {
        uint32_t w[4] = {0, 0, 0, 0};
        for (int i = 0; i < 16; ++i)
            if (t + i < k) w[i >> 2] |= (uint32_t)(uint8_t)row[t + i] << (8 * (i & 3));
        v = u32x4{w[0], w[1], w[2], w[3]};
    }
    return v;
}

// Tiles of 64 x 64 outputs, four waves of 32 x 32, blocks of 64 bytes of k staged through registers: rows of any alignment.
template <typename O>
__global__ __launch_bounds__(256) void k_i8_product_any(ProductArgs p)
{
    constexpr int kStride = 80;                         // bytes between rows in LDS: 16 rows at 16 different banks
    __shared__ __align__(16) int8_t ta[64 * kStride], tb[64 * kStride];
    const int64_t tiles_m = (p.m + 63) / 64;
    const int64_t m0 = (int64_t)(blockIdx.x % tiles_m) * 64, n0 = (int64_t)(blockIdx.x / tiles_m) * 64;
    const int lane = lane_id(), wave = threadIdx.x / 64, wm = wave % 2 * 32, wn = wave / 2 * 32;
    const int lr = threadIdx.x / 4, lc = threadIdx.x % 4 * 16;          // what this thread loads
    const int8_t* ra = m0 + lr < p.m ? p.a + (m0 + lr) * p.lda : nullptr;
    const int8_t* rb = n0 + lr < p.n ? p.b + (n0 + lr) * p.ldb : nullptr;
    intx4 acc[2][2] = {};
    for (int t = 0; t < p.k; t += 64) {
        const u32x4 zero = {0, 0, 0, 0};
        const u32x4 va = ra ? load16(ra, t + lc, p.k) : zero, vb = rb ? load16(rb, t + lc, p.k) : zero;
        __syncthreads();
        *(u32x4*)(ta + lr * kStride + lc) = va;
        *(u32x4*)(tb + lr * kStride + lc) = vb;
        __syncthreads();
        intx4 fa[2], fb[2];
        for (int i = 0; i < 2; ++i) {
            fa[i] = *(const intx4*)(ta + (wm + i * 16 + lane % 16) * kStride + lane / 16 * 16);
            fb[i] = *(const intx4*)(tb + (wn + i * 16 + lane % 16) * kStride + lane / 16 * 16);
        }
        for (int i = 0; i < 2; ++i)
            for (int j = 0; j < 2; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fb[j], fa[i], acc[i][j], 0, 0, 0);
    }
    for (int i = 0; i < 2; ++i) {
        const int64_t row = m0 + wm + i * 16 + lane % 16;
        if (row >= p.m) continue;
        const float sa = p.a_scale[row];
        for (int j = 0; j < 2; ++j)
            for (int e = 0; e < 4; ++e) {
                const int64_t col = n0 + wn + j * 16 + lane / 16 * 4 + e;
                if (col < p.n) ((O*)p.out)[row * p.ldo + col] = (O)scaled_sum(acc[i][j][e], sa, p.b_scale[col], p.bias, p.bias ? p.bias[col] : 0.0f);
            }
    }
}

static hipError_t launch_quantize(int dtype, const QuantizeArgs& a, hipStream_t s)
{
    const dim3 grid((unsigned)(a.m < (1 << 20) ? a.m : 1 << 20)), block(256);
    switch (dtype) {
    case HR_F32: hipLaunchKernelGGL((k_quantize<float, 256>), grid, block, 0, s, a); break;
    case HR_F16: hipLaunchKernelGGL((k_quantize<_Float16, 256>), grid, block, 0, s, a); break;
    default: hipLaunchKernelGGL((k_quantize<__bf16, 256>), grid, block, 0, s, a); break;
    }
    return hipGetLastError();
}

static hipError_t launch_product(int dtype, const ProductArgs& p, hipStream_t s)
{
    const dim3 grid((unsigned)((p.m + 63) / 64 * ((p.n + 63) / 64))), block(256);
    switch (dtype) {
    case HR_F32: hipLaunchKernelGGL(k_i8_product_any<float>, grid, block, 0, s, p); break;
    case HR_F16: hipLaunchKernelGGL(k_i8_product_any<_Float16>, grid, block, 0, s, p); break;
    default: hipLaunchKernelGGL(k_i8_product_any<__bf16>, grid, block, 0, s, p); break;
    }
    return hipGetLastError();
}

}  // namespace hr

// ---- C entry points
using namespace hr;

static bool known_type(int32_t dtype) { return dtype == HR_F32 || dtype == HR_F16 || dtype == HR_BF16; }

static int check_matrix(const char* name, const void* p, int64_t rows, int64_t k, int64_t ld, size_t es)
{
    if (rows > 0 && !p) return fail(HR_ERR_ARG, "%s is null", name);
    if (ld < k || ld > (1LL << 40)) return fail(HR_ERR_ARG, "rows of %s: %lld elements, %lld apart", name, (long long)k, (long long)ld);
    if ((uintptr_t)p % es) return fail(HR_ERR_ARG, "%s is not aligned to its elements", name);
    return HR_OK;
}

static int check_shape(int64_t m, int64_t n, int64_t k)
{
    if (m < 0 || m > (1 << 24)) return fail(HR_ERR_ARG, "m=%lld out of range", (long long)m);
    if (n < 0 || n > (1LL << 31) - 1) return fail(HR_ERR_ARG, "n=%lld out of range", (long long)n);
    if (k < 1 || k > HR_I8_K_MAX) return fail(HR_ERR_ARG, "k=%lld must be in 1..%d", (long long)k, HR_I8_K_MAX);
    // (tiles of 64 x 64 outputs, and a launch may not have 2^32 threads)
    if ((m + 63) / 64 * ((n + 63) / 64) >= (1LL << 24)) return fail(HR_ERR_UNSUPPORTED, "m=%lld x n=%lld: more outputs than one call takes", (long long)m, (long long)n);
    return HR_OK;
}

// workspace: the quantised rows of hr_i8_linear, then their scales
static int64_t padded_k(int64_t k) { return (k + 63) / 64 * 64; }
static size_t aligned(size_t bytes) { return (bytes + HR_WORKSPACE_ALIGN - 1) / HR_WORKSPACE_ALIGN * HR_WORKSPACE_ALIGN; }

extern "C" {

int hr_i8_quantize(const void* x, int64_t ldx, int32_t dtype, int64_t m, int64_t k, int8_t* q, int64_t ldq, float* scale, void* stream)
{
    if (!known_type(dtype)) return fail(HR_ERR_ARG, "unknown dtype %d", dtype);
    if (m < 0 || m > (1LL << 31) - 1) return fail(HR_ERR_ARG, "m=%lld out of range", (long long)m);
    if (k < 1 || k > HR_ROW_MAX) return fail(HR_ERR_ARG, "k=%lld must be in 1..%d", (long long)k, HR_ROW_MAX);
    if (int rc = check_matrix("x", x, m, k, ldx, element_bytes(dtype))) return rc;
    if (int rc = check_matrix("q", q, m, k, ldq, 1)) return rc;
    if (m == 0) return HR_OK;
    if (!scale) return fail(HR_ERR_ARG, "scale is null");
    QuantizeArgs a{x, ldx, m, (int)k, q, ldq, scale};
    HR_HIP(launch_quantize(dtype, a, (hipStream_t)stream));
    return HR_OK;
}

size_t hr_i8_workspace_bytes(int64_t m, int64_t n, int64_t k)
{
    if (check_shape(m, n, k)) return 0;
    return aligned((size_t)(m * padded_k(k))) + aligned((size_t)m * 4) + HR_WORKSPACE_ALIGN;
}

int hr_i8_product(const int8_t* a, int64_t lda, const float* a_scale, const int8_t* b, int64_t ldb, const float* b_scale,
                  const float* bias, int64_t m, int64_t n, int64_t k, void* out, int64_t ldo, int32_t out_dtype,
                  void* workspace, size_t workspace_bytes, void* stream)
{
    if (!known_type(out_dtype)) return fail(HR_ERR_ARG, "unknown out_dtype %d", out_dtype);
    if (int rc = check_shape(m, n, k)) return rc;
    if (int rc = check_matrix("a", a, m, k, lda, 1)) return rc;
    if (int rc = check_matrix("b", b, n, k, ldb, 1)) return rc;
    if (int rc = check_matrix("out", out, m && n, n, ldo, element_bytes(out_dtype))) return rc;
    if (m == 0 || n == 0) return HR_OK;
    if (!a_scale || !b_scale) return fail(HR_ERR_ARG, "a_scale / b_scale is null");
    if (int rc = check_workspace(workspace, workspace_bytes, hr_i8_workspace_bytes(m, n, k))) return rc;
    ProductArgs p{a, lda, a_scale, b, ldb, b_scale, bias, m, n, (int)k, out, ldo};
    HR_HIP(launch_product(out_dtype, p, (hipStream_t)stream));
    return HR_OK;
}

int hr_i8_linear(const void* x, int64_t ldx, int32_t x_dtype, const int8_t* b, int64_t ldb, const float* b_scale,
                 const float* bias, int64_t m, int64_t n, int64_t k, void* out, int64_t ldo, int32_t out_dtype,
                 void* workspace, size_t workspace_bytes, void* stream)
{
    if (!known_type(x_dtype)) return fail(HR_ERR_ARG, "unknown x_dtype %d", x_dtype);
    if (!known_type(out_dtype)) return fail(HR_ERR_ARG, "unknown out_dtype %d", out_dtype);
    if (int rc = check_shape(m, n, k)) return rc;
    if (int rc = check_matrix("x", x, m, k, ldx, element_bytes(x_dtype))) return rc;
    if (int rc = check_matrix("b", b, n, k, ldb, 1)) return rc;
    if (int rc = check_matrix("out", out, m && n, n, ldo, element_bytes(out_dtype))) return rc;
    if (m == 0 || n == 0) return HR_OK;
    if (!b_scale) return fail(HR_ERR_ARG, "b_scale is null");
    if (int rc = check_workspace(workspace, workspace_bytes, hr_i8_workspace_bytes(m, n, k))) return rc;
    int8_t* q = (int8_t*)workspace;
    float* scale = (float*)(q + aligned((size_t)(m * padded_k(k))));
    QuantizeArgs qa{x, ldx, m, (int)k, q, padded_k(k), scale};
    HR_HIP(launch_quantize(x_dtype, qa, (hipStream_t)stream));
    ProductArgs p{q, padded_k(k), scale, b, ldb, b_scale, bias, m, n, (int)k, out, ldo};
    HR_HIP(launch_product(out_dtype, p, (hipStream_t)stream));
    return HR_OK;
}

}  // extern "C"
