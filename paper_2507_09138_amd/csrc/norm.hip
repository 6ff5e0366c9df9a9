// Layer norm of rows and its gradients (hr_layers.h).
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "entry.h"
#include "hr_layers.h"
#include "wave.h"

// (what is subtracted here is a rounded product: with the product and the difference as one operation, a deviation would not be the same number in
// the sum that corrects the mean and in the result)
#pragma clang fp contract(off)

namespace hr {

struct NormArgs {
    const void* x; int64_t ldx, rows; int n;
    const void *weight, *bias;
    float eps;
    void* out; int64_t ldo; float* stats;
    // backward
    const void* dy; int64_t ldg;
    void* dx; int64_t ldgx;
    float* sums;                                         // long rows: [rows][2] sum g / n and sum g u / n
    float* parts;                                        // [groups][2][n] sums over some of the rows of dy u and of dy, or NULL
};

template <typename T> constexpr int kE = 16 / (int)sizeof(T);               // elements of a chunk
template <typename T> using Chunk = T __attribute__((ext_vector_type(16 / sizeof(T))));

// Chunk c of a row of n elements; zeros behind its end.  (Rows may begin at any element.)
template <typename T>
__device__ __forceinline__ Chunk<T> load_chunk(const T* row, int c, int n)
{
    constexpr int E = kE<T>;
    Chunk<T> v = {};
    if (c * E + E <= n) {
        __builtin_memcpy(&v, row + c * E, 16);
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (c * E + e < n) v[e] = row[c * E + e];
    }
    return v;
}
template <typename T>
__device__ __forceinline__ void store_chunk(T* row, int c, int n, const float* x)
{
    constexpr int E = kE<T>;
    Chunk<T> v;
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = (T)x[e];
    if (c * E + E <= n) {
        __builtin_memcpy(row + c * E, &v, 16);
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (c * E + e < n) row[c * E + e] = v[e];
    }
}
// E numbers of a vector of n, as floats; `other` where there is no vector or behind its end
template <int E, typename W>
__device__ __forceinline__ void load_weights(const void* at, int first, int n, float other, float* w)
{
#pragma unroll
    for (int e = 0; e < E; ++e) w[e] = at && first + e < n ? (float)((const W*)at)[first + e] : other;
}

template <typename C>
__device__ __forceinline__ float lane_swap(float v, C)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), C::value, 0xf, 0xf, false));
}
// The sum over the LANES lanes of a row, to all of them, in an order that depends on nothing but LANES.  More than a wave: through LDS, in
// one of two places by turns, so that one barrier a sum is enough (who writes a place has passed the barrier of the sum between).
struct Folds {
    float part[2][16][2];
};
template <int LANES>
__device__ __forceinline__ void fold_two(float& a, float& b, Folds& s, int& turn)
{
    auto fold = [](float v) __attribute__((always_inline)) {
        v += lane_swap(v, std::integral_constant<int, 0xb1>{});          // lane ^ 1
        v += lane_swap(v, std::integral_constant<int, 0x4e>{});          // lane ^ 2
        v += lane_swap(v, std::integral_constant<int, 0x141>{});         // the other four of eight
        v += lane_swap(v, std::integral_constant<int, 0x140>{});         // the other eight of sixteen
        if constexpr (LANES >= 64) {
            const int i = __builtin_bit_cast(int, v);
            auto of = [&](int l) __attribute__((always_inline)) { return __builtin_bit_cast(float, __builtin_amdgcn_readlane(i, l)); };
            v = (of(0) + of(16)) + (of(32) + of(48));
        }
        return v;
    };
    a = fold(a);
    b = fold(b);
    if constexpr (LANES > 64) {
        constexpr int WAVES = LANES / 64;
        float(*part)[2] = s.part[turn];
        turn ^= 1;
        if (lane_id() == 0) {
            part[threadIdx.x / 64][0] = a;
            part[threadIdx.x / 64][1] = b;
        }
        __syncthreads();
        a = b = 0.0f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) a += part[w][0], b += part[w][1];
    }
}

// ---- rows that LANES lanes hold, CH chunks of 16 bytes each, between their one read and their one write.  The mean is found first and the
// spread from what is left: the second fold also finds what the first mean is off by, so that a row far from 0 loses nothing.
template <typename T, typename W, int LANES, int CH>
__global__ __launch_bounds__(LANES > 256 ? LANES : 256) void k_norm(NormArgs a)
{
    constexpr int E = kE<T>, THREADS = LANES > 256 ? LANES : 256, ROWS = THREADS / LANES;
    constexpr bool KEEP = CH * E <= 16;                  // weights stay in registers from row to row
    __shared__ Folds folds;
    int turn = 0;
    const int t = threadIdx.x % LANES, n = a.n;
    const float over = 1.0f / (float)n;
    float w[KEEP ? CH : 1][E], b[KEEP ? CH : 1][E];
    auto weights = [&](int i, float* wi, float* bi) __attribute__((always_inline)) {
        load_weights<E, W>(a.weight, (i * LANES + t) * E, n, 1.0f, wi);
        load_weights<E, W>(a.bias, (i * LANES + t) * E, n, 0.0f, bi);
    };
    if constexpr (KEEP)
        for (int i = 0; i < CH; ++i) weights(i, w[i], b[i]);
    for (int64_t r0 = (int64_t)blockIdx.x * ROWS; r0 < a.rows; r0 += (int64_t)gridDim.x * ROWS) {
        const int64_t r = r0 + threadIdx.x / LANES;
        const bool in = r < a.rows;
        const T* row = (const T*)a.x + (in ? r : a.rows - 1) * a.ldx;
        Chunk<T> x[CH];
#pragma unroll
        for (int i = 0; i < CH; ++i) x[i] = load_chunk(row, i * LANES + t, n);
        float s0 = 0.0f, s1 = 0.0f;
#pragma unroll
        for (int i = 0; i < CH; ++i)
#pragma unroll
            for (int e = 0; e < E; ++e) s0 += (float)x[i][e];
        fold_two<LANES>(s0, s1, folds, turn);
        const float first = s0 * over;
        s0 = s1 = 0.0f;
#pragma unroll
        for (int i = 0; i < CH; ++i)
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float d = (i * LANES + t) * E + e < n ? (float)x[i][e] - first : 0.0f;
                s0 += d;
                s1 = fmaf(d, d, s1);
            }
        fold_two<LANES>(s0, s1, folds, turn);
        const float off = s0 * over, rstd = 1.0f / sqrtf(s1 * over - off * off + a.eps);
        if (!in) continue;
        if (t == 0 && a.stats) {
            a.stats[2 * r] = first + off;
            a.stats[2 * r + 1] = rstd;
        }
        T* out = (T*)a.out + r * a.ldo;
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            if ((i * LANES + t) * E >= n) continue;
            float wi[E], bi[E], y[E];
            if constexpr (!KEEP) weights(i, wi, bi);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                if constexpr (KEEP) wi[e] = w[i][e], bi[e] = b[i][e];
                y[e] = fmaf(((float)x[i][e] - first - off) * rstd, wi[e], bi[e]);
            }
            store_chunk(out, i * LANES + t, n, y);
        }
    }
}

// longer rows are read three times, by 1024 threads each
template <typename T, typename W>
__global__ __launch_bounds__(1024) void k_norm_long(NormArgs a)
{
    constexpr int E = kE<T>;
    __shared__ Folds folds;
    int turn = 0;
    const int n = a.n, chunks = (n + E - 1) / E;
    const float over = 1.0f / (float)n;
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const T* row = (const T*)a.x + r * a.ldx;
        float s0 = 0.0f, s1 = 0.0f;
        for (int c = threadIdx.x; c < chunks; c += 1024) {
            const Chunk<T> x = load_chunk(row, c, n);
#pragma unroll
            for (int e = 0; e < E; ++e) s0 += (float)x[e];
        }
        fold_two<1024>(s0, s1, folds, turn);
        const float first = s0 * over;
        s0 = s1 = 0.0f;
        for (int c = threadIdx.x; c < chunks; c += 1024) {
            const Chunk<T> x = load_chunk(row, c, n);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float d = c * E + e < n ? (float)x[e] - first : 0.0f;
                s0 += d;
                s1 = fmaf(d, d, s1);
            }
        }
        fold_two<1024>(s0, s1, folds, turn);
        const float off = s0 * over, rstd = 1.0f / sqrtf(s1 * over - off * off + a.eps);
        if (threadIdx.x == 0 && a.stats) {
            a.stats[2 * r] = first + off;
            a.stats[2 * r + 1] = rstd;
        }
        T* out = (T*)a.out + r * a.ldo;
        for (int c = threadIdx.x; c < chunks; c += 1024) {
            const Chunk<T> x = load_chunk(row, c, n);
            float w[E], b[E], y[E];
            load_weights<E, W>(a.weight, c * E, n, 1.0f, w);
            load_weights<E, W>(a.bias, c * E, n, 0.0f, b);
#pragma unroll
            for (int e = 0; e < E; ++e) y[e] = fmaf(((float)x[e] - first - off) * rstd, w[e], b[e]);
            store_chunk(out, c, n, y);
        }
    }
}

// ---- gradients of rows that LANES lanes hold; sums over the workgroup's rows stay in registers until its last
template <typename T, typename W, int LANES, int CH>
__global__ __launch_bounds__(LANES > 256 ? LANES : 256) void k_norm_backward(NormArgs a)
{
    constexpr int E = kE<T>, THREADS = LANES > 256 ? LANES : 256, ROWS = THREADS / LANES;
    __shared__ Folds folds;
    __shared__ float sums[ROWS > 1 ? ROWS * LANES * CH * E : 1];
    int turn = 0;
    const int t = threadIdx.x % LANES, n = a.n;
    const float over = 1.0f / (float)n;
    float w[CH][E], dw[CH][E] = {}, db[CH][E] = {};
    for (int i = 0; i < CH; ++i) load_weights<E, W>(a.weight, (i * LANES + t) * E, n, 1.0f, w[i]);
    for (int64_t r0 = (int64_t)blockIdx.x * ROWS; r0 < a.rows; r0 += (int64_t)gridDim.x * ROWS) {
        const int64_t r = r0 + threadIdx.x / LANES, at = min(r, a.rows - 1);
        const bool in = r < a.rows;
        Chunk<T> x[CH], dy[CH];
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            x[i] = load_chunk((const T*)a.x + at * a.ldx, i * LANES + t, n);
            dy[i] = load_chunk((const T*)a.dy + at * a.ldg, i * LANES + t, n);
        }
        const float mean = a.stats[2 * at], rstd = a.stats[2 * at + 1];
        float s0 = 0.0f, s1 = 0.0f;
#pragma unroll
        for (int i = 0; i < CH; ++i)
#pragma unroll
            for (int e = 0; e < E; ++e) {
                // (behind the row's end dy is 0, and u has to be a number)
                const float u = (i * LANES + t) * E + e < n ? ((float)x[i][e] - mean) * rstd : 0.0f, d = (float)dy[i][e], g = d * w[i][e];
                s0 += g;
                s1 = fmaf(g, u, s1);
                if (in) {
                    dw[i][e] = fmaf(d, u, dw[i][e]);
                    db[i][e] += d;
                }
            }
        fold_two<LANES>(s0, s1, folds, turn);
        const float c1 = s0 * over, c2 = s1 * over;
        if (!in || !a.dx) continue;
        T* out = (T*)a.dx + r * a.ldgx;
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            if ((i * LANES + t) * E >= n) continue;
            float y[E];
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float u = ((float)x[i][e] - mean) * rstd, g = (float)dy[i][e] * w[i][e];
                y[e] = rstd * (g - c1 - u * c2);
            }
            store_chunk(out, i * LANES + t, n, y);
        }
    }
    if (!a.parts) return;
    float* to = a.parts + (int64_t)blockIdx.x * 2 * n;
    auto write = [&](float(*x)[E], float* at) __attribute__((always_inline)) {
        if constexpr (ROWS > 1) {                        // the rows of the workgroup, in their order
            __syncthreads();
#pragma unroll
            for (int i = 0; i < CH; ++i)
#pragma unroll
                for (int e = 0; e < E; ++e) sums[(threadIdx.x / LANES) * LANES * CH * E + (i * LANES + t) * E + e] = x[i][e];
            __syncthreads();
            for (int j = threadIdx.x; j < n; j += THREADS) {
                float s = 0.0f;
#pragma unroll
                for (int q = 0; q < ROWS; ++q) s += sums[q * LANES * CH * E + j];
                at[j] = s;
            }
        } else {
#pragma unroll
            for (int i = 0; i < CH; ++i)
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if ((i * LANES + t) * E + e < n) at[(i * LANES + t) * E + e] = x[i][e];
        }
    };
    write(dw, to);
    write(db, to + n);
}

// ---- longer rows: the two sums of every row, then stripes of 256 chunks of columns, some of the rows each
template <typename T, typename W>
__global__ __launch_bounds__(1024) void k_norm_sums(NormArgs a)
{
    constexpr int E = kE<T>;
    __shared__ Folds folds;
    int turn = 0;
    const int n = a.n, chunks = (n + E - 1) / E;
    const float over = 1.0f / (float)n;
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const float mean = a.stats[2 * r], rstd = a.stats[2 * r + 1];
        float s0 = 0.0f, s1 = 0.0f;
        for (int c = threadIdx.x; c < chunks; c += 1024) {
            const Chunk<T> x = load_chunk((const T*)a.x + r * a.ldx, c, n), dy = load_chunk((const T*)a.dy + r * a.ldg, c, n);
            float w[E];
            load_weights<E, W>(a.weight, c * E, n, 1.0f, w);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float u = c * E + e < n ? ((float)x[e] - mean) * rstd : 0.0f, g = (float)dy[e] * w[e];
                s0 += g;
                s1 = fmaf(g, u, s1);
            }
        }
        fold_two<1024>(s0, s1, folds, turn);
        if (threadIdx.x == 0) {
            a.sums[2 * r] = s0 * over;
            a.sums[2 * r + 1] = s1 * over;
        }
    }
}
template <typename T, typename W>
__global__ __launch_bounds__(256) void k_norm_stripe(NormArgs a)
{
    constexpr int E = kE<T>;
    const int n = a.n, c = blockIdx.x * 256 + threadIdx.x;
    if (c * (int64_t)E >= n) return;
    float w[E], dw[E] = {}, db[E] = {};
    load_weights<E, W>(a.weight, c * E, n, 1.0f, w);
    for (int64_t r = blockIdx.y; r < a.rows; r += gridDim.y) {
        const Chunk<T> x = load_chunk((const T*)a.x + r * a.ldx, c, n), dy = load_chunk((const T*)a.dy + r * a.ldg, c, n);
        const float mean = a.stats[2 * r], rstd = a.stats[2 * r + 1], c1 = a.sums[2 * r], c2 = a.sums[2 * r + 1];
        float y[E];
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float u = ((float)x[e] - mean) * rstd, d = (float)dy[e];
            dw[e] = fmaf(d, u, dw[e]);
            db[e] += d;
            y[e] = rstd * (d * w[e] - c1 - u * c2);
        }
        if (a.dx) store_chunk((T*)a.dx + r * a.ldgx, c, n, y);
    }
    if (!a.parts) return;
    float* to = a.parts + (int64_t)blockIdx.y * 2 * n;
    for (int e = 0; e < E; ++e)
        if (c * E + e < n) to[c * E + e] = dw[e], to[n + c * E + e] = db[e];
}

// ---- the sums of the groups of rows, in their order: 16 threads for 64 columns, 16 shares of the groups
template <typename W>
__global__ __launch_bounds__(256) void k_norm_join(const float* parts, int groups, int n, void* grad_weight, void* grad_bias)
{
    __shared__ float sums[16][64];
    const int64_t all = 2 * (int64_t)n, col = (int64_t)blockIdx.x * 64;
    const int lane = threadIdx.x % 16 * 4, share = threadIdx.x / 16;
    float s[4] = {0, 0, 0, 0};
    for (int g = share; g < groups; g += 16)
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (col + lane + e < all) s[e] += parts[g * all + col + lane + e];
#pragma unroll
    for (int e = 0; e < 4; ++e) sums[share][lane + e] = s[e];
    __syncthreads();
    if (threadIdx.x < 64 && col + threadIdx.x < all) {
        float v = 0.0f;
        for (int q = 0; q < 16; ++q) v += sums[q][threadIdx.x];
        const int64_t j = col + threadIdx.x;
        void* to = j < n ? grad_weight : grad_bias;
        if (to) ((W*)to)[j < n ? j : j - n] = (W)v;
    }
}

// ---- which kernel
constexpr int kHeldColumns = 16384;                      // most columns of rows whose gradients workgroups hold
constexpr int kGroups = 512;                             // most workgroups of them
static int64_t groups_for(int64_t rows, int64_t n)
{
    const int64_t most = n <= kHeldColumns ? kGroups : std::max<int64_t>(1, (int64_t)kGroups * 4096 / n);
    return std::min(rows, most);
}

template <typename F>
static auto with_types(int dtype, int weight_dtype, F&& f)
{
    return with_type(dtype, [&](auto t) {
        using T = decltype(t);
        if (weight_dtype == HR_F32) return f(T{}, float{});
        return f(T{}, T{});
    });
}

template <typename T, typename W>
static void launch_norm(const NormArgs& a, hipStream_t s)
{
    const int64_t chunks = (a.n + kE<T> - 1) / kE<T>;
    auto go = [&](auto kernel, int threads, int rows) {
        const int64_t want = (a.rows + rows - 1) / rows, most = 256 * (2048 / threads);
        hipLaunchKernelGGL(kernel, dim3((unsigned)std::min(want, most)), dim3(threads), 0, s, a);
    };
    if (chunks <= 16) go(k_norm<T, W, 16, 1>, 256, 16);
    else if (chunks <= 32) go(k_norm<T, W, 16, 2>, 256, 16);
    else if (chunks <= 64) go(k_norm<T, W, 64, 1>, 256, 4);
    else if (chunks <= 128) go(k_norm<T, W, 64, 2>, 256, 4);
    else if (chunks <= 256) go(k_norm<T, W, 256, 1>, 256, 1);
    else if (chunks <= 512) go(k_norm<T, W, 256, 2>, 256, 1);
    else if (chunks <= 1024) go(k_norm<T, W, 256, 4>, 256, 1);
    else if (chunks <= 4096) go(k_norm<T, W, 1024, 4>, 1024, 1);
    else go(k_norm_long<T, W>, 1024, 1);
}

template <typename T, typename W>
static void launch_norm_backward(const NormArgs& a, void* grad_weight, void* grad_bias, hipStream_t s)
{
    const int64_t chunks = (a.n + kE<T> - 1) / kE<T>, most = groups_for(a.rows, a.n);
    int64_t groups = 0;
    auto go = [&](auto kernel, int threads, int rows) {
        groups = std::min((a.rows + rows - 1) / rows, most);
        hipLaunchKernelGGL(kernel, dim3((unsigned)groups), dim3(threads), 0, s, a);
    };
    if (a.rows == 0) {
    } else if (a.n > kHeldColumns) {
        hipLaunchKernelGGL((k_norm_sums<T, W>), dim3((unsigned)std::min<int64_t>(a.rows, 512)), dim3(1024), 0, s, a);
        groups = most;
        hipLaunchKernelGGL((k_norm_stripe<T, W>), dim3((unsigned)((chunks + 255) / 256), (unsigned)groups), dim3(256), 0, s, a);
    } else if (chunks <= 16) go(k_norm_backward<T, W, 16, 1>, 256, 16);
    else if (chunks <= 32) go(k_norm_backward<T, W, 16, 2>, 256, 16);
    else if (chunks <= 64) go(k_norm_backward<T, W, 64, 1>, 256, 4);
    else if (chunks <= 128) go(k_norm_backward<T, W, 64, 2>, 256, 4);
    else if (chunks <= 256) go(k_norm_backward<T, W, 256, 1>, 256, 1);
    else if (chunks <= 512) go(k_norm_backward<T, W, 256, 2>, 256, 1);
    else if (chunks <= 1024) go(k_norm_backward<T, W, 512, 2>, 512, 1);
    else if (chunks <= 2048) go(k_norm_backward<T, W, 1024, 2>, 1024, 1);
    else if constexpr (sizeof(T) == 4) go(k_norm_backward<T, W, 1024, 4>, 1024, 1);
    if (a.parts || a.rows == 0) {
        if (!grad_weight && !grad_bias) return;
        hipLaunchKernelGGL(k_norm_join<W>, dim3((unsigned)((2 * (int64_t)a.n + 63) / 64)), dim3(256), 0, s, a.parts, (int)groups, a.n, grad_weight, grad_bias);
    }
}

static int check_norm(const void* x, int64_t ldx, int32_t dtype, int64_t rows, int64_t n, int32_t weight_dtype)
{
    if (!known_type(dtype)) return fail(HR_ERR_ARG, "unknown dtype %d", dtype);
    if (weight_dtype != HR_F32 && weight_dtype != dtype) return fail(HR_ERR_ARG, "weight_dtype %d: want float32 or that of x", weight_dtype);
    if (rows < 0 || rows > (1LL << 31) - 1) return fail(HR_ERR_ARG, "rows=%lld out of range", (long long)rows);
    if (n < 1 || n > HR_ROW_MAX) return fail(HR_ERR_ARG, "n=%lld must be in 1..%d", (long long)n, HR_ROW_MAX);
    return check_matrix("x", x, rows, n, ldx, element_bytes(dtype));
}
static int check_vector(const char* name, const void* p, int32_t dtype)
{
    return (uintptr_t)p % element_bytes(dtype) ? fail(HR_ERR_ARG, "%s is not aligned to its elements", name) : HR_OK;
}

}  // namespace hr

// ---- C entry points
using namespace hr;

extern "C" {

int hr_layer_norm(const void* x, int64_t ldx, int32_t dtype, int64_t rows, int64_t n, const void* weight, const void* bias,
                  int32_t weight_dtype, float eps, void* out, int64_t ldo, float* out_stats, void* stream)
{
    if (int rc = check_norm(x, ldx, dtype, rows, n, weight_dtype)) return rc;
    if (!(eps >= 0) || !std::isfinite(eps)) return fail(HR_ERR_ARG, "eps=%g", (double)eps);
    if (int rc = check_matrix("out", out, rows, n, ldo, element_bytes(dtype))) return rc;
    if (out == x && ldo != ldx && rows > 1) return fail(HR_ERR_ARG, "out is x with another distance between rows");
    if (int rc = check_vector("weight", weight, weight_dtype)) return rc;
    if (int rc = check_vector("bias", bias, weight_dtype)) return rc;
    if (int rc = check_vector("out_stats", out_stats, HR_F32)) return rc;
    if (rows == 0) return HR_OK;
    NormArgs a{x, ldx, rows, (int)n, weight, bias, eps, out, ldo, out_stats};
    with_types(dtype, weight_dtype, [&](auto t, auto w) { launch_norm<decltype(t), decltype(w)>(a, (hipStream_t)stream); });
    HR_HIP(hipGetLastError());
    return HR_OK;
}

size_t hr_layer_norm_workspace_bytes(int64_t rows, int64_t n)
{
    if (check_norm(nullptr, n, HR_F32, rows < 0 ? -1 : 0, n, HR_F32) || rows > (1LL << 31) - 1) return 0;
    return aligned((size_t)(groups_for(rows, n) * 2 * n * 4)) + aligned((size_t)rows * 8) + HR_WORKSPACE_ALIGN;
}

int hr_layer_norm_backward(const void* x, int64_t ldx, int32_t dtype, int64_t rows, int64_t n, const void* weight, int32_t weight_dtype,
                           const float* stats, const void* grad_out, int64_t ldg, void* grad_x, int64_t ldgx, void* grad_weight,
                           void* grad_bias, void* workspace, size_t workspace_bytes, void* stream)
{
    if (int rc = check_norm(x, ldx, dtype, rows, n, weight_dtype)) return rc;
    const size_t es = element_bytes(dtype);
    if (int rc = check_matrix("grad_out", grad_out, rows, n, ldg, es)) return rc;
    if (grad_x)
        if (int rc = check_matrix("grad_x", grad_x, rows, n, ldgx, es)) return rc;
    if (grad_x && grad_x == grad_out && ldgx != ldg && rows > 1) return fail(HR_ERR_ARG, "grad_x is grad_out with another distance between rows");
    if (rows > 0 && !stats) return fail(HR_ERR_ARG, "stats is null");
    if (int rc = check_vector("stats", stats, HR_F32)) return rc;
    if (int rc = check_vector("weight", weight, weight_dtype)) return rc;
    if (int rc = check_vector("grad_weight", grad_weight, weight_dtype)) return rc;
    if (int rc = check_vector("grad_bias", grad_bias, weight_dtype)) return rc;
    if (int rc = check_workspace(workspace, workspace_bytes, hr_layer_norm_workspace_bytes(rows, n))) return rc;
    NormArgs a{x, ldx, rows, (int)n, weight, nullptr, 0, nullptr, 0, const_cast<float*>(stats), grad_out, ldg, grad_x, ldgx};
    a.sums = (float*)workspace;
    if (grad_weight || grad_bias) a.parts = (float*)((char*)workspace + aligned((size_t)rows * 8));
    with_types(dtype, weight_dtype, [&](auto t, auto w) { launch_norm_backward<decltype(t), decltype(w)>(a, grad_weight, grad_bias, (hipStream_t)stream); });
    HR_HIP(hipGetLastError());
    return HR_OK;
}

}  // extern "C"
