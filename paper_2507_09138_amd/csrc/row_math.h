// Rows of scores: how they are read in chunks of 16 bytes, their maximum and sums, and folds over a workgroup.
#pragma once
#include <float.h>
#include <math.h>

#include "common.h"
#include "hr_scores.h"
#include "wave.h"

namespace hr {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kLowest2 = -2000.0f;                 // 2^kLowest2 is 0, and products with it stay finite

template <typename T> using vec_of = T __attribute__((ext_vector_type(16 / sizeof(T))));       // 16 bytes

// Scores as whole numbers in the same order (-0 and +0 alike); everything at or below kNoCandidate is -inf.
constexpr uint32_t kNoCandidate = 0x007fffffu;
__device__ __forceinline__ uint32_t order_key(float z)
{
    const uint32_t b = __builtin_bit_cast(uint32_t, z + 0.0f);
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float order_value(uint32_t key)
{
    return __builtin_bit_cast(float, key ^ ((uint32_t)((int32_t)~key >> 31) | 0x80000000u));
}

// A row of n scores.  Chunks are the 16-byte pieces of memory it lies in, so that every load is aligned wherever the row
// starts; the first and the last may hold fewer of its entries.
template <typename T>
struct Row {
    static constexpr int E = 16 / sizeof(T);
    const T* z;
    int n, before, nchunks;             // before: places of chunk 0 in front of the row

    __device__ __forceinline__ Row(const void* base, int64_t offset, int n_) : z((const T*)base + offset), n(n_)
    {
        before = (int)(((uintptr_t)z & 15) / sizeof(T));
        nchunks = (int)(((int64_t)before + n + E - 1) / E);
    }
    // scores of chunk c, -inf where it is not the row's; returns the entry of its first place (negative in front of the row)
    __device__ __forceinline__ int load(int c, float* v) const
    {
        const int first = c * E - before;
        if (first >= 0 && first + E <= n) {
            const vec_of<T> t = *(const vec_of<T>*)(z + first);
#pragma unroll
            for (int e = 0; e < E; ++e) v[e] = (float)t[e];
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e) v[e] = first + e >= 0 && first + e < n ? (float)z[first + e] : -INFINITY;
        }
        return first;
    }
    __device__ __forceinline__ float at(int64_t i) const { return i >= 0 && i < n ? (float)z[i] : -INFINITY; }
};

// A chunk that Row::load read, to a row of the output; vector stores where that row is aligned as well.
template <typename T>
__device__ __forceinline__ void store_chunk(T* out, int n, int first, const float* v)
{
    constexpr int E = 16 / sizeof(T);
    if (first >= 0 && first + E <= n && ((uintptr_t)(out + first) & 15) == 0) {
        vec_of<T> t;
#pragma unroll
        for (int e = 0; e < E; ++e) t[e] = (T)v[e];
        *(vec_of<T>*)(out + first) = t;
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (first + e >= 0 && first + e < n) out[first + e] = (T)v[e];
    }
}

template <int THREADS>
struct RowShared {
    static constexpr int kWaves = THREADS / 64;
    float part[3][kWaves];
};
struct ListShared {
    int id[HR_LIST_MAX];
    float c[HR_LIST_MAX], z[HR_LIST_MAX];
};

// Sum / largest over a workgroup, to all threads, in the same order every time.
template <int THREADS, typename F>
__device__ __forceinline__ float group_fold(float v, RowShared<THREADS>& sh, F f)
{
    for (int d = 32; d > 0; d >>= 1) v = f(v, __shfl_xor(v, d));
    if (THREADS > 64) {
        __syncthreads();
        if (lane_id() == 0) sh.part[0][threadIdx.x / 64] = v;
        __syncthreads();
        v = sh.part[0][0];
        for (int w = 1; w < THREADS / 64; ++w) v = f(v, sh.part[0][w]);
    }
    return v;
}
template <int THREADS>
__device__ __forceinline__ float group_sum(float v, RowShared<THREADS>& sh) { return group_fold<THREADS>(v, sh, [](float x, float y) { return x + y; }); }
// (a NaN stays: what is compared with it is not larger)
template <int THREADS>
__device__ __forceinline__ float group_max(float v, RowShared<THREADS>& sh) { return group_fold<THREADS>(v, sh, [](float x, float y) { return fmaxf(x, y); }); }

// Maximum and sums of scores.  An empty one has the lowest finite number as its maximum, so that differences from it are
// -inf or finite, never NaN, except where a score is NaN or +inf: then S0 becomes NaN and stays it.
struct RowStat {
    float m, s0, s1;                    // s1 in base 2

    __device__ __forceinline__ void clear() { m = -FLT_MAX; s0 = s1 = 0.0f; }
    __device__ __forceinline__ void rescale(float to, float c2)
    {
        const float d = fmaxf((m - to) * c2, kLowest2), f = __builtin_amdgcn_exp2f(d);
        s1 = f * fmaf(d, s0, s1);
        s0 *= f;
        m = to;
    }
    template <int E>
    __device__ __forceinline__ void add(const float* v, float c2)
    {
        float top = m;
#pragma unroll
        for (int e = 0; e < E; ++e) top = fmaxf(top, v[e]);
        if (top > m) rescale(top, c2);
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float x = (v[e] - m) * c2, t = __builtin_amdgcn_exp2f(x);
            s0 += t;
            s1 = fmaf(fmaxf(x, kLowest2), t, s1);
        }
    }
    __device__ __forceinline__ void merge(float m2, float a, float b, float c2)
    {
        RowStat o{m2, a, b};
        const float top = fmaxf(m, m2);
        if (m < top) rescale(top, c2);
        if (m2 < top) o.rescale(top, c2);
        s0 += o.s0;
        s1 += o.s1;
    }
    __device__ __forceinline__ float top() const { return s0 == 0.0f ? -INFINITY : m; }
    __device__ __forceinline__ float log_sum() const { return s0 == 0.0f ? 0.0f : logf(s0); }
    // (rounding may leave a sharp row a little below 0)
    __device__ __forceinline__ float entropy(float logsum) const
    {
        if (s0 == 0.0f) return 0.0f;
        const float h = logsum - kLn2 * (s1 / s0);
        return h < 0.0f ? 0.0f : h;
    }
    __device__ __forceinline__ float log_p(float z, float scale, float logsum) const
    {
        return z == -INFINITY ? -INFINITY : (z - m) * scale - logsum;
    }
};

// of a whole row, to all threads of a workgroup
template <typename T, int THREADS>
__device__ __forceinline__ RowStat row_stats(const Row<T>& row, float c2, RowShared<THREADS>& sh)
{
    RowStat st;
    st.clear();
    for (int c = threadIdx.x; c < row.nchunks; c += THREADS) {
        float v[Row<T>::E];
        row.load(c, v);
        st.template add<Row<T>::E>(v, c2);
    }
    for (int d = 32; d > 0; d >>= 1) st.merge(__shfl_xor(st.m, d), __shfl_xor(st.s0, d), __shfl_xor(st.s1, d), c2);
    if (THREADS > 64) {
        const int w = threadIdx.x / 64;
        __syncthreads();
        if (lane_id() == 0) { sh.part[0][w] = st.m; sh.part[1][w] = st.s0; sh.part[2][w] = st.s1; }
        __syncthreads();
        st = RowStat{sh.part[0][0], sh.part[1][0], sh.part[2][0]};
        for (int i = 1; i < THREADS / 64; ++i) st.merge(sh.part[0][i], sh.part[1][i], sh.part[2][i], c2);
    }
    return st;
}

struct LogprobsArgs {
    const void* logits; int64_t ld, rows; int n; float scale;
    const int64_t* given; int ngiven, k;
    float *logprobs, *entropy, *norm; int64_t* top_ids; float* top_logprobs;
};
struct LogprobsBackwardArgs {
    const void* logits; int64_t ld, rows; int n; float scale;
    const int64_t* given; int ngiven;
    const float *entropy, *norm, *grad_logprobs, *grad_entropy;
    void* grad; int64_t ldg;
};
struct DistillArgs {
    const void* logits; int64_t ld, rows; int n; float scale;
    const int64_t* ids; const float* teacher; int k;
    const float* weights;
    float *loss, *norm, *q;
    void* grad; int64_t ldg;
};

}  // namespace hr
