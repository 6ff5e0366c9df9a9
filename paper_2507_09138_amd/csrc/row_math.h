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
    using V = T __attribute__((ext_vector_type(E)));
    const T* z;
    int n, before, nchunks;             // before: places of chunk 0 in front of the row
    int lo, hi;                         // chunks lo .. hi-1 are the row's throughout

    __device__ __forceinline__ Row(const void* base, int64_t offset, int n_) : z((const T*)base + offset), n(n_)
    {
        before = (int)(((uintptr_t)z & 15) / sizeof(T));
        nchunks = (int)(((int64_t)before + n + E - 1) / E);
        lo = before > 0;
        hi = (int)(((int64_t)before + n) / E);
    }
    __device__ __forceinline__ int first(int c) const { return c * E - before; }      // entry of a chunk's first place
    // A chunk as it lies in memory; what lies at the edges or behind the row is some other chunk of it, to be replaced by fix().
    // (A row that is no whole chunk has nothing that could be loaded: 0.)
    __device__ __forceinline__ V raw(int c) const
    {
        if (hi <= lo) return V{};
        c = c < lo ? lo : (c < hi ? c : hi - 1);
        return *(const V*)(z + first(c));
    }
    // The same where the chunk is the row's in part or not at all: -inf in the places that are not.
    __device__ __forceinline__ void fix(int c, float* v) const
    {
        if (c >= lo && c < hi) return;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int i = first(c) + e;
            v[e] = c < nchunks && i >= 0 && i < n ? (float)z[i] : -INFINITY;
        }
    }
    __device__ __forceinline__ void unpack(int c, V t, float* v) const
    {
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = (float)t[e];
        fix(c, v);
    }
    __device__ __forceinline__ int load(int c, float* v) const
    {
        unpack(c, raw(c), v);
        return first(c);
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
    // a chunk, top its largest score
    template <int E, bool ENTROPY>
    __device__ __forceinline__ void add(const float* v, float top, float c2)
    {
        if (top > m) rescale(top, c2);
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float x = (v[e] - m) * c2, t = __builtin_amdgcn_exp2f(x);
            s0 += t;
            if (ENTROPY) s1 = fmaf(fmaxf(x, kLowest2), t, s1);
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

// Largest scores of stretches of a row: what the search for its best entries starts from.  A slot is 2^shift chunks.
template <int THREADS>
struct Slots {
    static constexpr int kMax = 4 * THREADS;
    uint32_t key[kMax];
    // few enough slots: chunks one by one, or 2, 4, 8, 16 .. of them together
    static __host__ __device__ int shift_for(int nchunks)
    {
        int s = 0;
        while (nchunks > kMax << s) ++s;
        return s;
    }
};

// largest of 2^min(shift, 4) neighbouring lanes
__device__ __forceinline__ float neighbours_max(float v, int shift)
{
    auto step = [&](auto ctrl) __attribute__((always_inline)) {
        v = fmaxf(v, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), decltype(ctrl)::value, 0xf, 0xf, false)));
    };
    using std::integral_constant;
    if (shift >= 1) step(integral_constant<int, 0xb1>{});       // quad_perm: lane ^ 1
    if (shift >= 2) step(integral_constant<int, 0x4e>{});       // quad_perm: lane ^ 2
    if (shift >= 3) step(integral_constant<int, 0x141>{});      // row_half_mirror: the other four of eight lanes
    if (shift >= 4) step(integral_constant<int, 0x140>{});      // row_mirror: the other eight of sixteen
    return v;
}

// Maximum and sums of chunks begin .. end-1 of a row (begin a multiple of 16), to all threads of a workgroup.  A thread asks for
// four chunks at a time; with several waves per SIMD that is enough under way.  TOP: the slots' largest scores as well
// (slots of the row's chunk 0 on; they have to be cleared before if shift > 4).
template <typename T, int THREADS, bool ENTROPY, bool TOP>
__device__ __forceinline__ RowStat row_stats(const Row<T>& row, int begin, int end, float c2, RowShared<THREADS>& sh, uint32_t* slots, int shift)
{
    constexpr int U = 4, E = Row<T>::E;
    RowStat st;
    st.clear();
    for (int c0 = begin; c0 < end; c0 += U * THREADS) {
        typename Row<T>::V raw[U];
#pragma unroll
        for (int u = 0; u < U; ++u) raw[u] = row.raw(c0 + u * THREADS + (int)threadIdx.x);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int c = c0 + u * THREADS + (int)threadIdx.x;
            if (c0 + u * THREADS < end) {
                float v[E];
                row.unpack(c < end ? c : row.nchunks, raw[u], v);
                float top = v[0];
#pragma unroll
                for (int e = 1; e < E; ++e) top = fmaxf(top, v[e]);
                st.template add<E, ENTROPY>(v, top, c2);
                if (TOP) {
                    top = neighbours_max(top, shift);
                    if (c < end && (c & ((1 << (shift < 4 ? shift : 4)) - 1)) == 0) {
                        if (shift <= 4) slots[c >> shift] = order_key(top);
                        else atomicMax(&slots[c >> shift], order_key(top));
                    }
                }
            }
        }
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
