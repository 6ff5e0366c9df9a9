// Rows of scores: how they are read in chunks of 16 bytes, their maximum and sums, and folds over a workgroup.
#pragma once
#include <float.h>
#include <math.h>

#include "common.h"
#include "hr_scores.h"
#include "wave.h"

namespace hr {

typedef int intx4 __attribute__((ext_vector_type(4)));

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
// starts.  Chunks lo .. hi-1 are the row's throughout; what it has of the chunk before and of the one behind (fewer than E
// entries each, the edges) is taken entry by entry.
template <typename T>
struct Row {
    static constexpr int E = 16 / sizeof(T);
    using V = T __attribute__((ext_vector_type(E)));
    const T* z;
    int n, before, nchunks;             // before: places of chunk 0 in front of the row
    int lo, hi;

    __device__ __forceinline__ Row(const void* base, int64_t offset, int n_) : z((const T*)base + offset), n(n_)
    {
        before = (int)(((uintptr_t)z & 15) / sizeof(T));
        nchunks = (int)(((int64_t)before + n + E - 1) / E);
        lo = before > 0;
        hi = (int)(((int64_t)before + n) / E);
    }
    __device__ __forceinline__ bool edges() const { return lo > 0 || hi < nchunks; }
    __device__ __forceinline__ int first(int c) const { return c * E - before; }      // entry of a chunk's first place
    // chunk c, or where it is not the row's throughout the nearest one that is (there has to be one)
    __device__ __forceinline__ V raw(int c) const
    {
        c = min(max(c, lo), hi - 1);
        return *(const V*)((const char*)z - before * (int)sizeof(T) + (uint32_t)c * 16u);
    }
    // entry of the edges that thread t < 2 E looks after, or -1
    __device__ __forceinline__ int edge(int t) const
    {
        const int i = t < E ? (lo > 0 ? t : n) : (hi < nchunks && hi >= lo ? first(hi) + t - E : n);
        return t < 2 * E && i < n && (t >= E || i < E - before) ? i : -1;
    }
    // a chunk's scores, whichever it is: -inf in the places that are not the row's
    __device__ __forceinline__ int load(int c, float* v) const
    {
        if (c >= lo && c < hi) {
            const V t = raw(c);
#pragma unroll
            for (int e = 0; e < E; ++e) v[e] = (float)t[e];
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e) v[e] = (float)at(first(c) + e);
        }
        return first(c);
    }
    __device__ __forceinline__ float at(int64_t i) const { return i >= 0 && i < n ? (float)z[i] : -INFINITY; }
};

// What a thread holds of a row while it goes over it: two requests of U chunks.  Afterwards the last ones: a those of `at`, b the U behind.
template <int U, typename T>
struct Held {
    typename Row<T>::V a[U], b[U];
    int at;
};

// f(raw chunk, c, in) for the chunks of begin .. end-1 (begin a multiple of 16) that are the row's throughout, U at a time for
// every thread, all threads alike: in is false for a thread that has none.  The next U chunks are asked for before the last ones
// are worked on; what is asked for behind the row's end is its last chunk, again.  first() is called once, behind the first request.
template <int THREADS, int U, typename T, typename F, typename G>
__device__ __forceinline__ void for_chunks(const Row<T>& row, int begin, int end, Held<U, T>& h, F&& f, G&& first)
{
    const int stop = min(end, row.hi);
    h.at = begin;
    if (stop <= max(begin, row.lo)) {
        first();
        return;
    }
    auto load = [&](typename Row<T>::V* r, int c0) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < U; ++u) r[u] = row.raw(c0 + u * THREADS + (int)threadIdx.x);
    };
    auto work = [&](typename Row<T>::V* r, int c0) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int c = c0 + u * THREADS + (int)threadIdx.x;
            if (c0 + u * THREADS < stop) f(r[u], c, c >= row.lo && c < stop);
        }
    };
    load(h.a, begin);
    first();
    for (int c0 = begin;; c0 += 2 * U * THREADS) {
        load(h.b, c0 + U * THREADS);
        work(h.a, c0);
        h.at = c0;
        const bool more = c0 + 2 * U * THREADS < stop;
        if (more) load(h.a, c0 + 2 * U * THREADS);
        work(h.b, c0 + U * THREADS);
        if (!more) return;
    }
}
// f for the chunks that are still held (of begin .. end-1 as before); those before h.at are not among them
template <int THREADS, int U, typename T, typename F>
__device__ __forceinline__ void for_held(const Row<T>& row, int begin, int end, const Held<U, T>& h, F&& f)
{
    const int stop = min(end, row.hi);
    if (stop <= max(begin, row.lo)) return;
#pragma unroll
    for (int u = 0; u < 2 * U; ++u) {
        const int c = h.at + u * THREADS + (int)threadIdx.x;
        if (h.at + u * THREADS < stop) f(u < U ? h.a[u % U] : h.b[u % U], c, c >= row.lo && c < stop);
    }
}

// Chunk c of the row in the output, which may be aligned otherwise.
template <typename T>
__device__ __forceinline__ void store_chunk(T* out, const float* v)
{
    vec_of<T> t;
#pragma unroll
    for (int e = 0; e < 16 / (int)sizeof(T); ++e) t[e] = (T)v[e];
    if (((uintptr_t)out & 15) == 0) __builtin_nontemporal_store(t, (vec_of<T>*)out);
    else __builtin_memcpy(out, &t, 16);
}

template <int THREADS>
struct RowShared {
    static constexpr int kWaves = THREADS / 64;
    float part[4][kWaves];
};
struct ListShared {
    __align__(16) int id[HR_LIST_MAX];
    float c[HR_LIST_MAX], z[HR_LIST_MAX];
    float loss;
    bool some;
};

// Folds over the lanes of a wave and over a workgroup, to all of them, in the same order every time.
__device__ __forceinline__ float bits_float(uint32_t v) { return __builtin_bit_cast(float, v); }
__device__ __forceinline__ float lanes_max(float v)          // (a NaN is left out)
{
    return bits_float(wave_fold(__builtin_bit_cast(uint32_t, v), [](uint32_t x, uint32_t y) { return __builtin_bit_cast(uint32_t, fmaxf(bits_float(x), bits_float(y))); }));
}
__device__ __forceinline__ float lanes_sum(float v)
{
    return bits_float((uint32_t)__builtin_amdgcn_readlane(__builtin_bit_cast(int, wave_add(v)), 63));
}
// one number of every wave, a lane each; rest elsewhere
template <int THREADS>
__device__ __forceinline__ float of_waves(float* part, float v, float rest)
{
    __syncthreads();
    if (lane_id() == 0) part[threadIdx.x / 64] = v;
    __syncthreads();
    return lane_id() < THREADS / 64 ? part[lane_id()] : rest;
}
template <int THREADS>
__device__ __forceinline__ float group_sum(float v, RowShared<THREADS>& sh)
{
    v = lanes_sum(v);
    return THREADS == 64 ? v : lanes_sum(of_waves<THREADS>(sh.part[0], v, 0.0f));
}
template <int THREADS>
__device__ __forceinline__ float group_max(float v, RowShared<THREADS>& sh)
{
    v = lanes_max(v);
    return THREADS == 64 ? v : lanes_max(of_waves<THREADS>(sh.part[0], v, -INFINITY));
}

constexpr float kFar = 16777216.0f;    // (2^24; see Sums)

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
    // of all lanes of a wave together: what every lane has is brought to the largest maximum, then added up
    __device__ __forceinline__ void fold_lanes(float c2)
    {
        rescale(lanes_max(m), c2);
        s0 = lanes_sum(s0);
        s1 = lanes_sum(s1);
    }
    // of all threads of a workgroup; whether one of them raises flag 1 where the maximum is very low, or flag 2 (Sums)
    template <int THREADS>
    __device__ __forceinline__ bool fold(float c2, RowShared<THREADS>& sh, int flags)
    {
        fold_lanes(c2);
        const auto any = [](int f) { return (__any(f & 1) ? 1 : 0) | (__any(f & 2) ? 2 : 0); };
        const auto raised = [&](int f) { return (f & 2) != 0 || ((f & 1) != 0 && !(m * c2 > -kFar / 2)); };
        flags = any(flags);
        if (THREADS == 64) return raised(flags);
        __syncthreads();
        const int w = threadIdx.x / 64, i = lane_id();
        if (i == 0) { sh.part[0][w] = m; sh.part[1][w] = s0; sh.part[2][w] = s1; sh.part[3][w] = (float)flags; }
        __syncthreads();
        clear();
        flags = 0;
        if (i < THREADS / 64) { m = sh.part[0][i]; s0 = sh.part[1][i]; s1 = sh.part[2][i]; flags = (int)sh.part[3][i]; }
        fold_lanes(c2);
        return raised(any(flags));
    }
    __device__ __forceinline__ float top() const { return s0 == 0.0f ? -INFINITY : m; }
    // (the largest score's term is 1: a sum below is its rounding, and would make ln p of that score positive)
    __device__ __forceinline__ float log_sum() const { return s0 == 0.0f ? 0.0f : logf(s0 < 1.0f ? 1.0f : s0); }
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

// The same sums while a thread goes over its chunks, in fewer instructions: exponents are x = z c2 - r, one operation, of a reference
// r that stays until a score's term passes 2^8, and products x exp(x) are made without regard to z = -inf, whose NaN has the chunk's
// looked over again.  What r is rounded by is in every exponent alike, so it may not be large: scores with z c2 beyond 2^24 (no model
// gives any) have the row summed up once more the other way, those below -2^24 (masks) add nothing where the maximum is above -2^23.
// Against RowStat::add for every chunk: 8192 rows of 8192 bfloat16 26.7 -> 24.9 us, 2048 of 32768 float16 28.0 -> 24.7 (both read
// at over 5 TB/s), 2048 of 131072 102 -> 99.7 but, with two thirds of them -inf, 98.9 -> 105; float32, a chunk of four, the same.
struct Sums {
    float r, limit, s0, s1, best;
    bool far;                           // a score times c2 was above kFar

    __device__ __forceinline__ void clear(float c2) { r = s0 = s1 = 0.0f; limit = -kFar / c2; best = -INFINITY; far = false; }
    __device__ __forceinline__ int flags() const { return (best > -INFINITY ? 1 : 0) | (far ? 2 : 0); }
    // a chunk, top its largest score
    template <int E, bool ENTROPY>
    __device__ __forceinline__ void add(const float* v, float top, float c2, float step)
    {
        best = fmaxf(best, top);
        if (top > limit) {
#pragma clang fp contract(off)          // (r - to has to be that of the rounded product, which every exponent is taken from)
            const float to = top * c2, d = fmaxf(r - to, kLowest2), f = s0 == 0.0f ? 0.0f : __builtin_amdgcn_exp2f(d);
            s1 = f * fmaf(d, s0, s1);
            s0 *= f;
            r = to;
            limit = top + step;
            far |= !(to < kFar);
        }
        float part = 0.0f;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float x = fmaf(v[e], c2, -r), t = __builtin_amdgcn_exp2f(x);
            s0 += t;
            if (ENTROPY) part = fmaf(x, t, part);
        }
        if (ENTROPY) {
            if (part != part) {
                part = 0.0f;
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const float x = fmaf(v[e], c2, -r);
                    part = fmaf(fmaxf(x, kLowest2), __builtin_amdgcn_exp2f(x), part);
                }
            }
            s1 += part;
        }
    }
    // with the largest score as the maximum
    __device__ __forceinline__ RowStat stat(float c2) const
    {
        RowStat st;
        st.clear();
        if (best > -FLT_MAX) st.m = best;
        const float d = s0 == 0.0f ? 0.0f : -fmaf(st.m, c2, -r), f = __builtin_amdgcn_exp2f(d);
        st.s1 = f * fmaf(d, s0, s1);
        st.s0 = f * s0;
        return st;
    }
};

// Largest scores of stretches of a row: what the search for its best entries starts from.  A stretch is `span` chunks that one
// thread reads one after the other: nothing has to be exchanged between lanes to know its largest score.
template <int THREADS>
struct Slots {
    static constexpr int kPer = THREADS >= 1024 ? 4 : 8;             // of a thread
    uint32_t key[kPer][THREADS];
    static __device__ int span_for(int nchunks) { return (nchunks + THREADS * kPer - 1) / (THREADS * kPer); }
};

// Maximum and sums of chunks begin .. end-1 of a row (begin a multiple of 16; the edges if begin is 0), to all threads of a workgroup.
// TOP: the slots of this thread as well (none of the edges).  first() is called once while the first chunks are on their way.
template <typename T, int THREADS, bool ENTROPY, bool TOP, typename G>
__device__ __forceinline__ RowStat row_stats(const Row<T>& row, int begin, int end, float c2, RowShared<THREADS>& sh, Slots<THREADS>* slots, int span, Held<4, T>& held, G&& first)
{
    constexpr int E = Row<T>::E;
    Sums sums;
    sums.clear(c2);
    const float step = 8.0f / c2;
    float best = -INFINITY;
    int left = span, slot = 0;
    if (TOP) {
#pragma unroll
        for (int i = 0; i < Slots<THREADS>::kPer; ++i) slots->key[i][threadIdx.x] = 0;
    }
    for_chunks<THREADS>(row, begin, end, held, [&](const typename Row<T>::V& raw, int c, bool in) __attribute__((always_inline)) {
        float v[E];
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = (float)raw[e];
        float top = v[0];
#pragma unroll
        for (int e = 1; e < E; ++e) top = fmaxf(top, v[e]);
        if (in) {
            sums.template add<E, ENTROPY>(v, top, c2, step);
            if (TOP) best = fmaxf(best, top);
        }
        if (TOP && --left == 0) {
            slots->key[slot++][threadIdx.x] = order_key(best);
            left = span;
            best = -INFINITY;
        }
    }, first);
    if (TOP && left < span) slots->key[slot][threadIdx.x] = order_key(best);
    const int edge = begin == 0 && row.edges() ? row.edge(threadIdx.x) : -1;
    const float at_edge = edge >= 0 ? (float)row.z[edge] : -INFINITY;
    if (edge >= 0) sums.template add<1, ENTROPY>(&at_edge, at_edge, c2, step);
    RowStat st = sums.stat(c2);
    if (st.template fold<THREADS>(c2, sh, sums.flags())) {
        st.clear();
        for (int c = max(begin, row.lo) + (int)threadIdx.x; c < min(end, row.hi); c += THREADS) {
            float v[E], top = -INFINITY;
            row.load(c, v);
#pragma unroll
            for (int e = 0; e < E; ++e) top = fmaxf(top, v[e]);
            st.template add<E, ENTROPY>(v, top, c2);
        }
        if (edge >= 0) st.template add<1, ENTROPY>(&at_edge, at_edge, c2);
        st.template fold<THREADS>(c2, sh, 0);
    }
    return st;
}

// Few long rows are cut in parts, a workgroup of kPartThreads each, whose sums and slots a second launch puts together.
constexpr int kPartThreads = 256, kMostParts = 16;
struct Parts {
    int n, len;                         // parts of a row (0: whole rows), chunks of each: a multiple of kPartThreads
    float* stats;                       // [rows][n][4]: m, S0, S1
    uint32_t* slots;                    // [rows][n][kPartThreads]: the largest score that each thread has seen
};

// the parts' sums together, to all threads of a wave
__device__ __forceinline__ RowStat joined_stats(const Parts& parts, int64_t r, float c2)
{
    RowStat st;
    st.clear();
    const int i = lane_id();
    if (i < parts.n) {
        const floatx4 v = *(const floatx4*)(parts.stats + (r * parts.n + i) * 4);
        st.m = v[0]; st.s0 = v[1]; st.s1 = v[2];
    }
    st.fold_lanes(c2);
    return st;
}

struct LogprobsArgs {
    const void* logits; int64_t ld, rows; int n; float scale;
    const int64_t* given; int ngiven, k;
    float *logprobs, *entropy, *norm; int64_t* top_ids; float* top_logprobs;
    Parts parts;
};
struct LogprobsBackwardArgs {
    const void* logits; int64_t ld, rows; int n; float scale;
    const int64_t* given; int ngiven;
    const float *entropy, *norm, *grad_logprobs, *grad_entropy;
    void* grad; int64_t ldg;
    int slice;                          // chunks of a row that a workgroup takes
};
struct DistillArgs {
    const void* logits; int64_t ld, rows; int n; float scale;
    const int64_t* ids; const float* teacher; int k;
    const float* weights;
    float *loss, *norm, *q;
    void* grad; int64_t ldg;
    Parts parts;
    int slice;
};

}  // namespace hr
