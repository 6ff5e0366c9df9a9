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

// Piece c of a row of n elements: E of them from `start` on, of which those from element `skip` of the piece on are its own (the others are the piece's
// before: what does not end with a whole piece ends with one that begins earlier, and pieces behind the row's end have none of their own).
// Rows may begin at any element.
template <typename T>
struct Piece {
    Chunk<T> v;
    int start, skip;
};
template <typename T>
__device__ __forceinline__ void place(Piece<T>& p, int c, int n)
{
    p.start = min(c * kE<T>, n - kE<T>);
    p.skip = min(c * kE<T> - p.start, kE<T>);
}
// (TINY: rows shorter than a piece.  The loads of other rows stand in no branch: the compiler waits for a load where a branch ends.)
template <int E, bool TINY, typename W>
__device__ __forceinline__ void load_some(const W* at, int start, W* x)
{
    if constexpr (!TINY) {
        __builtin_memcpy(x, at + start, E * sizeof(W));
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] = start + e >= 0 ? at[start + e] : (W)0.0f;
    }
}
template <bool TINY = false, typename T>
__device__ __forceinline__ Piece<T> load_piece(const T* row, int c, int n)
{
    Piece<T> p;
    place(p, c, n);
    T x[kE<T>];
    load_some<kE<T>, TINY>(row, p.start, x);
    __builtin_memcpy(&p.v, x, 16);
    return p;
}
template <typename T>
__device__ __forceinline__ void store_piece(T* row, const Piece<T>& p, const float* x)
{
    Chunk<T> v;
#pragma unroll
    for (int e = 0; e < kE<T>; ++e) v[e] = (T)x[e];
    if (p.skip == 0) {
        __builtin_memcpy(row + p.start, &v, 16);
    } else {
#pragma unroll
        for (int e = 0; e < kE<T>; ++e)
            if (e >= p.skip) row[p.start + e] = v[e];
    }
}
// the numbers of a vector that lie at a piece, as floats; `other` where there is no vector
template <int E, typename W, bool TINY = false>
__device__ __forceinline__ void load_weights(const void* at, int start, float other, float* w)
{
    W x[E];
    if (at) load_some<E, TINY>((const W*)at, start, x);
#pragma unroll
    for (int e = 0; e < E; ++e) w[e] = at ? (float)x[e] : other;
}
// Forgets what a chunk's elements were as floats, and where its piece lies: between two passes over many pieces the chunks alone stay in registers.
template <typename T>
__device__ __forceinline__ void forget(Chunk<T>& x)
{
    u32x4 v = __builtin_bit_cast(u32x4, x);
    asm volatile("" : "+v"(v));
    x = __builtin_bit_cast(Chunk<T>, v);
}
__device__ __forceinline__ int anew(int t)
{
    asm volatile("" : "+v"(t));
    return t;
}
// piece c, with the elements it has
template <typename T>
__device__ __forceinline__ Piece<T> piece_of(const Chunk<T>& v, int c, int n)
{
    Piece<T> p;
    place(p, c, n);
    p.v = v;
    return p;
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
        const int first = threadIdx.x / LANES * WAVES;   // (of this row)
        if (lane_id() == 0) {
            part[threadIdx.x / 64][0] = a;
            part[threadIdx.x / 64][1] = b;
        }
        __syncthreads();
        a = b = 0.0f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) a += part[first + w][0], b += part[first + w][1];
    }
}

// 1 / sqrt(spread^2 + eps).  (Of a row of equal numbers far from 0 the difference of two squares may come out below 0, by more than eps; a NaN stays one.)
__device__ __forceinline__ float over_spread(float square, float eps) { return 1.0f / sqrtf((square < 0.0f ? 0.0f : square) + eps); }

// ---- rows that LANES lanes hold, CH chunks of 16 bytes each, between their one read and their one write.  The mean is found first and the
// spread from what is left: the second fold also finds what the first mean is off by, so that a row far from 0 loses nothing.
// Bound by memory, in and out: 16384 x 4096 bfloat16 57 us (4.7 TB/s, a copy's rate), 65536 x 768 39 (5.1), 262144 x 128 24 (5.6), 8192 x 8192 float32 91 (5.9);
// 512 x 50021 float32 58 (3.5: a row fills a compute unit's registers, and the next one waits until it has been written).  One row of 768 takes 3.
template <typename T, typename W, int LANES, int CH, bool TINY = false>
__global__ __launch_bounds__(LANES > 256 ? LANES : 256, LANES == 1024 && CH == 4 && sizeof(T) == 2 ? 8 : 1) void k_norm(NormArgs a)
{
    constexpr int E = kE<T>, THREADS = LANES > 256 ? LANES : 256, ROWS = THREADS / LANES;
    constexpr bool KEEP = CH * E <= 16;                  // weights stay in registers from row to row
    __shared__ Folds folds;
    int turn = 0;
    const int t = threadIdx.x % LANES, n = a.n;
    const float over = 1.0f / (float)n;
    float w[KEEP ? CH : 1][E], b[KEEP ? CH : 1][E];
    auto weights = [&](const Piece<T>& p, float* wi, float* bi) __attribute__((always_inline)) {
        load_weights<E, W, TINY>(a.weight, p.start, 1.0f, wi);
        load_weights<E, W, TINY>(a.bias, p.start, 0.0f, bi);
    };
    if constexpr (KEEP)
        for (int i = 0; i < CH; ++i) weights(piece_of<T>(Chunk<T>{}, i * LANES + t, n), w[i], b[i]);
    // (AHEAD: large workgroups are few on a compute unit, and ask for their next row before they fold the last one's sums; where two of 1024 threads fit
    // without, as those of 16 bits do, that is faster: 2048 x 32768 bfloat16 65 us for 71)
    constexpr bool AHEAD = (LANES == 512 || (LANES == 1024 && sizeof(T) == 4)) && CH <= 4;
    auto load = [&](int64_t r0, Chunk<T>* x) __attribute__((always_inline)) {
        const T* row = (const T*)a.x + min(r0 + threadIdx.x / LANES, a.rows - 1) * a.ldx;
#pragma unroll
        for (int i = 0; i < CH; ++i) x[i] = load_piece<TINY>(row, i * LANES + t, n).v;
    };
    Chunk<T> x[CH], next[CH];
    if constexpr (AHEAD) load((int64_t)blockIdx.x * ROWS, next);
    for (int64_t r0 = (int64_t)blockIdx.x * ROWS; r0 < a.rows; r0 += (int64_t)gridDim.x * ROWS) {
        const int64_t r = r0 + threadIdx.x / LANES;
        const bool in = r < a.rows;
        int at = t;
        if constexpr (AHEAD) {
#pragma unroll
            for (int i = 0; i < CH; ++i) x[i] = next[i];
            load(r0 + (int64_t)gridDim.x * ROWS, next);
        } else {
            load(r0, x);
        }
        float s0 = 0.0f, s1 = 0.0f;
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const Piece<T> p = piece_of<T>(x[i], i * LANES + at, n);
#pragma unroll
            for (int e = 0; e < E; ++e) s0 += e >= p.skip ? (float)p.v[e] : 0.0f;
        }
        fold_two<LANES>(s0, s1, folds, turn);
        const float first = s0 * over;
        s0 = s1 = 0.0f;
        if constexpr (!KEEP) at = anew(t);
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            if constexpr (!KEEP) forget<T>(x[i]);
            const Piece<T> p = piece_of<T>(x[i], i * LANES + at, n);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float d = e >= p.skip ? (float)p.v[e] - first : 0.0f;
                s0 += d;
                s1 = fmaf(d, d, s1);
            }
        }
        fold_two<LANES>(s0, s1, folds, turn);
        const float off = s0 * over, rstd = over_spread(s1 * over - off * off, a.eps);
        if (!in) continue;
        if (t == 0 && a.stats) {
            a.stats[2 * r] = first + off;
            a.stats[2 * r + 1] = rstd;
        }
        T* out = (T*)a.out + r * a.ldo;
        if constexpr (!KEEP) at = anew(t);
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            float wi[E], bi[E], y[E];
            if constexpr (!KEEP) {
                forget<T>(x[i]);
                asm volatile("" ::: "memory");           // (the weights of one piece at a time)
            }
            const Piece<T> p = piece_of<T>(x[i], i * LANES + at, n);
            if constexpr (!KEEP) weights(p, wi, bi);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                if constexpr (KEEP) wi[e] = w[i][e], bi[e] = b[i][e];
                y[e] = fmaf(((float)p.v[e] - first - off) * rstd, wi[e], bi[e]);
            }
            if (p.skip < E) store_piece(out, p, y);
        }
    }
}

// longer rows (256 KB and more) are read three times, by 1024 threads each: the second and third time from the caches where rows are few
template <typename T, typename W>
__global__ __launch_bounds__(1024) void k_norm_long(NormArgs a)
{
    constexpr int E = kE<T>, U = 4;
    __shared__ Folds folds;
    int turn = 0;
    const int n = a.n, chunks = (n + E - 1) / E;
    const float over = 1.0f / (float)n;
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const T* row = (const T*)a.x + r * a.ldx;
        // f of every piece, U of them asked for at once (behind the row's end: pieces without elements)
        auto pass = [&](auto f) __attribute__((always_inline)) {
            for (int c0 = threadIdx.x; c0 < chunks; c0 += 1024 * U) {
                Piece<T> x[U];
#pragma unroll
                for (int u = 0; u < U; ++u) x[u] = load_piece(row, min(c0 + u * 1024, chunks), n);
#pragma unroll
                for (int u = 0; u < U; ++u) f(x[u]);
            }
        };
        float s0 = 0.0f, s1 = 0.0f;
        pass([&](const Piece<T>& x) __attribute__((always_inline)) {
#pragma unroll
            for (int e = 0; e < E; ++e) s0 += e >= x.skip ? (float)x.v[e] : 0.0f;
        });
        fold_two<1024>(s0, s1, folds, turn);
        const float first = s0 * over;
        s0 = s1 = 0.0f;
        pass([&](const Piece<T>& x) __attribute__((always_inline)) {
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float d = e >= x.skip ? (float)x.v[e] - first : 0.0f;
                s0 += d;
                s1 = fmaf(d, d, s1);
            }
        });
        fold_two<1024>(s0, s1, folds, turn);
        const float off = s0 * over, rstd = over_spread(s1 * over - off * off, a.eps);
        if (threadIdx.x == 0 && a.stats) {
            a.stats[2 * r] = first + off;
            a.stats[2 * r + 1] = rstd;
        }
        T* out = (T*)a.out + r * a.ldo;
        pass([&](const Piece<T>& x) __attribute__((always_inline)) {
            float w[E], b[E], y[E];
            load_weights<E, W>(a.weight, x.start, 1.0f, w);
            load_weights<E, W>(a.bias, x.start, 0.0f, b);
#pragma unroll
            for (int e = 0; e < E; ++e) y[e] = fmaf(((float)x.v[e] - first - off) * rstd, w[e], b[e]);
            store_piece(out, x, y);
        });
    }
}

// ---- gradients of rows that LANES lanes hold; sums over the workgroup's rows stay in registers until its last.  Bound by memory, two in and one out, as
// long as enough waves are there to ask: 16384 x 4096 bfloat16 84 us (4.8 TB/s), 65536 x 768 55, float32 121 (5.0), 8192 x 8192 float32 156 (5.2).
// Workgroups of 512 threads, at most 512 of them, 128 registers a lane: with 256 threads 91, 68 and 168 us for the first three.
template <typename T, typename W, int LANES, int CH, bool TINY = false, int THREADS = (LANES > 256 ? LANES : 256)>
__global__ __launch_bounds__(THREADS, THREADS == 512 ? 4 : 1) void k_norm_backward(NormArgs a)
{
    constexpr int E = kE<T>, ROWS = THREADS / LANES;
    __shared__ Folds folds;
    __shared__ float sums[ROWS > 1 ? ROWS * LANES * CH * E : 1];
    int turn = 0;
    const int t = threadIdx.x % LANES, n = a.n;
    const float over = 1.0f / (float)n;
    float w[CH][E], dw[CH][E] = {}, db[CH][E] = {};
    for (int i = 0; i < CH; ++i) {
        Piece<T> p;
        place(p, i * LANES + t, n);
        load_weights<E, W, TINY>(a.weight, p.start, 1.0f, w[i]);
    }
    for (int64_t r0 = (int64_t)blockIdx.x * ROWS; r0 < a.rows; r0 += (int64_t)gridDim.x * ROWS) {
        const int64_t r = r0 + threadIdx.x / LANES, at = min(r, a.rows - 1);
        const bool in = r < a.rows;
        Chunk<T> x[CH], dy[CH];
        int lane = t;
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            x[i] = load_piece<TINY>((const T*)a.x + at * a.ldx, i * LANES + lane, n).v;
            dy[i] = load_piece<TINY>((const T*)a.dy + at * a.ldg, i * LANES + lane, n).v;
        }
        const float mean = a.stats[2 * at], rstd = a.stats[2 * at + 1];
        float s0 = 0.0f, s1 = 0.0f;
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const Piece<T> p = piece_of<T>(x[i], i * LANES + lane, n);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const bool own = e >= p.skip;
                const float u = own ? ((float)p.v[e] - mean) * rstd : 0.0f, d = own ? (float)dy[i][e] : 0.0f, g = own ? d * w[i][e] : 0.0f;
                s0 += g;
                s1 = fmaf(g, u, s1);
                if (in) {
                    dw[i][e] = fmaf(d, u, dw[i][e]);
                    db[i][e] += d;
                }
            }
        }
        fold_two<LANES>(s0, s1, folds, turn);
        const float c1 = s0 * over, c2 = s1 * over;
        if (!in || !a.dx) continue;
        T* out = (T*)a.dx + r * a.ldgx;
        lane = anew(t);
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            forget<T>(x[i]);
            forget<T>(dy[i]);
            const Piece<T> p = piece_of<T>(x[i], i * LANES + lane, n);
            if (p.skip >= E) continue;
            float y[E];
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float u = ((float)p.v[e] - mean) * rstd, g = (float)dy[i][e] * w[i][e];
                y[e] = rstd * (g - c1 - u * c2);
            }
            store_piece(out, p, y);
        }
    }
    if (!a.parts) return;
    float* to = a.parts + (int64_t)blockIdx.x * 2 * n;
    auto write = [&](float(*x)[E], float* at) __attribute__((always_inline)) {
        Piece<T> p;
        if constexpr (ROWS > 1) {                        // the rows of the workgroup, in their order
            __syncthreads();
#pragma unroll
            for (int i = 0; i < CH; ++i) {
                place(p, i * LANES + t, n);
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (e >= p.skip) sums[(threadIdx.x / LANES) * LANES * CH * E + p.start + e] = x[i][e];
            }
            __syncthreads();
            for (int j = threadIdx.x; j < n; j += THREADS) {
                float s = 0.0f;
#pragma unroll
                for (int q = 0; q < ROWS; ++q) s += sums[q * LANES * CH * E + j];
                at[j] = s;
            }
        } else {
#pragma unroll
            for (int i = 0; i < CH; ++i) {
                place(p, i * LANES + t, n);
                if (p.skip == 0) {
                    __builtin_memcpy(at + p.start, x[i], E * 4);
                } else {
#pragma unroll
                    for (int e = 0; e < E; ++e)
                        if (e >= p.skip) at[p.start + e] = x[i][e];
                }
            }
        }
    };
    write(dw, to);
    write(db, to + n);
}

// ---- longer rows, whose sums over rows do not fit the registers beside them: the two sums of every row, then stripes of 256 chunks of columns, some
// of the rows each.  Both inputs are read twice: 512 x 50021 float32 39 (5.3 TB/s) and 58 us (5.3); the order of the second makes no difference.
template <typename T, typename W>
__global__ __launch_bounds__(1024) void k_norm_sums(NormArgs a)
{
    constexpr int E = kE<T>, U = 4;
    __shared__ Folds folds;
    int turn = 0;
    const int n = a.n, chunks = (n + E - 1) / E;
    const float over = 1.0f / (float)n;
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const T *xr = (const T*)a.x + r * a.ldx, *dr = (const T*)a.dy + r * a.ldg;
        const float mean = a.stats[2 * r], rstd = a.stats[2 * r + 1];
        float s0 = 0.0f, s1 = 0.0f;
        for (int c0 = threadIdx.x; c0 < chunks; c0 += 1024 * U) {
            Piece<T> x[U], dy[U];
            float w[U][E];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int c = min(c0 + u * 1024, chunks);                        // (behind the row's end: a piece without elements)
                x[u] = load_piece(xr, c, n);
                dy[u] = load_piece(dr, c, n);
                load_weights<E, W>(a.weight, x[u].start, 1.0f, w[u]);
            }
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const bool own = e >= x[u].skip;
                    const float v = own ? ((float)x[u].v[e] - mean) * rstd : 0.0f, g = own ? (float)dy[u].v[e] * w[u][e] : 0.0f;
                    s0 += g;
                    s1 = fmaf(g, v, s1);
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
    Piece<T> p;
    place(p, c, n);
    load_weights<E, W>(a.weight, p.start, 1.0f, w);
    constexpr int U = 4;                                 // rows at once; those behind the last one are it again, and take no part
    for (int64_t r0 = blockIdx.y; r0 < a.rows; r0 += U * (int64_t)gridDim.y) {
        Piece<T> x[U], dy[U];
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const int64_t r = min(r0 + i * (int64_t)gridDim.y, a.rows - 1);
            x[i] = load_piece((const T*)a.x + r * a.ldx, c, n);
            dy[i] = load_piece((const T*)a.dy + r * a.ldg, c, n);
        }
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const int64_t r = r0 + i * (int64_t)gridDim.y;
            if (r >= a.rows) break;
            const float mean = a.stats[2 * r], rstd = a.stats[2 * r + 1], c1 = a.sums[2 * r], c2 = a.sums[2 * r + 1];
            float y[E];
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float u = ((float)x[i].v[e] - mean) * rstd, d = (float)dy[i].v[e];
                dw[e] = fmaf(d, u, dw[e]);
                db[e] += d;
                y[e] = rstd * (d * w[e] - c1 - u * c2);
            }
            if (a.dx) store_piece((T*)a.dx + r * a.ldgx, x[i], y);
        }
    }
    if (!a.parts) return;
    float* to = a.parts + (int64_t)blockIdx.y * 2 * n;
#pragma unroll
    for (int e = 0; e < E; ++e)
        if (e >= p.skip) to[p.start + e] = dw[e], to[n + p.start + e] = db[e];
}

// ---- the sums of the groups of rows, in an order that depends on nothing but their number: SHARES threads take every SHARES-th group of four columns.
// 128 where there may be many groups (with 32 shares 8.6 us instead of 4 for 359 groups of 67 columns, a chain of round trips), 16 for the few of long rows.
template <typename W, int SHARES>
__global__ __launch_bounds__(1024) void k_norm_join(const float* parts, int groups, int n, void* grad_weight, void* grad_bias)
{
    constexpr int FOURS = 1024 / SHARES, COLS = 4 * FOURS, PARTS = 256 / COLS;            // (256 threads add 16 shares each)
    __shared__ floatx4 sums[SHARES][FOURS];
    __shared__ float some[PARTS][COLS];
    const int64_t all = 2 * (int64_t)n;
    const int share = threadIdx.x / FOURS, c = threadIdx.x % COLS;
    for (int64_t first = (int64_t)blockIdx.x * COLS; first < all; first += (int64_t)gridDim.x * COLS) {
        const int64_t col = first + threadIdx.x % FOURS * 4;
        floatx4 s = {0, 0, 0, 0};
        if (col + 4 <= all) {
#pragma unroll 4
            for (int g = share; g < groups; g += SHARES) {
                floatx4 v;
                __builtin_memcpy(&v, parts + g * all + col, 16);
                s += v;
            }
        } else {
            for (int g = share; g < groups; g += SHARES)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (col + e < all) s[e] += parts[g * all + col + e];
        }
        sums[share][threadIdx.x % FOURS] = s;
        __syncthreads();
        if (threadIdx.x < 256) {
            float v = 0.0f;
#pragma unroll
            for (int q = 0; q < 16; ++q) v += sums[threadIdx.x / COLS * 16 + q][c / 4][c % 4];
            some[threadIdx.x / COLS][c] = v;
        }
        __syncthreads();
        if (threadIdx.x < COLS) {
            const int64_t j = first + c;
            float v = 0.0f;
#pragma unroll
            for (int q = 0; q < PARTS; ++q) v += some[q][c];
            void* to = j < n ? grad_weight : grad_bias;
            if (j < all && to) ((W*)to)[j < n ? j : j - n] = (W)v;
        }
    }
}

// ---- which kernel
constexpr int kHeldColumns = 16384;                      // most columns of rows whose gradients workgroups hold: sums over rows take 2 x 16 registers of 1024 lanes
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

// The fewest lanes that hold a row in two chunks each, four and more where a workgroup is the row; large workgroups are filled by looking a row ahead
// (4096 x 16384 bfloat16: 1024 lanes and two chunks 99 us, 512 and four, a row ahead, 67).  Sixteen chunks of 16 bits and their weights in 16 bits do not quite fit 128
// registers (12 to 20 bytes a lane in scratch; bfloat16 rows with float32 weights do): 512 x 131072 bfloat16 71 us with weights in float32, 76 in bfloat16.
template <typename T, typename W>
static void launch_norm(const NormArgs& a, hipStream_t s)
{
    const int64_t chunks = (a.n + kE<T> - 1) / kE<T>;
    auto go = [&](auto kernel, int threads, int rows) {
        const int64_t want = (a.rows + rows - 1) / rows, most = 256 * (2048 / threads);
        hipLaunchKernelGGL(kernel, dim3((unsigned)std::min(want, most)), dim3(threads), 0, s, a);
    };
    if (a.n < kE<T>) go(k_norm<T, W, 16, 1, true>, 256, 16);
    else if (chunks <= 16) go(k_norm<T, W, 16, 1>, 256, 16);
    else if (chunks <= 32) go(k_norm<T, W, 16, 2>, 256, 16);
    else if (chunks <= 64) go(k_norm<T, W, 64, 1>, 256, 4);
    else if (chunks <= 128) go(k_norm<T, W, 64, 2>, 256, 4);
    else if (chunks <= 256) go(k_norm<T, W, 256, 1>, 256, 1);
    else if (chunks <= 512) go(k_norm<T, W, 256, 2>, 256, 1);
    else if (chunks <= 1024) go(k_norm<T, W, 256, 4>, 256, 1);
    else if (chunks <= 2048) go(k_norm<T, W, 512, 4>, 512, 1);
    else if (chunks <= 4096) go(k_norm<T, W, 1024, 4>, 1024, 1);
    else if (chunks <= 8192) go(k_norm<T, W, 1024, 8>, 1024, 1);
    else if (chunks <= 16384) go(k_norm<T, W, 1024, 16>, 1024, 1);
    else go(k_norm_long<T, W>, 1024, 1);
}

// The same for gradients, two chunks of x and of its gradient's rows a lane and the sums of both over the rows.  Where one workgroup of 1024 fills a compute
// unit there are 256 (4096 x 16384 bfloat16 84 + 7 us to join them; 512, in turns, 94 + 16).
template <typename T, typename W>
static void launch_norm_backward(const NormArgs& a, void* grad_weight, void* grad_bias, hipStream_t s)
{
    const int64_t chunks = (a.n + kE<T> - 1) / kE<T>, most = groups_for(a.rows, a.n);
    int64_t groups = 0;
    auto go = [&](auto kernel, int threads, int rows) {
        groups = std::min((a.rows + rows - 1) / rows, threads == 1024 && rows == 1 ? std::min<int64_t>(most, 256) : most);
        hipLaunchKernelGGL(kernel, dim3((unsigned)groups), dim3(threads), 0, s, a);
    };
    if (a.rows == 0) {
    } else if (a.n > kHeldColumns) {
        hipLaunchKernelGGL((k_norm_sums<T, W>), dim3((unsigned)std::min<int64_t>(a.rows, 512)), dim3(1024), 0, s, a);
        // (three workgroups a compute unit: 58 us instead of 66 with eight, 512 x 50021 float32)
        groups = std::min<int64_t>(most, std::max<int64_t>(1, 768 / ((chunks + 255) / 256)));
        hipLaunchKernelGGL((k_norm_stripe<T, W>), dim3((unsigned)((chunks + 255) / 256), (unsigned)groups), dim3(256), 0, s, a);
    } else if (a.n < kE<T>) go(k_norm_backward<T, W, 16, 1, true>, 256, 16);
    else if (chunks <= 16) go(k_norm_backward<T, W, 16, 1>, 256, 16);
    else if (chunks <= 32) go(k_norm_backward<T, W, 16, 2>, 256, 16);
    else if (chunks <= 64) go(k_norm_backward<T, W, 64, 1, false, 512>, 512, 8);
    else if (chunks <= 128) go(k_norm_backward<T, W, 64, 2, false, 512>, 512, 8);
    else if (chunks <= 256) go(k_norm_backward<T, W, 256, 1, false, 512>, 512, 2);
    else if (chunks <= 512) go(k_norm_backward<T, W, 256, 2, false, 512>, 512, 2);
    else if (chunks <= 1024) go(k_norm_backward<T, W, 512, 2>, 512, 1);
    else if (chunks <= 2048) go(k_norm_backward<T, W, 1024, 2>, 1024, 1);
    else if constexpr (sizeof(T) == 4) go(k_norm_backward<T, W, 1024, 4>, 1024, 1);
    if (a.parts || a.rows == 0) {
        if (!grad_weight && !grad_bias) return;
        auto join = [&](auto kernel, int columns) {
            const int64_t blocks = std::min<int64_t>((2 * (int64_t)a.n + columns - 1) / columns, 1 << 20);
            hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(1024), 0, s, a.parts, (int)groups, a.n, grad_weight, grad_bias);
        };
        a.n > kHeldColumns ? join(k_norm_join<W, 16>, 256) : join(k_norm_join<W, 128>, 32);
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
