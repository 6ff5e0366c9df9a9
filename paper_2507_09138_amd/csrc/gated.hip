// The gated half of a feed-forward block, act(x w_gate') * (x w_up'), and its gradients (hr_layers.h): which kernels, and all but the tiles.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "entry.h"
#include "tile.h"
#include "tile_plan.h"

namespace hr {

template <typename T> constexpr int kE = 16 / (int)sizeof(T);            // elements of 16 bytes

// 16 bytes of a row from an element on that may lie anywhere: whole words of 4 bytes and a shift (a load of 16 bytes that begins inside a word takes
// four times as long; the word behind them is read only where it holds some of them)
template <typename T>
__device__ __forceinline__ u32x4 load16_words(const T* at)
{
    u32x4 v;
    if constexpr (sizeof(T) == 4) {
        __builtin_memcpy(&v, at, 16);
    } else {
        const uint32_t* from = (const uint32_t*)((uintptr_t)at & ~(uintptr_t)3);
        const uint32_t shift = (uint32_t)(uintptr_t)at & 3;
        uint32_t w[5];
        __builtin_memcpy(w, __builtin_assume_aligned(from, 4), 16);
        w[4] = from[shift ? 4 : 3];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = __builtin_amdgcn_alignbyte(w[i + 1], w[i], shift);
    }
    return v;
}

// 16 bytes of a row from element t on, zeros from element n on; rows may begin at any element
template <typename T>
__device__ __forceinline__ u32x4 load16(const T* row, int t, int n)
{
    u32x4 v;
    if (t + kE<T> <= n) {
        __builtin_memcpy(&v, row + t, 16);
    } else {                                             // (every load is one: with a branch around each they would wait for each other)
        T x[kE<T>];
#pragma unroll
        for (int e = 0; e < kE<T>; ++e) x[e] = row[min(t + e, n - 1)];
#pragma unroll
        for (int e = 0; e < kE<T>; ++e)
            if (t + e >= n) x[e] = (T)0.0f;
        __builtin_memcpy(&v, x, 16);
    }
    return v;
}

// ---- rows that tiles cannot take as they are (they begin at other places than multiples of 16 bytes, are no multiple of that long, or lie too far apart for
// 32-bit offsets), copied with zeros behind them to multiples of 128 bytes: those of up to three matrices, one after the other.  8192 x 4096 and 2 x 10752 x 4096
// bfloat16 75 us beside 1110 for the products, 777 x 1024 and 2 x 1333 x 1024 binary16 9 beside 14 (tiles that stage such rows through registers: 28).
struct PadArgs {
    const void* x[3]; int64_t ld[3], rows[3];
    int n;
    char* out; int64_t ldo;                              // (in bytes)
};
template <typename T>
__global__ __launch_bounds__(256) void k_pad(PadArgs a)
{
    const int64_t pieces = a.ldo / 16, to1 = a.rows[0], to2 = to1 + a.rows[1], all = (to2 + a.rows[2]) * pieces;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / pieces;
        const int of = r < to1 ? 0 : r < to2 ? 1 : 2;
        const T* row = (const T*)a.x[of] + (r - (of == 0 ? 0 : of == 1 ? to1 : to2)) * a.ld[of];
        *(u32x4*)(a.out + i * 16) = load16(row, (int)(i - r * pieces) * kE<T>, a.n);
    }
}

// ---- 64 x 64 elements turned in LDS: rows of 64 elements and one word, so that the elements of a column lie in different banks
template <typename T> constexpr int kTurn = 64 + 4 / (int)sizeof(T);
template <typename T>
__device__ __forceinline__ void turn_in(T* tile, int r, int c, u32x4 v)           // 16 bytes of row r from column c on
{
#pragma unroll
    for (int e = 0; e < 4; ++e) *(uint32_t*)(tile + r * kTurn<T> + c + e * (4 / (int)sizeof(T))) = v[e];
}
template <typename T>
__device__ __forceinline__ u32x4 turn_out(const T* tile, int c, int r)            // 16 bytes of column c from row r on
{
    T x[kE<T>];
#pragma unroll
    for (int e = 0; e < kE<T>; ++e) x[e] = tile[(r + e) * kTurn<T> + c];
    u32x4 v;
    __builtin_memcpy(&v, x, 16);
    return v;
}

// What the products of the gradients take, laid out by one launch: matrix instructions want both operands' k in rows, and a product for a matrix's gradient
// has tokens for k, the one for x's has columns of both matrices.  Bound by memory: 8192 x 4096 x 10752 bfloat16 2.07 GB in 417 us (5.0 TB/s); turned by
// the products themselves the same elements would be turned once for every tile that takes them.  Workgroups of 64 x 64 elements, in this order:
struct LayOutArgs {
    const float* pre; const void* dh; int64_t ldh; int act;
    const void* gate; int64_t ldg;
    const void* up; int64_t ldu;
    const void* x; int64_t ldx;
    int m, k, f, fp, mp;                                 // fp, mp: with the zeros behind them
    void* rows;                                          // gradients of gate and up, [m][2 fp]: the gate's, zeros, up's, zeros; or NULL
    void* cols;                                          // and [2 f][mp], zeros behind each; or NULL
    void* turned_w;                                      // with rows: both matrices, [k][2 fp], zeros behind each
    void* turned_x;                                      // with cols: x, [k][mp], zeros behind
    int blocks_d, blocks_w;                              // workgroups of the gradients, of each matrix
    const uint32_t *of_row, *of_col;                     // kRaised: see k_largest
};
// eight or four floats of a row of n from t on, zeros behind its end
template <int E>
__device__ __forceinline__ void load_floats(const float* row, int t, int n, float* v)
{
    if (t + E <= n) {
        __builtin_memcpy(v, row + t, E * 4);
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = row[min(t + e, n - 1)];
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (t + e >= n) v[e] = 0.0f;
    }
}
// ---- the largest magnitude of each row of d_gate and d_up together, and of each of their columns, as bits (of numbers without a sign they are in order, and it
// makes no difference in which order the largest is found).  A wave takes 512 columns of one row after the other.  Bound by memory, pre and grad_out once
// more: 8192 x 10752 binary16 185 us (4.7 TB/s), 777 x 1333 11 and 2.4 for the zeros before.
struct LargestArgs {
    const float* pre; const void* dh; int64_t ldh; int act;
    int m, f, rows;                                      // rows: of a workgroup
    uint32_t *of_row, *of_col;                           // [m], [2 f]; zeros before
};
template <typename T>
__global__ __launch_bounds__(256) void k_largest(LargestArgs a)
{
    constexpr int E = kE<T>;
    __shared__ uint32_t most[2][64 * E];
    for (int i = threadIdx.x; i < 2 * 64 * E; i += 256) most[0][i] = 0;
    __syncthreads();
    const int lane = lane_id(), wave = threadIdx.x / 64, c = blockIdx.x * 64 * E + lane * E;
    uint32_t gate[E] = {}, up[E] = {};
    const int64_t begin = (int64_t)blockIdx.y * a.rows, end = min(begin + a.rows, (int64_t)a.m);
    constexpr int U = 2;                                 // rows at once; those behind the last one are it again
    auto pass = [&](auto whole) __attribute__((always_inline)) {
        for (int64_t r0 = begin + wave; r0 < end; r0 += 4 * U) {
            u32x4 raw[U];
            float z[U][E], w[U][E];
#pragma unroll
            for (int j = 0; j < U; ++j) {
                const int64_t r = min(r0 + 4 * j, end - 1);
                const float* at = a.pre + r * 2 * a.f;
                const T* dh = (const T*)a.dh + r * a.ldh;
                if constexpr (decltype(whole)::value) {
                    __builtin_memcpy(&raw[j], dh + c, 16);
                    __builtin_memcpy(z[j], at + c, E * 4);
                    __builtin_memcpy(w[j], at + a.f + c, E * 4);
                } else {
                    raw[j] = load16(dh, c, a.f);
                    load_floats<E>(at, c, a.f, z[j]);
                    load_floats<E>(at + a.f, c, a.f, w[j]);
                }
            }
#pragma unroll
            for (int j = 0; j < U; ++j) {
                T d[E];
                __builtin_memcpy(d, &raw[j], 16);
                uint32_t row = 0;
#pragma unroll
                for (int e = 0; e < E; ++e) {            // (behind the row's end all three are 0)
                    float slope;
                    const float v = act_value(z[j][e], a.act, slope);
                    const uint32_t dg = __builtin_bit_cast(uint32_t, (float)d[e] * w[j][e] * slope) & 0x7fffffffu, du = __builtin_bit_cast(uint32_t, (float)d[e] * v) & 0x7fffffffu;
                    gate[e] = max(gate[e], dg);
                    up[e] = max(up[e], du);
                    row = max(row, max(dg, du));
                }
                row = wave_fold(row, [](uint32_t x, uint32_t y) { return x > y ? x : y; });
                if (lane == 0) atomicMax(a.of_row + min(r0 + 4 * j, end - 1), row);
            }
        }
    };
    if ((blockIdx.x + 1) * 64 * E <= (unsigned)a.f) pass(std::true_type{});
    else pass(std::false_type{});
#pragma unroll
    for (int e = 0; e < E; ++e) {
        atomicMax(&most[0][lane * E + e], gate[e]);
        atomicMax(&most[1][lane * E + e], up[e]);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * 64 * E; i += 256) {
        const int which = i / (64 * E), col = blockIdx.x * 64 * E + i % (64 * E);
        if (col < a.f) atomicMax(a.of_col + (int64_t)which * a.f + col, most[which][i % (64 * E)]);
    }
}

template <typename T>
__global__ __launch_bounds__(256) void k_lay_out(LayOutArgs a)
{
    __shared__ __align__(16) T tiles[2][64 * kTurn<T>];
    constexpr int E = kE<T>, PER = 64 / E, N = 64 * PER / 256;
    int block = blockIdx.x;
    if (block < a.blocks_d) {
        const int across = (a.fp + 63) / 64, r0 = block / across * 64, c0 = block % across * 64;
        auto gradients = [&](auto whole) __attribute__((always_inline)) {
            u32x4 raw[N];
            float z[N][E], w[N][E];
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const int i = threadIdx.x + j * 256, r = i / PER, c = i % PER * E;
                const float* at = a.pre + (int64_t)(r0 + r) * 2 * a.f;
                const T* dh = (const T*)a.dh + (int64_t)(r0 + r) * a.ldh;
                if constexpr (decltype(whole)::value) {
                    __builtin_memcpy(&raw[j], dh + c0 + c, 16);
                    __builtin_memcpy(z[j], at + c0 + c, E * 4);
                    __builtin_memcpy(w[j], at + a.f + c0 + c, E * 4);
                } else {
                    raw[j] = u32x4{0, 0, 0, 0};
#pragma unroll
                    for (int e = 0; e < E; ++e) z[j][e] = w[j][e] = 0.0f;
                    if (r0 + r < a.m) {
                        raw[j] = load16(dh, c0 + c, a.f);
                        load_floats<E>(at, c0 + c, a.f, z[j]);
                        load_floats<E>(at + a.f, c0 + c, a.f, w[j]);
                    }
                }
            }
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const int i = threadIdx.x + j * 256, r = i / PER, c = i % PER * E;
                T d[E], dg[E], du[E];
                u32x4 g, u;
                __builtin_memcpy(d, &raw[j], 16);
                int by = 0;
                if constexpr (kRaised<T>) by = raised_by(a.of_row[min(r0 + r, a.m - 1)]);
#pragma unroll
                for (int e = 0; e < E; ++e) {            // (behind a row's end all three are 0, and so are both gradients)
                    float slope;
                    const float v = act_value(z[j][e], a.act, slope);
                    z[j][e] = (float)d[e] * w[j][e] * slope;
                    w[j][e] = (float)d[e] * v;
                    dg[e] = (T)(kRaised<T> ? __builtin_ldexpf(z[j][e], by) : z[j][e]);
                    du[e] = (T)(kRaised<T> ? __builtin_ldexpf(w[j][e], by) : w[j][e]);
                }
                __builtin_memcpy(&g, dg, 16);
                __builtin_memcpy(&u, du, 16);
                if (a.rows && r0 + r < a.m && c0 + c < a.fp) {
                    T* at = (T*)a.rows + (int64_t)(r0 + r) * 2 * a.fp + c0 + c;
                    *(u32x4*)at = g;
                    *(u32x4*)(at + a.fp) = u;
                }
                if constexpr (kRaised<T>) {
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        const int col = min(c0 + c + e, a.f - 1);
                        dg[e] = (T)__builtin_ldexpf(z[j][e], raised_by(a.of_col[col]));
                        du[e] = (T)__builtin_ldexpf(w[j][e], raised_by(a.of_col[a.f + col]));
                    }
                    __builtin_memcpy(&g, dg, 16);
                    __builtin_memcpy(&u, du, 16);
                }
                turn_in(tiles[0], r, c, g);
                turn_in(tiles[1], r, c, u);
            }
        };
        // (no branch between the loads of blocks that are whole: the compiler waits where one ends)
        if (r0 + 64 <= a.m && c0 + 64 <= a.f) gradients(std::true_type{});
        else gradients(std::false_type{});
        if (!a.cols) return;
        __syncthreads();
        for (int i = threadIdx.x; i < 2 * 64 * PER; i += 256) {
            const int up = i / (64 * PER), c = i / PER % 64, r = i % PER * E;
            if (c0 + c < a.f && r0 + r < a.mp) *(u32x4*)((T*)a.cols + ((int64_t)up * a.f + c0 + c) * a.mp + r0 + r) = turn_out(tiles[up], c, r);
        }
        return;
    }
    block -= a.blocks_d;
    const bool of_w = a.rows && block < 2 * a.blocks_w, of_up = of_w && block >= a.blocks_w;
    if (of_w) block -= of_up ? a.blocks_w : 0;
    else if (a.rows) block -= 2 * a.blocks_w;
    const T* from = (const T*)(of_w ? (of_up ? a.up : a.gate) : a.x);
    const int64_t ld = of_w ? (of_up ? a.ldu : a.ldg) : a.ldx;
    const int n = of_w ? a.f : a.m, padded = of_w ? a.fp : a.mp;                 // rows of what is turned
    T* out = of_w ? (T*)a.turned_w + (of_up ? a.fp : 0) : (T*)a.turned_x;
    const int64_t ldo = of_w ? 2 * a.fp : a.mp;
    const int across = (a.k + 63) / 64, r0 = block / across * 64, c0 = block % across * 64;
    u32x4 some[N];
    if (r0 + 64 <= n && c0 + 64 <= a.k) {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const int i = threadIdx.x + j * 256;
            __builtin_memcpy(&some[j], from + (int64_t)(r0 + i / PER) * ld + c0 + i % PER * E, 16);
        }
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const int i = threadIdx.x + j * 256, r = i / PER;
            some[j] = r0 + r < n ? load16(from + (int64_t)(r0 + r) * ld, c0 + i % PER * E, a.k) : u32x4{0, 0, 0, 0};
        }
    }
#pragma unroll
    for (int j = 0; j < N; ++j) turn_in(tiles[0], (threadIdx.x + j * 256) / PER, (threadIdx.x + j * 256) % PER * E, some[j]);
    __syncthreads();
#pragma unroll
    for (int i = threadIdx.x; i < 64 * PER; i += 256) {
        const int c = i / PER, r = i % PER * E;
        if (c0 + c < a.k && r0 + r < padded) *(u32x4*)(out + (c0 + c) * ldo + r0 + r) = turn_out(tiles[0], c, r);
    }
}

template <typename T>
__global__ __launch_bounds__(256) void k_clear(T* x, int64_t ld, int64_t rows, int64_t n)
{
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < rows * n; i += (int64_t)gridDim.x * 256) x[i / n * ld + i % n] = (T)0.0f;
}

// ---- up to 16 MT rows x: bound by reading the matrices once.  A workgroup takes 8 NT columns of the result, its waves parts of k; the first operand of
// a matrix instruction is eight rows of each matrix.  Here straight to registers, U steps at once, from rows that may begin anywhere: 64 bytes of a
// line at a time (one row of 4096 bfloat16 against 10752 of each matrix 35 us), and of rows that begin inside a word whole words and a shift (of 4097 70, 16
// rows 90).
constexpr int kFewRows = 32;
template <typename T, int MT, int NT, int U>
__global__ __launch_bounds__(1024) void k_gated_few(const T* x, int64_t ldx, const T* gate, int64_t ldg, const T* up, int64_t ldu, int m, int k, int f, int act, T* out,
                                                    int64_t ldo, float* pre)
{
    constexpr int K = 4 * kE<T>, SHARES = 16 / (MT * NT);
    __shared__ floatx4 sums[SHARES][MT * NT][64];
    const int lane = lane_id(), wave = threadIdx.x / 64, share = blockDim.x / 64, row = lane % 16, first = blockIdx.x * 8 * NT;
    const int steps = (k + K - 1) / K, begin = steps * wave / share, stop = steps * (wave + 1) / share, end = min(stop, k / K), t0 = lane / 16 * kE<T>;
    const T *w[NT], *xr[MT];
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        const int col = min(first + 8 * j + row % 8, f - 1);
        w[j] = (row < 8 ? gate + (int64_t)col * ldg : up + (int64_t)col * ldu) + t0;
    }
#pragma unroll
    for (int i = 0; i < MT; ++i) xr[i] = x + (int64_t)min(row + 16 * i, m - 1) * ldx + t0;
    floatx4 acc[MT][NT] = {};
    // U whole steps from s on; behind the last one it is asked for again, and not multiplied
    auto batch = [&](int s, auto full) __attribute__((always_inline)) {
        u32x4 a[U][MT], b[U][NT];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int t = (decltype(full)::value ? s + u : min(s + u, end - 1)) * K;
#pragma unroll
            for (int j = 0; j < NT; ++j) b[u][j] = load16_words(w[j] + t);
#pragma unroll
            for (int i = 0; i < MT; ++i) a[u][i] = load16_words(xr[i] + t);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (!decltype(full)::value && s + u >= end) break;
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int j = 0; j < NT; ++j) acc[i][j] = multiply(T{}, b[u][j], a[u][i], acc[i][j]);
        }
    };
    int s = begin;
    for (; s + U <= end; s += U) batch(s, std::true_type{});
    if (s < end) batch(s, std::false_type{});
    if (stop > end && stop > begin) {                    // the last step of rows that are no whole steps
        const int t = end * K;
        u32x4 a[MT];
#pragma unroll
        for (int i = 0; i < MT; ++i) a[i] = load16(xr[i], t, k - t0);
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            const u32x4 b = load16(w[j], t, k - t0);
#pragma unroll
            for (int i = 0; i < MT; ++i) acc[i][j] = multiply(T{}, b, a[i], acc[i][j]);
        }
    }
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) sums[wave][i * NT + j][lane] = acc[i][j];
    __syncthreads();
    for (int q = wave; q < MT * NT; q += share) {
        floatx4 v = sums[0][q][lane];
        for (int p = 1; p < share; ++p) v += sums[p][q][lane];
        float u[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) u[e] = __shfl(v[e], lane ^ 32);         // (lanes 32 .. 63 hold up's sums)
        const int r = row + q / NT * 16, c = first + q % NT * 8 + lane / 16 * 4;
        if (lane >= 32 || r >= m) continue;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (c + e >= f) continue;
            float slope;
            out[r * ldo + c + e] = (T)(act_value(v[e], act, slope) * u[e]);
            if (pre) {
                pre[(int64_t)r * 2 * f + c + e] = v[e];
                pre[((int64_t)r * 2 + 1) * f + c + e] = u[e];
            }
        }
    }
}

// ---- the same for rows at multiples of 16 bytes: whole lines, straight to LDS.  Every wave has a ring of D blocks of 128 bytes of k of its own: of NT times
// eight rows of each matrix, and of 8 XT rows x; no barrier but for the sums of the waves.  A load brings 8 rows, the 16-byte pieces of row r at
// place piece ^ r % 8, so that the lanes of a read lie in different banks.  k 4096, f 10752, bfloat16, us (through registers): 1 row 31.5 (35.4), 4 rows 31.9 (41),
// 16 rows 34.3 (56), 32 rows 41.6 (55); 5.6 TB/s for one row, start and end among them.
template <typename T, int NT, int XT, int D>
__global__ __launch_bounds__(512) void k_gated_ring(const T* x, int64_t ldx, const T* gate, int64_t ldg, const T* up, int64_t ldu, int m, int k, int f, int act, T* out,
                                                    int64_t ldo, float* pre)
{
    constexpr int MT = (XT + 1) / 2, LOADS = 2 * NT + XT;
    extern __shared__ __align__(1024) char lds[];
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), share = blockDim.x / 64, row = lane % 16, first = blockIdx.x * 8 * NT;
    const int bytes = k * (int)sizeof(T), blocks = (bytes + 127) / 128, begin = blocks * wave / share, end = blocks * (wave + 1) / share;
    const int piece = ((lane & 7) ^ (lane >> 3)) * 16;
    char* const ring = lds + wave * D * LOADS * 1024;
    // (offsets of rows from the first one: within 2^31 bytes, the host sees to it)
    uint32_t off[LOADS];
    const char *g0 = (const char*)(gate + (int64_t)first * ldg), *u0 = (const char*)(up + (int64_t)first * ldu);
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        const uint32_t r = min(8 * j + lane / 8, f - 1 - first);
        off[2 * j] = r * (uint32_t)(ldg * sizeof(T)) + piece;
        off[2 * j + 1] = r * (uint32_t)(ldu * sizeof(T)) + piece;
    }
#pragma unroll
    for (int i = 0; i < XT; ++i) off[2 * NT + i] = min(8 * i + lane / 8, m - 1) * (uint32_t)(ldx * sizeof(T)) + piece;
    auto request = [&](int block, int slot) __attribute__((always_inline)) {
        const int k0 = block * 128;
        const uint32_t back = k0 + piece < bytes ? 0 : piece;            // (pieces behind the rows' end: the block's first instead, and zeros later)
#pragma unroll
        for (int i = 0; i < LOADS; ++i)
            lds_dma16((i >= 2 * NT ? (const char*)x : (i & 1 ? u0 : g0)) + k0, off[i] - back, lds_addr(ring) + (slot * LOADS + i) * 1024);
    };
#pragma unroll
    for (int u = 0; u < D; ++u)
        if (begin + u < end) request(begin + u, u);
    floatx4 acc[MT][NT] = {};
    const int frag = row * 128, xfrag = 2 * NT * 1024 + row % (8 * min(XT, 2)) * 128, place = ((lane / 16) ^ (lane & 7)) * 16;
    for (int s0 = begin; s0 < end; s0 += D) {
#pragma unroll
        for (int u = 0; u < D; ++u) {
            const int s = s0 + u;
            if (s >= end) break;
            if (s + D <= end) wait_vmcnt<(D - 1) * LOADS>();
            else wait_vmcnt<0>();
            char* at = ring + u * LOADS * 1024;
            if (s == blocks - 1 && bytes % 128 && s * 128 + piece >= bytes) {
#pragma unroll
                for (int i = 0; i < LOADS; ++i) *(u32x4*)(at + i * 1024 + lane * 16) = u32x4{0, 0, 0, 0};
            }
            wave_sync();
            u32x4 a[2][MT], b[2][NT];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
#pragma unroll
                for (int j = 0; j < NT; ++j) b[h][j] = *(const u32x4*)(at + j * 2048 + frag + (place ^ (h * 64)));
#pragma unroll
                for (int i = 0; i < MT; ++i) a[h][i] = *(const u32x4*)(at + xfrag + i * 2048 + (place ^ (h * 64)));
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");           // the block is in registers: its place may be filled again
            if (s + D < end) request(s + D, u);
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int j = 0; j < NT; ++j) acc[i][j] = multiply(T{}, b[h][j], a[h][i], acc[i][j]);
        }
    }
    __syncthreads();                                     // (every wave's requests have landed and its blocks have been read)
    floatx4(*sums)[MT * NT][64] = (floatx4(*)[MT * NT][64])lds;
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) sums[wave][i * NT + j][lane] = acc[i][j];
    __syncthreads();
    for (int q = wave; q < MT * NT; q += share) {
        floatx4 v = sums[0][q][lane];
        for (int p = 1; p < share; ++p) v += sums[p][q][lane];
        float u[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) u[e] = __shfl(v[e], lane ^ 32);         // (lanes 32 .. 63 hold up's sums)
        const int r = row + q / NT * 16, c = first + q % NT * 8 + lane / 16 * 4;
        if (lane >= 32 || r >= m) continue;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (c + e >= f) continue;
            float slope;
            out[r * ldo + c + e] = (T)(act_value(v[e], act, slope) * u[e]);
            if (pre) {
                pre[(int64_t)r * 2 * f + c + e] = v[e];
                pre[((int64_t)r * 2 + 1) * f + c + e] = u[e];
            }
        }
    }
}

// ---- which kernel

// rows that requests of 16 bytes reach; offsets inside a tile are 32-bit numbers
static bool in_tiles(const void* p, int64_t ld, size_t es) { return (uintptr_t)p % 16 == 0 && ld * es % 16 == 0 && ld * es <= (1 << 22); }
static int check_gated(int64_t m, int64_t k, int64_t f, int32_t dtype, int32_t activation)
{
    if (!known_type(dtype)) return fail(HR_ERR_ARG, "unknown dtype %d", dtype);
    if (m < 0 || m > HR_GATED_MAX) return fail(HR_ERR_ARG, "m=%lld must be in 0..%d", (long long)m, HR_GATED_MAX);
    if (k < 1 || k > HR_GATED_MAX) return fail(HR_ERR_ARG, "k=%lld must be in 1..%d", (long long)k, HR_GATED_MAX);
    if (f < 1 || f > HR_GATED_MAX) return fail(HR_ERR_ARG, "f=%lld must be in 1..%d", (long long)f, HR_GATED_MAX);
    if (activation < HR_SILU || activation > HR_GELU_TANH) return fail(HR_ERR_ARG, "unknown activation %d", activation);
    // (workgroups of 64 x 64 elements of every matrix, and a launch may not have 2^32 threads)
    auto blocks = [](int64_t r, int64_t c) { return (r + 64) / 64 * ((c + 64) / 64); };
    if (blocks(m, 2 * f) + blocks(2 * f, k) + blocks(m, k) >= (1 << 24))
        return fail(HR_ERR_UNSUPPORTED, "m=%lld, k=%lld, f=%lld: larger matrices than one call takes", (long long)m, (long long)k, (long long)f);
    return HR_OK;
}

struct GatedArgs {
    const void* x; int64_t ldx;
    const void* gate; int64_t ldg;
    const void* up; int64_t ldu;
    int64_t m, k, f; int act;
    void* out; int64_t ldo; float* pre;
};

// workspace: x and both matrices with padded rows (whether a call copies them is known by its addresses only); sums of the parts of k
static size_t padded_bytes(int64_t m, int64_t k, int64_t f, size_t es) { return aligned((size_t)((m + 2 * f) * padded(k, es))); }

// Tiles and workspace of more than kFewRows rows.  The tiles are those of the next multiple of 64 rows, so that a workspace for fewer rows is found without
// asking for every number of them.
struct GatedPlan {
    Tiling tiling;
    TileArgs p;
    size_t sums, all;                                    // where they begin, and the end
};
static int64_t next_64(int64_t m) { return (m + 63) / 64 * 64; }
static GatedPlan gated_plan(int64_t m, int64_t k, int64_t f, size_t es)
{
    GatedPlan g{};
    g.p.m = next_64(m);
    g.p.n = f;
    g.p.k = (int)padded(k, es);
    g.tiling = plan_tiles(true, es, &g.p, 1);
    g.sums = padded_bytes(m, k, f, es);
    g.all = g.sums + sums_bytes(true, g.p) + HR_WORKSPACE_ALIGN;
    g.p.m = m;
    g.p.large = std::min(g.p.large, m);
    return g;
}
// The most that m rows or fewer take; a multiple of `step` rows takes as much as the fewer ones that go with it.  at_most(rows): a bound that falls with them.
template <typename F, typename G>
static size_t for_fewer_too(int64_t m, int64_t step, F&& takes, G&& at_most)
{
    size_t most = takes(m);
    for (int64_t rows = (m - 1) / step * step; rows > 0 && at_most(rows) > most; rows -= step) most = std::max(most, takes(rows));
    return most;
}

template <typename T>
static hipError_t launch_gated(const GatedArgs& g, const GatedPlan& plan, char* ws, hipStream_t s)
{
    constexpr size_t es = sizeof(T);
    if (g.m <= kFewRows) {
        auto ring = [&](auto kernel, int nt, int xt, int depth) {
            const int64_t groups = (g.f + 8 * nt - 1) / (8 * nt);
            const int share = few_share(groups, g.k * es, 4), lds = share * depth * (2 * nt + xt) * 1024;
            if (lds > 64 * 1024)
                if (hipError_t e = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024)) return e;
            hipLaunchKernelGGL(kernel, dim3((unsigned)groups), dim3(64 * share), lds, s, (const T*)g.x, g.ldx, (const T*)g.gate, g.ldg, (const T*)g.up, g.ldu, (int)g.m, (int)g.k, (int)g.f,
                               g.act, (T*)g.out, g.ldo, g.pre);
            return hipGetLastError();
        };
        auto go = [&](auto kernel, int columns, int most) {
            const int64_t groups = (g.f + columns - 1) / columns;
            hipLaunchKernelGGL(kernel, dim3((unsigned)groups), dim3(64 * few_share(groups, g.k * es, most)), 0, s, (const T*)g.x, g.ldx, (const T*)g.gate, g.ldg, (const T*)g.up, g.ldu,
                               (int)g.m, (int)g.k, (int)g.f, g.act, (T*)g.out, g.ldo, g.pre);
        };
        if (g.k * es % 16 == 0 && in_tiles(g.x, g.ldx, es) && in_tiles(g.gate, g.ldg, es) && in_tiles(g.up, g.ldu, es))
            return g.m <= 16 ? ring(k_gated_ring<T, 2, 2, 2>, 2, 2, 2) : ring(k_gated_ring<T, 2, 4, 3>, 2, 4, 3);
        if (g.m <= 4) go(k_gated_few<T, 1, 1, 8>, 8, 16);
        else if (g.m <= 16) go(k_gated_few<T, 1, 2, 4>, 16, 8);
        else go(k_gated_few<T, 2, 2, 4>, 16, 4);
        return hipGetLastError();
    }
    TileArgs p = plan.p;
    p.end = g.k * es % 16 == 0 ? (int)(g.k * es) : p.k;  // (behind it a copy has zeros, where there is one)
    // what tiles cannot take as it is is copied first, row by row
    struct { const void* at; int64_t ld, rows; const char** to; int64_t* lds; } in[3] = {
        {g.x, g.ldx, g.m, &p.a, &p.lda}, {g.gate, g.ldg, g.f, &p.b, &p.ldb}, {g.up, g.ldu, g.f, &p.up, &p.ldup}};
    PadArgs pad{};
    pad.n = (int)g.k;
    pad.out = ws;
    pad.ldo = p.k;
    int64_t copied = 0;
    for (int i = 0; i < 3; ++i) {
        const bool fits = g.k * es % 16 == 0 && in_tiles(in[i].at, in[i].ld, es);
        pad.x[i] = in[i].at;
        pad.ld[i] = in[i].ld;
        pad.rows[i] = fits ? 0 : in[i].rows;
        *in[i].to = fits ? (const char*)in[i].at : ws + copied * p.k;
        *in[i].lds = fits ? in[i].ld * (int64_t)es : p.k;
        copied += pad.rows[i];
    }
    if (copied > 0) {
        hipLaunchKernelGGL(k_pad<T>, dim3((unsigned)std::min<int64_t>((copied * (p.k / 16) + 255) / 256, 1 << 20)), dim3(256), 0, s, pad);
        if (hipError_t e = hipGetLastError()) return e;
    }
    p.out = g.out;
    p.ldo = g.ldo;
    p.pre = g.pre;
    p.act = g.act;
    p.sums = (float*)(ws + plan.sums);
    return launch_tiles<T, true>(plan.tiling, TilePair{{p}}, 1, s);
}

// workspace of the gradients: those of gate and up as rows, [m][2 fp], and as columns, [2 f][mp]; both matrices turned, [k][2 fp]; x turned, [k][mp];
// bits of the largest of each row and of each column (binary16), sums of the parts of the products' k.  fp, mp: whole blocks.
struct BackwardPlan {
    int64_t fp, mp;                                      // elements
    size_t rows, cols, w, x, largest, sums, sums2, all;  // where each begins, and the end
    Tiling tiling;
    TileArgs p[2];                                       // the product for x's gradient, the one for the matrices' (the same parts whichever are wanted)
};
static BackwardPlan backward_plan(int64_t m, int64_t k, int64_t f, int32_t dtype, bool tiles = true)
{
    const size_t es = element_bytes(dtype);
    const bool raised = dtype == HR_F16;
    BackwardPlan p{};
    const int64_t fb = padded(f, es), mb = padded(m, es);
    p.fp = fb / es;
    p.mp = mb / es;
    p.rows = 0;
    p.cols = p.rows + aligned((size_t)(m * 2 * fb));
    p.w = p.cols + aligned((size_t)(2 * f * mb));
    p.x = p.w + aligned((size_t)(k * 2 * fb));
    p.largest = p.x + aligned((size_t)(k * mb));
    p.sums = p.largest + (raised ? aligned((size_t)(m + 2 * f) * 4) : 0);
    p.all = p.sums + HR_WORKSPACE_ALIGN;
    if (m == 0 || !tiles) return p;
    for (int i = 0; i < 2; ++i) {
        TileArgs& t = p.p[i];
        t.m = i ? 2 * f : p.mp;                          // (whole blocks of rows: see gated_plan)
        t.n = k;
        t.k = t.end = (int)(i ? mb : 2 * fb);
        t.lda = t.ldb = t.k;
    }
    p.tiling = plan_tiles(false, es, p.p, 2);
    p.sums2 = p.sums + sums_bytes(false, p.p[0]);
    p.all = p.sums2 + sums_bytes(false, p.p[1]) + HR_WORKSPACE_ALIGN;
    p.p[0].m = m;
    p.p[0].large = std::min(p.p[0].large, m);
    return p;
}

// most that the sums of parts of k of a product take: see plan_tiles
static size_t most_sums(int64_t m, int64_t n, size_t es) { return (size_t)std::min<int64_t>(kMostSums, kMostParts * m * n * (int64_t)es) + HR_WORKSPACE_ALIGN; }

}  // namespace hr

// ---- C entry points
using namespace hr;

extern "C" {

size_t hr_gated_workspace_bytes(int64_t m, int64_t k, int64_t f, int32_t dtype)
{
    if (check_gated(m, k, f, dtype, HR_SILU)) return 0;
    const size_t es = element_bytes(dtype);
    if (m <= kFewRows) return HR_WORKSPACE_ALIGN;
    return for_fewer_too(m, 64, [&](int64_t rows) { return gated_plan(rows, k, f, es).all; },
                         [&](int64_t rows) { return padded_bytes(rows, k, f, es) + most_sums(rows, f, 8) + HR_WORKSPACE_ALIGN; });
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
    const GatedPlan plan = m > kFewRows ? gated_plan(m, k, f, es) : GatedPlan{};
    if (int rc = check_workspace(workspace, workspace_bytes, std::max<size_t>(plan.all, HR_WORKSPACE_ALIGN))) return rc;
    const GatedArgs g{x, ldx, w_gate, ldwg, w_up, ldwu, m, k, f, activation, out, ldo, out_pre};
    HR_HIP(with_type(dtype, [&](auto t) { return launch_gated<decltype(t)>(g, plan, (char*)workspace, (hipStream_t)stream); }));
    return HR_OK;
}

size_t hr_gated_backward_workspace_bytes(int64_t m, int64_t k, int64_t f, int32_t dtype)
{
    if (check_gated(m, k, f, dtype, HR_SILU)) return 0;
    const int64_t step = 128 / (int64_t)element_bytes(dtype);
    return for_fewer_too(m, step, [&](int64_t rows) { return backward_plan(rows, k, f, dtype).all; },
                         [&](int64_t rows) {
                             const BackwardPlan p = backward_plan(rows, k, f, dtype, false);
                             return p.sums + most_sums(rows, k, 4) + most_sums(2 * f, k, 4) + HR_WORKSPACE_ALIGN;
                         });
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
    const BackwardPlan plan = backward_plan(m, k, f, dtype);
    if (int rc = check_workspace(workspace, workspace_bytes, plan.all)) return rc;
    if (!grad_x && !grad_w_gate) return HR_OK;
    hipStream_t s = (hipStream_t)stream;
    char *rows = (char*)workspace + plan.rows, *cols = (char*)workspace + plan.cols, *turned_w = (char*)workspace + plan.w, *turned_x = (char*)workspace + plan.x;
    HR_HIP(with_type(dtype, [&](auto t) -> hipError_t {
        using T = decltype(t);
        if (m == 0) {                                    // (sums over no rows)
            if (!grad_w_gate) return hipSuccess;
            const unsigned blocks = (unsigned)std::min<int64_t>((f * k + 255) / 256, 1 << 20);
            hipLaunchKernelGGL(k_clear<T>, dim3(blocks), dim3(256), 0, s, (T*)grad_w_gate, ldgg, f, k);
            hipLaunchKernelGGL(k_clear<T>, dim3(blocks), dim3(256), 0, s, (T*)grad_w_up, ldgu, f, k);
            return hipGetLastError();
        }
        LayOutArgs l{pre, grad_out, ldgo, activation, w_gate, ldwg, w_up, ldwu, x, ldx, (int)m, (int)k, (int)f, (int)plan.fp, (int)plan.mp};
        l.rows = grad_x ? rows : nullptr;
        l.cols = grad_w_gate ? cols : nullptr;
        l.turned_w = turned_w;
        l.turned_x = turned_x;
        auto blocks = [](int64_t r, int64_t c) { return (int)((r + 63) / 64 * ((c + 63) / 64)); };
        uint32_t* const largest = (uint32_t*)((char*)workspace + plan.largest);
        if constexpr (kRaised<T>) {
            l.of_row = largest;
            l.of_col = largest + m;
            const int64_t words = m + 2 * f, across = (f + 511) / 512;
            hipLaunchKernelGGL(k_clear<float>, dim3((unsigned)std::min<int64_t>((words + 255) / 256, 1 << 20)), dim3(256), 0, s, (float*)largest, words, (int64_t)1, words);
            // (a thousand workgroups where there is work for them, at least 8 rows each)
            const int64_t take = std::max<int64_t>(8, std::min<int64_t>(256, m * across / 1024 / 8 * 8));
            hipLaunchKernelGGL(k_largest<T>, dim3((unsigned)across, (unsigned)((m + take - 1) / take)), dim3(256), 0, s,
                               LargestArgs{pre, grad_out, ldgo, activation, (int)m, (int)f, (int)take, largest, largest + m});
        }
        l.blocks_d = blocks(plan.mp, plan.fp);
        l.blocks_w = blocks(plan.fp, k);
        hipLaunchKernelGGL(k_lay_out<T>, dim3((unsigned)(l.blocks_d + (grad_x ? 2 * l.blocks_w : 0) + (grad_w_gate ? blocks(plan.mp, k) : 0))), dim3(256), 0, s, l);
        TilePair pair{};
        int count = 0;
        if (grad_x) {
            TileArgs& p = pair.p[count++] = plan.p[0];
            p.sums = (float*)((char*)workspace + plan.sums);
            p.a = rows;
            p.largest = largest;
            p.b = turned_w;
            p.out = grad_x;
            p.ldo = ldgx;
            p.split = m;
        }
        if (grad_w_gate) {
            TileArgs& p = pair.p[count++] = plan.p[1];
            p.sums = (float*)((char*)workspace + plan.sums2);
            p.a = cols;
            p.largest = largest + m;
            p.b = turned_x;
            p.out = grad_w_gate;
            p.out2 = grad_w_up;
            p.ldo = ldgg;
            p.ldo2 = ldgu;
            p.split = f;
        }
        if (hipError_t e = launch_tiles<T, false>(plan.tiling, pair, count, s)) return e;
        return hipGetLastError();
    }));
    return HR_OK;
}

}  // extern "C"
