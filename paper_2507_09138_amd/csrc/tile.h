// Products of floating point matrices in tiles (16-bit types and float32), and the gated block's arithmetic: what gated*.hip share.
#pragma once
#include <type_traits>

#include "common.h"
#include "hr_layers.h"
#include "wave.h"

namespace hr {

// ---- activations: the value and the slope.  All three are z times a share p of 0 .. 1 that one exponential gives; 2^x and 1 / x as the hardware has them
// (within a unit of the last place).  GELU is off by at most 8 units of its own last place wherever it is a normal number; the other two by a few units of the
// last place of z, below 0 relative to themselves by |z| of them.
constexpr float kLog2e = 1.4426950408889634f, kSqrt2OverPi = 0.7978845608028654f, kOverSqrt2Pi = 0.3989422804014327f, kLn2 = 0.6931471805599453f;

// The normal distribution p(z) and e = exp(-z^2 / 2), from polynomials fitted for this (least largest relative error).  |z| <= 1: (p - 1 / 2) / z, even, in z^2
// (1e-9).  Beyond: p(-|z|) = e t P(t), t = 1 / (1 + 0.4 |z|), up to 13.4, where e leaves float32's range (0.8e-7).  e is taken with what z^2 and its
// product with log2 e are off by (without: 5e-6 of e at 12).
__device__ __forceinline__ float normal_share(float z, float& e)
{
    constexpr float kHalf = -0.5f * kLog2e, kHalfRest = -9.62981517e-9f;                     // -log2 e / 2, and what float32 lacks of it
    const float x = fminf(fabsf(z), 16.0f), t = __builtin_amdgcn_rcpf(fmaf(x, 0.4f, 1.0f));
    const float square = x * x, rest = fmaf(x, x, -square), power = square * kHalf;
    const float off = fmaf(square, kHalf, -power) + fmaf(rest, kHalf, square * kHalfRest);
    e = __builtin_amdgcn_exp2f(power);
    e = fmaf(e, off * kLn2, e);
    const float q = fmaf(t, fmaf(t, fmaf(t, fmaf(t, fmaf(t, fmaf(t, 0.0681211948f, -0.186427504f), 0.105362579f), 0.0555409156f), 0.139002189f), 0.159100011f), 0.159595788f) * t * e;
    const float s = fmaf(square, fmaf(square, fmaf(square, fmaf(square, fmaf(square, -7.65420828e-06f, 0.000113486371f), -0.00118632999f), 0.00997332297f), -0.0664903596f), 0.398942292f);
    return x <= 1.0f ? fmaf(z, s, 0.5f) : z < 0.0f ? q : 1.0f - q;
}

__device__ __forceinline__ float act_value(float z, int act, float& slope)
{
    if (act == HR_GELU) {
        float e;
        const float p = normal_share(z, e);
        slope = fmaf(z * e, kOverSqrt2Pi, p);
        return z * p;
    }
    float y = z, dy = 1.0f;
    if (act == HR_GELU_TANH) {                           // (1 + tanh y) / 2 = 1 / (1 + exp(-2 y)); beyond 50 it is 0 or 1
        const float c = fminf(fmaxf(z, -50.0f), 50.0f), c2 = c * c;
        y = 2 * kSqrt2OverPi * c * fmaf(0.044715f, c2, 1.0f);
        dy = 2 * kSqrt2OverPi * fmaf(3 * 0.044715f, c2, 1.0f);
    }
    const float p = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(y * -kLog2e));
    slope = fmaf(z * (1.0f - p) * p, dy, p);
    return z * p;
}

// Gradients of gate and up in binary16 have a power of two for each of their rows, and in the copy that is turned for each of their columns: with it the
// largest of them lies in 2^14 .. 2^15, so that none is too large for the type and those that are too small for it are less than a rounding of what they
// are added to.  Here its exponent, from the bits of that largest magnitude (0 where it is 0, infinite or NaN).  Multiplying by it is exact.
__device__ __forceinline__ int raised_by(uint32_t largest)
{
    return largest == 0 || largest >= 0x7f800000u ? 0 : 141 - (int)(largest >> 23);
}
template <typename T> constexpr bool kRaised = std::is_same_v<T, _Float16>;

// 16 bytes of k a lane, lane l those of row l % 16 from byte 16 (l / 16) on of a step of 64: one matrix instruction of 16 bits, four of 32 (the
// k of a step in another order, the same for both operands).  The first operand's rows are the result's rows, four of them in the registers of
// lane l, 4 (l / 16) .. + 3, in column l % 16: with the rows of b first a lane holds four neighbouring outputs of a row of a.
__device__ __forceinline__ floatx4 multiply(_Float16, u32x4 b, u32x4 a, floatx4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, b), __builtin_bit_cast(half8, a), c, 0, 0, 0);
}
__device__ __forceinline__ floatx4 multiply(__bf16, u32x4 b, u32x4 a, floatx4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, b), __builtin_bit_cast(bf16x8, a), c, 0, 0, 0);
}
__device__ __forceinline__ floatx4 multiply(float, u32x4 b, u32x4 a, floatx4 c)
{
#pragma unroll
    for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(__builtin_bit_cast(float, (uint32_t)b[e]), __builtin_bit_cast(float, (uint32_t)a[e]), c, 0, 0, 0);
    return c;
}

// What tiles take: out[i, j] = sum_t a[i, t] b[j, t], all distances in bytes.  Rows begin at multiples of 16 bytes and are a multiple of 16 long.
struct TileArgs {
    const char* a; int64_t lda;
    const char* b; int64_t ldb;                          // gated: the gate's matrix
    const char* up; int64_t ldup;                        // gated: up's
    int64_t m, n; int k, end;                            // n: columns of the result; end: the length of a row, k: that in whole blocks of 128
    int64_t row0, large;                                 // its first row here; how many rows large tiles take, the others small ones (set by plan_tiles)
    int parts, part_k;                                   // parts of k (part_k bytes each, a multiple of 128), and where there are more than one
    int slots;                                           // workgroups, a multiple of 8
    float* sums;                                         // their sums, [parts][m][n], gated [parts][m][2][n]
    void* out; int64_t ldo;                              // elements apart
    void* out2; int64_t ldo2, split;                     // rows from `split` on go to out2
    float* pre; int act;                                 // gated
    const uint32_t* largest;                             // kRaised gradients: bits of the largest magnitude of each row of a, which is raised by its power of two
};

// One product, or two in one launch: workgroups from `first` on are the second's.
struct TilePair {
    TileArgs p[2];
    unsigned first;
};

// N neighbouring outputs of a row, as far as they are there
template <int N, typename O>
__device__ __forceinline__ void store_some(O* at, int64_t col, int64_t n, const float* v)
{
    typedef O outs __attribute__((ext_vector_type(N)));
    outs o;
#pragma unroll
    for (int e = 0; e < N; ++e) o[e] = (O)v[e];
    if (col + N <= n) {
        __builtin_memcpy(at + col, &o, sizeof o);
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (col + e < n) at[col + e] = o[e];
    }
}

// N neighbouring results of a row: of both matrices where the block is gated.
template <typename T, bool GATED, int N>
__device__ __forceinline__ void finish(const TileArgs& p, int64_t row, int64_t col, const float* v, const float* up)
{
    row += p.row0;
    if constexpr (GATED) {
        float h[N], slope;
#pragma unroll
        for (int e = 0; e < N; ++e) h[e] = act_value(v[e], p.act, slope) * up[e];
        store_some<N>((T*)p.out + row * p.ldo, col, p.n, h);
        if (p.pre) {
            store_some<N>(p.pre + row * 2 * p.n, col, p.n, v);
            store_some<N>(p.pre + (row * 2 + 1) * p.n, col, p.n, up);
        }
    } else if constexpr (kRaised<T>) {
        const int by = raised_by(p.largest[row]);
        float x[N];
#pragma unroll
        for (int e = 0; e < N; ++e) x[e] = __builtin_ldexpf(v[e], -by);
        store_some<N>(row < p.split ? (T*)p.out + row * p.ldo : (T*)p.out2 + (row - p.split) * p.ldo2, col, p.n, x);
    } else {
        store_some<N>(row < p.split ? (T*)p.out + row * p.ldo : (T*)p.out2 + (row - p.split) * p.ldo2, col, p.n, v);
    }
}

// ---- tiles of BM x BN, a wave's share of them WM x 64.  Gated: the tile's BN rows b are BN / 2 of each matrix.
// Blocks of 128 bytes of k of both sides go straight to LDS, into one of NB buffers; rows of 128 bytes, whole lines.  A wave's load
// brings 8 rows; the 16-byte pieces of row r lie at place piece ^ r % 8, so that the lanes of a read lie in different banks.  The fragments of a
// step of 64 bytes are read while the step before is multiplied; where those of a block's second step have been read by all waves its buffer is
// filled again: one barrier a block.  Where there is no more than a tile for every compute unit nothing else hides the time that loads take: NB
// buffers, all but one on their way.  Else a workgroup goes from tile to tile and asks for the next one's first blocks before it writes its outputs.
// Bound by matrix instructions at the clock that power leaves (1.72 GHz, busy 68 % of it, no bank conflicts).  Gated, 8192 x 4096 x 10752 of both matrices,
// bfloat16 1210 us (1.19 P/s, with 705 MB of gate and up written; a library's product alone 1090); 8192 x 4096 x 21504 1210 (library 1083), 21504 x 4096 x
// 8192 1180 .. 1300 (1003), 4096^3 102 (92).  float32 141 T/s between start and end, of 154.
// TAIL: rows that are no whole blocks; with what they need for it the others would be 4 % slower.
template <typename T, bool GATED, int BM, int BN, int WM, int NB, bool TAIL>
__global__ __launch_bounds__(BM / WM * (BN / 64) * 64) void k_tiles(TilePair pair)
{
    const bool second = blockIdx.x >= pair.first;
    const TileArgs& p = pair.p[second];
    const int slot = (int)(blockIdx.x - (second ? pair.first : 0));
    constexpr int WN = 64, WAVES = BM / WM * (BN / WN), TM = WM / 16, TN = 4, BK = 128, UNITS = (BM + BN) / 8 / WAVES, BUF = (BM + BN) * BK;
    constexpr int COLS = GATED ? BN / 2 : BN;            // of the result
    static_assert(BM / 8 % WAVES == 0 && BN / 8 % WAVES == 0 && NB >= 2 && NB <= 4);
    extern __shared__ __align__(1024) char lds[];
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int wm = wave / (BN / WN) * WM, wn = wave % (BN / WN) * WN;
    const int piece = ((lane & 7) ^ (lane >> 3)) * 16;
    const uint32_t lds0 = lds_addr(lds);

    // Tiles that run at the same time on an XCD share its L2: each has a stretch of the parts' tiles, and takes them in blocks of four rows of tiles.
    const int m = (int)p.m, n = (int)p.n, tiles_m = (m + BM - 1) / BM, tiles_n = (n + COLS - 1) / COLS, tiles = tiles_m * tiles_n;
    const int stretch = (tiles * p.parts + 7) / 8, item0 = slot % 8 * stretch, end = min(stretch, tiles * p.parts - item0);
    int item = slot / 8, part = 0, k_begin = 0, blocks = 0, m0 = 0, n0 = 0;
    uint32_t off[UNITS];                                 // (rows of a tile lie within 2^31 bytes: the host sees to it)
    const char *ga = p.a, *gb = p.b, *gu = p.up;
    // What lies in row r of b's part of a buffer.  Rows 0 .. 15 and 16 .. 31 of 32 are four of each eight columns, so that a lane has eight neighbouring
    // outputs in two fragments; gated: 32 rows of the gate, then the same 32 of up.
    auto column_of = [&](int r) __attribute__((always_inline)) {
        const int c = (r & 12) << 1 | (r & 16) >> 2 | (r & 3);
        return GATED ? r / 64 * 32 + c : (r & ~31) | c;
    };
    auto is_up = [&](int i) __attribute__((always_inline)) { return GATED && (((i * WAVES + wave) * 8 - BM) & 32) != 0; };       // (of a load: the same for its 8 rows)
    auto aim = [&](int t) __attribute__((always_inline)) {
        part = (t + item0) / tiles;
        k_begin = part * p.part_k;
        blocks = (min(p.k, k_begin + p.part_k) - k_begin) / BK;
        t = t + item0 - part * tiles;
        const int g = t / (4 * tiles_n), rest = t - g * 4 * tiles_n, high = min(4, tiles_m - g * 4);
        m0 = (g * 4 + rest % high) * BM;
        n0 = rest / high * COLS;
        ga = p.a + (int64_t)m0 * p.lda;
        gb = p.b + (int64_t)n0 * p.ldb;
        if (GATED) gu = p.up + (int64_t)n0 * p.ldup;
#pragma unroll
        for (int i = 0; i < UNITS; ++i) {
            const int row = (i * WAVES + wave) * 8 + lane / 8;
            off[i] = (i * WAVES * 8 < BM ? (uint32_t)min(row, m - 1 - m0) * (uint32_t)p.lda
                                         : (uint32_t)min(column_of(row - BM), n - 1 - n0) * (uint32_t)(is_up(i) ? p.ldup : p.ldb)) + piece;
        }
    };
    auto request = [&](int block) __attribute__((always_inline)) {
        const int k0 = k_begin + block * BK;
        const uint32_t back = TAIL && k0 + piece >= p.end ? piece : 0;        // (pieces behind the rows' end: the block's first instead, and zeros later)
#pragma unroll
        for (int i = 0; i < UNITS; ++i)
            lds_dma16((i * WAVES * 8 < BM ? ga : (is_up(i) ? gu : gb)) + k0, off[i] - back, lds0 + (uint32_t)block % NB * BUF + (i * WAVES + wave) * 1024);
    };

    const int frag = (lane % 16) * BK + ((lane / 16) ^ (lane & 7)) * 16;
    floatx4 acc[TM][TN];
    u32x4 a[TM], b0[TN], b1[TN];
    auto place = [&](int block, int ks) __attribute__((always_inline)) { return lds + ((frag ^ (ks * 64)) + (uint32_t)block % NB * BUF); };
    auto read_b = [&](u32x4* f, int block, int ks) __attribute__((always_inline)) {
        const char* at = place(block, ks) + (BM + wn) * BK;
#pragma unroll
        for (int j = 0; j < TN; ++j) f[j] = *(const u32x4*)(at + j * 16 * BK);
    };
    // one step: fragments a and b; where a fragment of a has been used for the last time the next step's takes its registers
    // (at a raised priority: the wave that shares the SIMD and is behind does its reads and requests in between)
    auto step = [&](const u32x4* b, const char* next) __attribute__((always_inline)) {
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int i = 0; i < TM; ++i) {
#pragma unroll
            for (int j = 0; j < TN; ++j) acc[i][j] = multiply(T{}, b[j], a[i], acc[i][j]);
            a[i] = *(const u32x4*)(next + (wm + i * 16) * BK);
        }
        __builtin_amdgcn_s_setprio(0);
    };
    // Everything asked for has landed, up to block `next`, but for `behind` blocks that were asked for last, everything read is in registers: of all waves.
    auto meet = [&](int next, int behind) __attribute__((always_inline)) {
        if (NB > 2 && behind >= 2) wait_vmcnt<2 * UNITS>();
        else if (NB > 2 && behind == 1) wait_vmcnt<UNITS>();
        else wait_vmcnt<0>();
        if (const int k0 = k_begin + next * BK; TAIL && k0 + BK > p.end && next < blocks) {      // (what this wave asked for behind the rows' end)
            if (k0 + piece >= p.end) {
#pragma unroll
                for (int i = 0; i < UNITS; ++i) *(u32x4*)(lds + (uint32_t)next % NB * BUF + (i * WAVES + wave) * 1024 + lane * 16) = u32x4{0, 0, 0, 0};
            }
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };

    if (item >= end) return;
    aim(item);
#pragma unroll
    for (int b = 0; b < NB; ++b)
        if (b < blocks) request(b);
    for (;;) {
        meet(0, min(blocks, NB) - 1);
        read_b(b0, 0, 0);
#pragma unroll
        for (int i = 0; i < TM; ++i) a[i] = *(const u32x4*)(place(0, 0) + (wm + i * 16) * BK);
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j) acc[i][j] = floatx4{0, 0, 0, 0};
        for (int b = 0; b < blocks; ++b) {
            read_b(b1, b, 1);
            step(b0, place(b, 1));
            meet(b + 1, min(blocks - 2 - b, NB - 2));           // (nobody reads this block's buffer any more, the next block has landed)
            if (b + NB < blocks) request(b + NB);
            read_b(b0, b + 1, 0);                        // (behind the last block: whatever the buffer holds, not multiplied)
            step(b1, place(b + 1, 0));
        }
        const int mt = m0, nt = n0, of = part;
        item += p.slots / 8;
        const bool more = NB == 2 && item < end;         // (with more buffers the host launches a workgroup for every tile)
        if (more) {
            aim(item);
            request(0);                                  // (both buffers are free since the last meeting)
            if (blocks > 1) request(1);
        }
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            const int64_t row = mt + wm + i * 16 + lane % 16;
            if (row >= m) continue;
#pragma unroll
            for (int j = 0; j < TN; j += GATED ? 4 : 2) {
                const int64_t col = nt + (GATED ? wn / 2 : wn + j * 16) + lane / 16 * 8;
                float v[8], up[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    v[e] = acc[i][j + e / 4][e % 4];
                    if (GATED) up[e] = acc[i][(j + 2 + e / 4) % TN][e % 4];
                }
                if (p.parts > 1) {
                    float* at = p.sums + ((int64_t)of * m + row) * (GATED ? 2 : 1) * n;
                    store_some<8>(at, col, n, v);
                    if (GATED) store_some<8>(at + n, col, n, up);
                } else {
                    finish<T, GATED, 8>(p, row, col, v, up);
                }
            }
        }
        if (!more) break;
    }
}

// Adds up the parts of k (memory: 75 MB in 19 us, 4 TB/s): SHARES threads take every SHARES-th part of four columns, in order, and their sums are added in order.
template <typename T, bool GATED, int SHARES>
__global__ __launch_bounds__(256) void k_tiles_join(TilePair pair)
{
    const bool second = blockIdx.x >= pair.first;
    const TileArgs& p = pair.p[second];
    const int64_t block = blockIdx.x - (second ? pair.first : 0), blocks = second ? gridDim.x - pair.first : pair.first;
    constexpr int PER = 256 / SHARES;
    __shared__ floatx4 some[GATED ? 2 : 1][SHARES][PER];
    const int64_t fours = (p.n + 3) / 4, all = p.m * fours, stride = p.m * p.n * (GATED ? 2 : 1);
    const int at = threadIdx.x % PER, share = threadIdx.x / PER;
    for (int64_t i0 = block * PER; i0 < all; i0 += blocks * PER) {
        const int64_t i = min(i0 + at, all - 1), row = i / fours, col = (i - row * fours) * 4;
        const float* from = p.sums + row * (GATED ? 2 : 1) * p.n + col;
        const bool whole = col + 4 <= p.n;
        auto load = [&](const float* x) __attribute__((always_inline)) {
            floatx4 v = {0, 0, 0, 0};
            if (whole) {
                __builtin_memcpy(&v, x, 16);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (col + e < p.n) v[e] = x[e];
            }
            return v;
        };
        floatx4 v = {0, 0, 0, 0}, up = {0, 0, 0, 0};
#pragma unroll 4
        for (int s = share; s < p.parts; s += SHARES) {
            v += load(from + s * stride);
            if (GATED) up += load(from + s * stride + p.n);
        }
        if constexpr (SHARES > 1) {
            __syncthreads();
            some[0][share][at] = v;
            if (GATED) some[GATED ? 1 : 0][share][at] = up;
            __syncthreads();
            if (share > 0) continue;
#pragma unroll
            for (int q = 1; q < SHARES; ++q) {
                v += some[0][q][at];
                if (GATED) up += some[GATED ? 1 : 0][q][at];
            }
        }
        if (i0 + at < all) {
            float a[4], b[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) a[e] = v[e], b[e] = up[e];
            finish<T, GATED, 4>(p, row, col, a, b);
        }
    }
}

// ---- host: which tiles (gated.hip), and their launches
constexpr int kComputeUnits = 256;
struct Tiling { int bm, bn; };
// Of count products, 1 or 2.
template <typename T, bool GATED>
hipError_t launch_tiles(const Tiling& t, const TilePair& pair, int count, hipStream_t s);

}  // namespace hr
