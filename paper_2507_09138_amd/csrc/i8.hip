// Products in 8-bit integers with a scale for each row of both matrices, and the quantisation of rows (hr_scores.h).
#include <algorithm>
#include <type_traits>

#include "entry.h"
#include "i8_few.h"
#include "row_math.h"

namespace hr {


constexpr int kStep = 64;                                // bytes of k that one matrix instruction takes
constexpr int kStaticLds = 64 * 1024;                    // what a launch may ask for without saying so beforehand

struct QuantizeArgs {
    const void* x; int64_t ldx, m; int k;
    int8_t* q; int64_t ldq; float* scale;
    int padded;                                          // places that a row has in q, those behind k to be zeros
};

// ---- quantisation.  Rows are taken in pieces of 16 elements: 16 bytes of the result.
template <typename T>
__device__ __forceinline__ void load_piece(const T* row, int t, int k, float* v)        // zeros from element k on
{
    if (t + 16 <= k) {
        T x[16];
        __builtin_memcpy(x, row + t, sizeof x);          // (rows may start at any element)
#pragma unroll
        for (int e = 0; e < 16; ++e) v[e] = (float)x[e];
    } else {
#pragma unroll
        for (int e = 0; e < 16; ++e) v[e] = t + e < k ? (float)row[t + e] : 0.0f;
    }
}
// The largest magnitude of a piece as the bits of a float: in order, infinities and NaNs above all others.
__device__ __forceinline__ uint32_t largest_bits(const float* v)
{
    uint32_t b = 0;
#pragma unroll
    for (int e = 0; e < 16; ++e) b = max(b, __builtin_bit_cast(uint32_t, v[e]) & 0x7fffffffu);
    return b;
}
__device__ __forceinline__ float quant_scale(uint32_t largest) { return largest >= 0x7f800000u ? NAN : bits_float(largest) / 127.0f; }
// The quotient rounded to float32, then to a whole number.  A product with the reciprocal is off by 2^-23 of itself, 1.5e-5 at most: only
// where it lies that near to the middle of two whole numbers the quotient itself is needed.  A scale that small has no reciprocal, and where it is
// below 2^-126 few bits: the largest quotients may be up to 190, and are limited to 127.
__device__ __forceinline__ u32x4 quant_piece(const float* v, float scale)
{
    if (!(scale > 0.0f)) return u32x4{0, 0, 0, 0};
    const float inv = 1.0f / scale;
    float q[16];
    bool near = !(scale > 1e-37f);
#pragma unroll
    for (int e = 0; e < 16; ++e) {
        const float y = v[e] * inv;
        q[e] = rintf(y);
        near |= fabsf(y - q[e]) > 0.5f - 0x1p-15f;
    }
    if (near) {
#pragma unroll
        for (int e = 0; e < 16; ++e) q[e] = fminf(fmaxf(rintf(v[e] / scale), -127.0f), 127.0f);
    }
    uint32_t w[4];
#pragma unroll
    for (int d = 0; d < 4; ++d) {
        w[d] = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) w[d] |= ((uint32_t)(int)q[4 * d + e] & 0xffu) << (8 * e);
    }
    return u32x4{w[0], w[1], w[2], w[3]};
}

// LANES lanes take a row: 4 or 16 of a wave, a wave, or the workgroup.  Rows of up to PIECES pieces per lane are held in registers
// between the search for the largest magnitude and the rounding, longer ones are read again.
template <typename T, int LANES, int PIECES>
__global__ __launch_bounds__(256) void k_quantize(QuantizeArgs a)
{
    constexpr int ROWS = 256 / LANES;
    __shared__ uint32_t part[4];
    const int t = threadIdx.x % LANES;
    const int npieces = (a.k + 15) / 16;
    const bool whole = a.ldq % 16 == 0 && (uintptr_t)a.q % 16 == 0;
    for (int64_t r0 = (int64_t)blockIdx.x * ROWS; r0 < a.m; r0 += (int64_t)gridDim.x * ROWS) {
        const int64_t r = r0 + threadIdx.x / LANES;
        const bool in = r < a.m;
        const T* row = (const T*)a.x + (in ? r : a.m - 1) * a.ldx;
        float v[PIECES][16];
        uint32_t largest = 0;
        for (int p0 = 0; p0 < npieces; p0 += PIECES * LANES) {
#pragma unroll
            for (int i = 0; i < PIECES; ++i) {
                const int p = p0 + i * LANES + t;
                if (p < npieces) load_piece(row, p * 16, a.k, v[i]);
            }
#pragma unroll
            for (int i = 0; i < PIECES; ++i)
                if (p0 + i * LANES + t < npieces) largest = max(largest, largest_bits(v[i]));
        }
        // (of four or sixteen neighbouring lanes: lane ^ 1, ^ 2, the other four of eight, the other eight of sixteen)
        auto fold = [&](auto ctrl) __attribute__((always_inline)) {
            largest = max(largest, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)largest, decltype(ctrl)::value, 0xf, 0xf, false));
        };
        if (LANES <= 16) {
            fold(std::integral_constant<int, 0xb1>{});
            fold(std::integral_constant<int, 0x4e>{});
        }
        if (LANES == 16) {
            fold(std::integral_constant<int, 0x141>{});
            fold(std::integral_constant<int, 0x140>{});
        }
        if (LANES >= 64) largest = wave_fold(largest, [](uint32_t x, uint32_t y) { return x > y ? x : y; });
        if (LANES > 64) {
            __syncthreads();
            if (lane_id() == 0) part[threadIdx.x / 64] = largest;
            __syncthreads();
            largest = max(max(part[0], part[1]), max(part[2], part[3]));
        }
        const float scale = quant_scale(largest);
        if (in && t == 0) a.scale[r] = scale;
        int8_t* q = a.q + r * a.ldq;
        const bool held = npieces <= PIECES * LANES;
        for (int p0 = 0; p0 < npieces; p0 += PIECES * LANES) {
#pragma unroll
            for (int i = 0; i < PIECES; ++i) {
                const int p = p0 + i * LANES + t;
                if (!in || p >= npieces) continue;
                if (!held) load_piece(row, p * 16, a.k, v[i]);
                const u32x4 w = quant_piece(v[i], scale);
                if (whole && p * 16 + 16 <= a.padded) {
                    *(u32x4*)(q + p * 16) = w;
                } else {
                    for (int e = 0; e < 16; ++e)
                        if (p * 16 + e < a.padded) q[p * 16 + e] = (int8_t)(w[e / 4] >> (8 * (e % 4)));
                }
            }
        }
        for (int b = npieces * 16 + t; in && b < a.padded; b += LANES) q[b] = 0;
    }
}

// ---- products
struct ProductArgs {
    const int8_t* a; int64_t lda; const float* a_scale;
    const int8_t* b; int64_t ldb; const float* b_scale;
    const float* bias;
    int64_t m, n; int k;
    void* out; int64_t ldo;
    // more than one part: the parts of k, the bytes of each (a multiple of 128), and their sums [parts][m][n]
    int parts, part_k; int* sums;
    // k_i8_few: floats to be quantised in the place of a; waves that share 16 rows of b
    const void* x; int64_t ldx; int share;
};

// Matrix instructions take 16 bytes of a row per lane, lane l those of row l % 16 from byte 16 (l / 16) on of a step of 64: the
// first operand's rows are the result's rows, four of them in the registers of lane l, 4 (l / 16) .. + 3, in column l % 16.  The rows
// of b come first, so that a lane holds four neighbouring outputs of a row of a.

// 4 P neighbouring outputs: the exact sums, scaled, with the bias, rounded once.  whole: all of them are there.
template <typename O, int P = 1>
__device__ __forceinline__ void store_outputs(const ProductArgs& p, int64_t row, int64_t col, const intx4* sum, float sa, const floatx4* sb, const floatx4* bias, bool whole = false)
{
    typedef O outs __attribute__((ext_vector_type(4 * P)));
    outs o;
#pragma unroll
    for (int e = 0; e < 4 * P; ++e) {
        const float v = (float)sum[e / 4][e % 4] * sa;
        o[e] = (O)(p.bias ? fmaf(v, sb[e / 4][e % 4], bias[e / 4][e % 4]) : v * sb[e / 4][e % 4]);
    }
    O* at = (O*)p.out + row * p.ldo + col;
    if (whole || col + 4 * P <= p.n) {
        __builtin_memcpy(at, &o, sizeof o);
    } else {
#pragma unroll
        for (int e = 0; e < 4 * P; ++e)
            if (col + e < p.n) at[e] = o[e];
    }
}
__device__ __forceinline__ floatx4 load_four(const float* x, int64_t col, int64_t n)
{
    floatx4 v = {0, 0, 0, 0};
    if (col + 4 <= n) {
        __builtin_memcpy(&v, x + col, 16);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (col + e < n) v[e] = x[col + e];
    }
    return v;
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

// rows of a, copied with zeros behind them
__global__ __launch_bounds__(256) void k_i8_pad(const int8_t* a, int64_t lda, int64_t m, int k, int8_t* q, int64_t ldq)
{
    const int64_t pieces = ldq / 16;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < m * pieces; i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / pieces;
        *(u32x4*)(q + i * 16) = load16(a + r * lda, (int)(i - r * pieces) * 16, k);
    }
}

// ---- rows of any alignment: tiles of 64 x 64 outputs, four waves of 32 x 32, blocks of 64 bytes of k staged through registers.  Bound by the
// wait for each block, one at a time between two barriers (us here, and with b where the other kernels can read it: 1 x 65536 x 768 14.5, 13.6,
// 777 x 10007 x 1000 46, 26.5, 4096 x 4096 x 4096 194, 63, 11 x 4096 x 8192 73, 17): for matrices that a caller cannot lay out otherwise.
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
    for (int t = 0; t < p.k; t += kStep) {
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
    for (int j = 0; j < 2; ++j) {
        const int64_t col = n0 + wn + j * 16 + lane / 16 * 4;
        const floatx4 sb = load_four(p.b_scale, col, p.n), bias = p.bias ? load_four(p.bias, col, p.n) : floatx4{};
        for (int i = 0; i < 2; ++i) {
            const int64_t row = m0 + wm + i * 16 + lane % 16;
            if (row < p.m) store_outputs<O>(p, row, col, &acc[i][j], p.a_scale[row], &sb, &bias);
        }
    }
}

// ---- many rows on both sides: tiles of BM x BN outputs, a wave's share of them WM x WN
// Blocks of 128 bytes of k of both sides go straight to LDS (no registers), into one of two buffers; rows of 64 bytes, in four smaller
// buffers, halve the lines that the first-level cache keeps of every line it asks for: 8192 x 8192 x 8192 without any multiplication
// took 356 us that way.  The fragments of a step of 64 are read while the step before is multiplied, and where those of a block's second
// step have been read by all waves its buffer is filled again: one barrier a block, two steps for its loads to land.  A wave's load
// brings 8 rows; the 16-byte pieces of row r lie at place piece ^ r % 8, so that the lanes of a read lie in different banks (a read
// of 16 bytes a lane goes in turns of 16 lanes, rows 0 .. 3 and 12 .. 15 of one piece with rows 4 .. 11 of the next).
// Where there is no more than a tile for every compute unit nothing else hides the time that loads take: NB buffers, all but one on their way.
// Rows of a are a multiple of 128 bytes long, with zeros behind k.
// A workgroup takes tiles until there are none left.  It asks for the next one's first two blocks before it writes its outputs, and
// waits for those blocks only: the outputs have two blocks' time to be written.  Scales and bias come to LDS with a tile's blocks
// (SCALES; 64 x 256 leaves no room for them beside a second workgroup).
// bytes of LDS for scales and bias
__host__ __device__ constexpr int tile_scales(int bm, int bn) { return bm == 64 ? 0 : (bm + 2 * bn) * 4; }
template <typename O, int BM, int BN, int WM, int WN, int NB = 2>
__global__ __launch_bounds__(BM / WM * (BN / WN) * 64) void k_i8_product(ProductArgs p)
{
    constexpr int WAVES = BM / WM * (BN / WN), TM = WM / 16, TN = WN / 16, BK = 128, UNITS = (BM + BN) / 8 / WAVES, BUF = (BM + BN) * BK;
    static_assert(BM / 8 % WAVES == 0 && BN / 8 % WAVES == 0);
    // Outputs of 16 bits: a lane holds eight neighbouring ones, four of each of two tiles of 16 (see row_of).
    constexpr int P = sizeof(O) == 2 ? 2 : 1;
    constexpr bool SCALES = tile_scales(BM, BN) > 0;
    extern __shared__ __align__(1024) int8_t lds[];
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int wm = wave / (BN / WN) * WM, wn = wave % (BN / WN) * WN;
    const int k_begin = blockIdx.y * p.part_k, k_end = min(p.k, k_begin + p.part_k), blocks = (k_end - k_begin + BK - 1) / BK;
    const int piece = ((lane & 7) ^ (lane >> 3)) * 16;
    const uint32_t lds0 = lds_addr(lds);

    // Tiles that run at the same time on an XCD share its L2: each has a stretch of the tiles, and takes them in blocks of
    // four rows of tiles.
    const int m = (int)p.m, n = (int)p.n, tiles_m = (m + BM - 1) / BM, tiles_n = (n + BN - 1) / BN, tiles = tiles_m * tiles_n;
    const int stretch = (tiles + 7) / 8, tile0 = (int)(blockIdx.x % 8) * stretch, end = min(stretch, tiles - tile0);
    int tile = blockIdx.x / 8, m0 = 0, n0 = 0;
    uint32_t off[UNITS];                                // (rows of a tile lie within 2^31 bytes: the host sees to it)
    const int8_t *ga = p.a, *gb = p.b;
    // The row of b that lies in row r of its part of a buffer: with pairs of tiles, rows 0 .. 15 and 16 .. 31 of 32 are four of each eight, so
    // that lanes store 16 bytes and four of them 64 that lie together (8 and 32 before: 64 queries against 1 M rows of 768 214 us, 199 now).
    auto row_of = [&](int r) __attribute__((always_inline)) { return P == 1 ? r : (r & ~31) | (r & 12) << 1 | (r & 16) >> 2 | (r & 3); };
    auto aim = [&](int t) __attribute__((always_inline)) {
        t += tile0;
        const int g = t / (4 * tiles_n), rest = t - g * 4 * tiles_n, high = min(4, tiles_m - g * 4);
        m0 = (g * 4 + rest % high) * BM;
        n0 = rest / high * BN;
        ga = p.a + (int64_t)m0 * p.lda;
        gb = p.b + (int64_t)n0 * p.ldb;
#pragma unroll
        for (int i = 0; i < UNITS; ++i) {
            const int row = (i * WAVES + wave) * 8 + lane / 8;
            off[i] = (i * WAVES * 8 < BM ? (uint32_t)min(row, m - 1 - m0) * (uint32_t)p.lda
                                         : (uint32_t)min(row_of(row - BM), n - 1 - n0) * (uint32_t)p.ldb) + piece;
        }
    };
    auto request = [&](int block) __attribute__((always_inline)) {
        // (pieces of b behind the rows' end are the row's first one of the block instead: rows of a are zeros there)
        const int k0 = k_begin + block * BK;
        const uint32_t back = k0 + piece >= k_end ? piece : 0;
#pragma unroll
        for (int i = 0; i < UNITS; ++i)
            lds_dma16((i * WAVES * 8 < BM ? ga : gb) + k0, i * WAVES * 8 < BM ? off[i] : off[i] - back, lds0 + (uint32_t)block % NB * BUF + (i * WAVES + wave) * 1024);
    };

    const int frag = (lane % 16) * BK + ((lane / 16) ^ (lane & 7)) * 16;
    intx4 acc[TM][TN], a[TM], b0[TN], b1[TN];
    auto place = [&](int block, int ks) __attribute__((always_inline)) { return lds + ((frag ^ (ks * 64)) + (uint32_t)block % NB * BUF); };
    auto read_b = [&](intx4* f, int block, int ks) __attribute__((always_inline)) {
        const int8_t* at = place(block, ks) + (BM + wn) * BK;
#pragma unroll
        for (int j = 0; j < TN; ++j) f[j] = *(const intx4*)(at + j * 16 * BK);
    };
    // one step: fragments a and b; where a fragment of a has been used for the last time the next step's takes its registers
    // (at a raised priority: the wave that shares the SIMD and is behind does its reads and requests in between; 1 .. 2 %)
    auto step = [&](const intx4* b, const int8_t* next) __attribute__((always_inline)) {
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int i = 0; i < TM; ++i) {
#pragma unroll
            for (int j = 0; j < TN; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(b[j], a[i], acc[i][j], 0, 0, 0);
            a[i] = *(const intx4*)(next + (wm + i * 16) * BK);
        }
        __builtin_amdgcn_s_setprio(0);
    };
    // Everything asked for has landed, but for `behind` blocks that were asked for last, everything read is in registers: of all waves.
    // stores: but for the TM TN / P stores of a whole tile that were enqueued behind the blocks.
    auto meet = [&](bool stores, int behind) __attribute__((always_inline)) {
        if (NB > 2 && behind >= 2) wait_vmcnt<2 * UNITS>();
        else if (NB > 2 && behind == 1) wait_vmcnt<UNITS>();
        else if (stores) wait_vmcnt<TM * TN / P>();
        else wait_vmcnt<0>();
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };

    static_assert(NB >= 2 && NB <= 4);
    float* const scales = (float*)(lds + NB * BUF);      // of BM rows a, of BN rows b, BN of the bias
    auto request_scales = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < (BM + 2 * BN) / 64; i += WAVES) {
            const int u = i + wave;                     // 64 numbers each
            if (u >= (p.bias ? BM + 2 * BN : BM + BN) / 64) continue;
            const bool of_a = u < BM / 64;
            const int at = of_a ? m0 + u * 64 : n0 + (u - BM / 64) % (BN / 64) * 64, last = (of_a ? m : n) - 1;
            const float* from = of_a ? p.a_scale : (u < (BM + BN) / 64 ? p.b_scale : p.bias);
            const int first = min(at, last);
            lds_dma4(from + first, (uint32_t)min(lane, last - first) * 4, lds0 + NB * BUF + u * 256);
        }
    };

    if (tile >= end) return;
    aim(tile);
    if (NB > 2 && SCALES && p.parts == 1) request_scales();
#pragma unroll
    for (int b = 0; b < NB; ++b)
        if (b < blocks) request(b);
    bool stores = false;
    for (;;) {
        meet(stores, min(blocks, NB) - 1);
        if (NB == 2 && SCALES && p.parts == 1) request_scales();
        read_b(b0, 0, 0);
#pragma unroll
        for (int i = 0; i < TM; ++i) a[i] = *(const intx4*)(place(0, 0) + (wm + i * 16) * BK);
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j) acc[i][j] = intx4{0, 0, 0, 0};
        for (int b = 0; b < blocks; ++b) {
            read_b(b1, b, 1);
            step(b0, place(b, 1));
            meet(stores && b == 0 && blocks > 2, min(blocks - 2 - b, NB - 2));          // (nobody reads this block's buffer any more, the next block has landed)
            if (b + NB < blocks) request(b + NB);
            read_b(b0, b + 1, 0);                       // (behind the last block: whatever the buffer holds, not multiplied)
            step(b1, place(b + 1, 0));
        }
        const int mt = m0, nt = n0;
        tile += gridDim.x / 8;
        const bool more = NB == 2 && tile < end;        // (with more buffers the host launches a workgroup for every tile)
        if (more) {
            aim(tile);
            request(0);                                 // (both buffers are free since the last meeting)
            if (blocks > 1) request(1);
        }
        stores = mt + BM <= m && nt + BN <= n;

#pragma unroll
        for (int i = 0; i < TM; ++i) {
            const int row = mt + wm + i * 16 + lane % 16;
            if (!stores && row >= m) continue;
            float sa = 0.0f;
            if (p.parts == 1) sa = SCALES ? scales[wm + i * 16 + lane % 16] : p.a_scale[row];
#pragma unroll
            for (int j = 0; j < TN; j += P) {
                const int first = wn + j * 16 + lane / 16 * 4 * P, col = nt + first;
                if (p.parts > 1) {
                    int* at = p.sums + ((int64_t)blockIdx.y * m + row) * n + col;
#pragma unroll
                    for (int e = 0; e < 4 * P; e += 4) {
                        if (stores || col + e + 4 <= n) __builtin_memcpy(at + e, &acc[i][j + e / 4], 16);
                        else
                            for (int f = 0; f < 4; ++f)
                                if (col + e + f < n) at[e + f] = acc[i][j + e / 4][f];
                    }
                    continue;
                }
                floatx4 sb[P], bias[P];
#pragma unroll
                for (int e = 0; e < P; ++e) {
                    const float* at = scales + BM + first + 4 * e;
                    sb[e] = SCALES ? *(const floatx4*)at : load_four(p.b_scale, col + 4 * e, p.n);
                    bias[e] = !p.bias ? floatx4{} : (SCALES ? *(const floatx4*)(at + BN) : load_four(p.bias, col + 4 * e, p.n));
                }
                store_outputs<O, P>(p, row, col, &acc[i][j], sa, sb, bias, stores);
            }
        }
        if (!more) break;
    }
}

// adds up the parts of k: whole numbers, in any order the same
template <typename O>
__global__ __launch_bounds__(256) void k_i8_join(ProductArgs p)
{
    const int64_t fours = (p.n + 3) / 4;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < p.m * fours; i += (int64_t)gridDim.x * 256) {
        const int64_t row = i / fours, col = i % fours * 4;
        intx4 sum = {0, 0, 0, 0};
        for (int s = 0; s < p.parts; ++s) {
            const int* at = p.sums + ((int64_t)s * p.m + row) * p.n + col;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (col + e < p.n) sum[e] += at[e];
        }
        const floatx4 sb = load_four(p.b_scale, col, p.n), bias = p.bias ? load_four(p.bias, col, p.n) : floatx4{};
        store_outputs<O>(p, row, col, &sum, p.a_scale[row], &sb, &bias);
    }
}

// ---- up to 16 rows a: bound by reading b
// The rows of a lie in LDS.  Every wave takes 16 rows of b at a time and has four blocks of 128 bytes of them on their way to a ring of
// its own in LDS (whole lines: 16 rows of 64 bytes straight to registers reached 4.8 TB/s for 1 M rows of 768, this reaches 5.7); no barrier.
// p.share waves may take parts of k of the same rows, so that few rows of b keep the chip busy too.  With floats X in the place of
// int8 each workgroup quantises a itself: one launch less, from L2.
template <typename O, typename X>
__global__ __launch_bounds__(kFewWaves * 64) void k_i8_few(ProductArgs p)
{
    constexpr int THREADS = kFewWaves * 64;
    extern __shared__ __align__(1024) int8_t lds[];      // as i8_few.h has it
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int blocks = (p.k + 127) / 128, a_stride = few_stride(p.k), m = (int)p.m;
    int8_t* const rows = lds + kRingBytes;
    float* const a_scale = (float*)(lds + few_scales(m, p.k));
    uint32_t* const largest = (uint32_t*)a_scale + kFewRows;
    const int sub = wave % p.share, first = blocks * sub / p.share, cnt = blocks * (sub + 1) / p.share - first;     // this wave's blocks of every group
    const int at_once = kFewWaves / p.share;
    const int64_t groups = (p.n + 15) / 16, stride = (int64_t)gridDim.x * at_once;
    const int64_t g0 = (int64_t)blockIdx.x * at_once + wave / p.share;
    const int rounds = (int)((groups - (int64_t)blockIdx.x * at_once + stride - 1) / stride);         // (of the workgroup: the same for all waves)

    // Where the next block comes from.  Lane l brings piece l % 8 ^ l / 8 of row l / 8 (and of row 8 + l / 8) to place l % 8 of that row.
    const int piece = ((lane & 7) ^ (lane >> 3)) * 16;
    const int8_t* from = p.b;
    uint32_t off[2];
    int64_t load_group = g0;
    int load_block = 0;
    auto aim = [&]() __attribute__((always_inline)) {
        const int64_t g = min(load_group, groups - 1);   // (requests behind the end bring the last rows again)
        const int last = (int)min((int64_t)15, p.n - 1 - g * 16);
        from = p.b + g * 16 * p.ldb;
#pragma unroll
        for (int h = 0; h < 2; ++h) off[h] = (uint32_t)min(h * 8 + lane / 8, last) * (uint32_t)p.ldb + piece;
    };
    const uint32_t ring = lds_addr(lds) + wave * kRing * 2048;
    auto request = [&](int u) __attribute__((always_inline)) {
        const int k0 = (first + load_block) * 128;
        const uint32_t back = k0 + piece >= p.k ? piece : 0;        // (behind the rows' end: multiplied by 0)
#pragma unroll
        for (int h = 0; h < 2; ++h) lds_dma16(from + k0, off[h] - back, ring + u * 2048 + h * 1024);
        if (++load_block == cnt) {
            load_block = 0;
            load_group += stride;
            aim();
        }
    };
    aim();
#pragma unroll
    for (int u = 0; u < kRing; ++u) request(u);

    const int pieces = a_stride / 16;                    // (those behind the row are zeros)
    if constexpr (sizeof(X) == 1) {
        for (int i = threadIdx.x; i < m * pieces; i += THREADS) {
            const int r = i / pieces, t = i - r * pieces;
            *(u32x4*)(rows + i * 16) = load16(p.a + r * p.lda, t * 16, p.k);
        }
        if ((int)threadIdx.x < m) a_scale[threadIdx.x] = p.a_scale[threadIdx.x];
    } else {
        // (two pieces of every thread are held between the search for the largest and the rounding, others read again)
        float held[2][16];
        if (threadIdx.x < 16) largest[threadIdx.x] = 0;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int i = h * THREADS + threadIdx.x, r = i / pieces;
            if (i < m * pieces) load_piece((const X*)p.x + r * p.ldx, (i - r * pieces) * 16, p.k, held[h]);
        }
        __syncthreads();
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int i = h * THREADS + threadIdx.x;
            if (i < m * pieces) atomicMax(&largest[i / pieces], largest_bits(held[h]));
        }
        for (int i = 2 * THREADS + threadIdx.x; i < m * pieces; i += THREADS) {
            const int r = i / pieces;
            float v[16];
            load_piece((const X*)p.x + r * p.ldx, (i - r * pieces) * 16, p.k, v);
            atomicMax(&largest[r], largest_bits(v));
        }
        __syncthreads();
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int i = h * THREADS + threadIdx.x;
            if (i < m * pieces) *(u32x4*)(rows + i * 16) = quant_piece(held[h], quant_scale(largest[i / pieces]));
        }
        for (int i = 2 * THREADS + threadIdx.x; i < m * pieces; i += THREADS) {
            const int r = i / pieces;
            float v[16];
            load_piece((const X*)p.x + r * p.ldx, (i - r * pieces) * 16, p.k, v);
            *(u32x4*)(rows + i * 16) = quant_piece(v, quant_scale(largest[r]));
        }
        if ((int)threadIdx.x < m) a_scale[threadIdx.x] = quant_scale(largest[threadIdx.x]);
    }
    if (threadIdx.x == 0) *(u32x4*)(lds + few_zeros(m, p.k)) = u32x4{0, 0, 0, 0};
    __syncthreads();
    intx4* const sums = (intx4*)(lds + few_sums(m, p.k));

    const int row = lane % 16;
    const int8_t* const fa = rows + (row < m ? row * a_stride + lane / 16 * 16 : m * a_stride);
    const int fa_step = row < m ? kStep : 0;             // (rows that a has not got are the zeros)
    const int fb = wave * kRing * 2048 + row * 128 + ((lane / 16) ^ (lane & 7)) * 16;
    int64_t group = g0;
    int block = 0;
    intx4 acc = {0, 0, 0, 0};
    for (int s0 = 0; s0 < rounds * cnt; s0 += kRing) {
#pragma unroll
        for (int u = 0; u < kRing; ++u) {
            if (s0 + u >= rounds * cnt) continue;
            wait_vmcnt<2 * (kRing - 1)>();               // (stores in between only make it longer)
            const int8_t* a = fa + (first + block) * 2 * fa_step;
            const intx4 b0 = *(const intx4*)(lds + (fb + u * 2048)), b1 = *(const intx4*)(lds + ((fb ^ 64) + u * 2048));
            acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(b0, *(const intx4*)a, acc, 0, 0, 0);
            acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(b1, *(const intx4*)(a + fa_step), acc, 0, 0, 0);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");          // the block has been read: its place may be filled again
            request(u);
            if (++block < cnt) continue;
            block = 0;
            if (p.share > 1) {
                if (sub > 0) sums[(wave - 1) * 64 + lane] = acc;
                __syncthreads();
                if (sub == 0)
                    for (int w = 1; w < p.share; ++w) acc += sums[(wave + w - 1) * 64 + lane];
                __syncthreads();
            }
            if (sub == 0 && group < groups && row < m) {
                const int64_t col = group * 16 + lane / 16 * 4;
                const floatx4 sb = load_four(p.b_scale, col, p.n), bias = p.bias ? load_four(p.bias, col, p.n) : floatx4{};
                store_outputs<O>(p, row, col, &acc, a_scale[row], &sb, &bias);
            }
            acc = intx4{0, 0, 0, 0};
            group += stride;
        }
    }
    wait_vmcnt<0>();                                     // (nothing may arrive in LDS that is no longer this workgroup's)
}

// ---- which kernel
constexpr int64_t kFewBytes = 64 * 1024;                // rows a that every workgroup quantises for itself

static hipError_t launch_quantize(int dtype, const QuantizeArgs& a, hipStream_t s)
{
    // A piece for every lane; a workgroup for a row where that is not enough (us: 262144 rows of 768 float32 197 with two pieces per
    // lane of a wave, 186 with one; 100000 rows of 100 50 with a wave a row, 17 with 16 lanes; 4096 of 8192 bfloat16 25.8 read again, 23.4 held).
    const int lanes = a.k <= 64 ? 4 : (a.k <= 256 ? 16 : (a.k <= 1024 ? 64 : 256)), rows = 256 / lanes;
    const int64_t want = (a.m + rows - 1) / rows;
    const dim3 grid((unsigned)(want < (1 << 20) ? want : 1 << 20));
    with_type(dtype, [&](auto t) {
        using T = decltype(t);
        if (lanes == 4) hipLaunchKernelGGL((k_quantize<T, 4, 1>), grid, dim3(256), 0, s, a);
        else if (lanes == 16) hipLaunchKernelGGL((k_quantize<T, 16, 1>), grid, dim3(256), 0, s, a);
        else if (lanes == 64) hipLaunchKernelGGL((k_quantize<T, 64, 1>), grid, dim3(256), 0, s, a);
        else hipLaunchKernelGGL((k_quantize<T, 256, 2>), grid, dim3(256), 0, s, a);
    });
    return hipGetLastError();
}

template <typename O, typename X>
static hipError_t launch_few(ProductArgs p, hipStream_t s)
{
    p.share = few_share(p.n, p.k);
    const int lds = few_lds((int)p.m, p.k, p.share), at_once = kFewWaves / p.share;
    const int64_t groups = (p.n + 15) / 16, want = (groups + at_once - 1) / at_once, most = (lds <= kWorkgroupLds / 2 ? 2 : 1) * kCus;
    // (the most that any launch of it takes, not this one's: the attribute is the process's, and another thread may be between setting it and its launch)
    if (hipError_t e = hipFuncSetAttribute((const void*)k_i8_few<O, X>, hipFuncAttributeMaxDynamicSharedMemorySize, kWorkgroupLds)) return e;
    hipLaunchKernelGGL((k_i8_few<O, X>), dim3((unsigned)(want < most ? want : most)), dim3(kFewWaves * 64), lds, s, p);
    return hipGetLastError();
}

// Tiles (BM rows a, BN rows b): 256 x 256 or 128 x 128, whichever takes less time, or 64 x 256 for few rows a; in parts of k where
// the tiles are few.  Large tiles come in rounds of one for every compute unit, a round taking as long as about 780 small ones, two at a
// time on a compute unit; k 4096, float32 outputs, us with large and small ones: 2048 x 6400 (200 large tiles, 800 small ones) 58,
// 72, 3500 x 3000 (168, 672) 55, 55, 4096 x 4352 (272, 1088) 110, 88, 4096 x 6144 (384, 1536) 120, 122, 4096 x 8192 (512, 2048) 135, 153.
// (The 780 are of these: with other k, what a tile costs besides its steps weighs otherwise, and where both take as long they prove nothing.)
struct Tiling { int bm, bn, parts, part_k; };
static Tiling tiling_for(int64_t m, int64_t n, int64_t k)
{
    auto tiles = [&](int bm, int bn) { return (m + bm - 1) / bm * ((n + bn - 1) / bn); };
    Tiling t{128, 128, 1, (int)k};
    if (m <= 64) t.bm = 64, t.bn = 256;
    else if (tiles(128, 128) >= (tiles(256, 256) + kCus - 1) / kCus * 780) t.bm = t.bn = 256;
    const int64_t all = tiles(t.bm, t.bn);
    if (all > 0 && all < kCus) {
        const int64_t blocks = (k + 127) / 128, parts = std::min(kCus / all, blocks / 4);        // (four blocks of k at least)
        if (parts > 1) {
            t.part_k = (int)((blocks + parts - 1) / parts * 128);
            t.parts = (int)((k + t.part_k - 1) / t.part_k);
        }
    }
    return t;
}
static size_t sums_bytes(int64_t m, int64_t n, int64_t k)
{
    const Tiling t = tiling_for(m, n, k);
    return t.parts > 1 ? (size_t)t.parts * m * n * 4 : 0;
}

template <typename O>
static hipError_t launch_tiles(const Tiling& t, ProductArgs p, hipStream_t s)
{
    hipError_t e = hipSuccess;
    const int64_t tiles = (p.m + t.bm - 1) / t.bm * ((p.n + t.bn - 1) / t.bn);
    const bool deep = t.bm < 256 && tiles * t.parts <= kCus;
    auto go = [&](auto kernel, int waves, int buffers) {
        const size_t lds = (size_t)(t.bm + t.bn) * 128 * buffers + tile_scales(t.bm, t.bn);
        if (lds > kStaticLds) e = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (e == hipSuccess) hipLaunchKernelGGL(kernel, dim3((unsigned)(std::min((tiles + 7) / 8, (int64_t)kCus / 8 * (lds <= 80 * 1024 ? 2 : 1)) * 8), t.parts), dim3(waves * 64), lds, s, p);
    };
    p.parts = t.parts;
    p.part_k = t.part_k;
    if (t.bm == 256) go(k_i8_product<O, 256, 256, 128, 64>, 8, 2);
    else if (t.bm == 128) deep ? go(k_i8_product<O, 128, 128, 64, 32, 4>, 8, 4) : go(k_i8_product<O, 128, 128, 64, 32>, 8, 2);
    else deep ? go(k_i8_product<O, 64, 256, 64, 32, 3>, 8, 3) : go(k_i8_product<O, 64, 256, 64, 32>, 8, 2);
    if (e == hipSuccess && t.parts > 1) {
        const int64_t want = (p.m * ((p.n + 3) / 4) + 255) / 256;
        hipLaunchKernelGGL(k_i8_join<O>, dim3((unsigned)(want < (1 << 20) ? want : 1 << 20)), dim3(256), 0, s, p);
    }
    return e == hipSuccess ? hipGetLastError() : e;
}

// rows that requests of 16 bytes reach; offsets inside a tile are 32-bit numbers
static bool in_tiles(const void* p, int64_t ld) { return (uintptr_t)p % 16 == 0 && ld % 16 == 0 && ld < (1 << 22); }

static int64_t padded_k(int64_t k) { return (k + 127) / 128 * 128; }

// padded: room for the rows of a at multiples of 128 bytes (or those rows themselves)
static hipError_t launch_product(int dtype, const ProductArgs& p, int8_t* padded, hipStream_t s)
{
    return with_type(dtype, [&](auto o) -> hipError_t {
        using O = decltype(o);
        if (few_rows(p.m, p.n, p.k) && in_tiles(p.b, p.ldb)) return launch_few<O, int8_t>(p, s);
        if (in_tiles(p.b, p.ldb)) {
            ProductArgs t = p;
            if (p.k % 128 || !in_tiles(p.a, p.lda)) {
                t.a = padded;
                t.lda = padded_k(p.k);
                if (t.a != p.a) {
                    const int64_t want = (p.m * (t.lda / 16) + 255) / 256;
                    hipLaunchKernelGGL(k_i8_pad, dim3((unsigned)(want < (1 << 20) ? want : 1 << 20)), dim3(256), 0, s, p.a, p.lda, p.m, p.k, padded, t.lda);
                }
            }
            return launch_tiles<O>(tiling_for(p.m, p.n, p.k), t, s);
        }
        hipLaunchKernelGGL(k_i8_product_any<O>, dim3((unsigned)((p.m + 63) / 64 * ((p.n + 63) / 64))), dim3(256), 0, s, p);
        return hipGetLastError();
    });
}

}  // namespace hr

// ---- C entry points
using namespace hr;

static int check_shape(int64_t m, int64_t n, int64_t k)
{
    if (m < 0 || m > (1 << 24)) return fail(HR_ERR_ARG, "m=%lld out of range", (long long)m);
    if (n < 0 || n > (1LL << 31) - 1) return fail(HR_ERR_ARG, "n=%lld out of range", (long long)n);
    if (k < 1 || k > HR_I8_K_MAX) return fail(HR_ERR_ARG, "k=%lld must be in 1..%d", (long long)k, HR_I8_K_MAX);
    // (tiles of 64 x 64 outputs, and a launch may not have 2^32 threads; numbers of rows and tiles fit 32 bits)
    if (n > (1LL << 30) || (m + 63) / 64 * ((n + 63) / 64) >= (1LL << 24)) return fail(HR_ERR_UNSUPPORTED, "m=%lld x n=%lld: more outputs than one call takes", (long long)m, (long long)n);
    return HR_OK;
}

// workspace: rows a as the tiles want them (quantised ones, or copied ones), their scales, sums of the parts of k
static size_t rows_bytes(int64_t m, int64_t k) { return aligned((size_t)(m * padded_k(k))); }
static size_t scales_bytes(int64_t m) { return aligned((size_t)m * 4); }

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
    QuantizeArgs a{x, ldx, m, (int)k, q, ldq, scale, (int)std::min((k + 63) / 64 * 64, ldq)};
    HR_HIP(launch_quantize(dtype, a, (hipStream_t)stream));
    return HR_OK;
}

size_t hr_i8_workspace_bytes(int64_t m, int64_t n, int64_t k)
{
    if (check_shape(m, n, k)) return 0;
    // (fewer rows may be cut in more parts; the most sums of rows in as many tiles are those of whole tiles.  Rows beyond 128 x 256 tiles
    // are never cut)
    size_t sums = sums_bytes(m, n, k);
    for (int64_t rows = std::min(m - 1, (int64_t)128 * kCus) / 128 * 128; rows > 0; rows -= 128) sums = std::max(sums, sums_bytes(rows, n, k));
    if (m > 64) sums = std::max(sums, sums_bytes(64, n, k));
    return rows_bytes(m, k) + scales_bytes(m) + aligned(sums) + HR_WORKSPACE_ALIGN;
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
    p.sums = (int*)((char*)workspace + rows_bytes(m, k) + scales_bytes(m));
    HR_HIP(launch_product(out_dtype, p, (int8_t*)workspace, (hipStream_t)stream));
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
    float* scale = (float*)(q + rows_bytes(m, k));
    if (few_rows(m, n, k) && in_tiles(b, ldb) && m * k * (int64_t)element_bytes(x_dtype) <= kFewBytes) {
        ProductArgs p{nullptr, 0, nullptr, b, ldb, b_scale, bias, m, n, (int)k, out, ldo};
        p.x = x;
        p.ldx = ldx;
        HR_HIP(with_type(out_dtype, [&](auto o) { return with_type(x_dtype, [&](auto e) { return launch_few<decltype(o), decltype(e)>(p, (hipStream_t)stream); }); }));
        return HR_OK;
    }
    QuantizeArgs qa{x, ldx, m, (int)k, q, padded_k(k), scale, (int)padded_k(k)};
    HR_HIP(launch_quantize(x_dtype, qa, (hipStream_t)stream));
    ProductArgs p{q, padded_k(k), scale, b, ldb, b_scale, bias, m, n, (int)k, out, ldo};
    p.sums = (int*)((char*)scale + scales_bytes(m));
    HR_HIP(launch_product(out_dtype, p, q, (hipStream_t)stream));
    return HR_OK;
}

}  // extern "C"
