// Products of few rows a (k_i8_few): how a workgroup's LDS is laid out, and which shapes fit it.  Plain arithmetic of the host and of the kernel.
#pragma once
#include "common.h"

namespace hr {

constexpr int kCus = 256;
constexpr int kWorkgroupLds = 160 * 1024;                // most LDS of a workgroup on gfx950
constexpr int kFewRows = 16, kFewWaves = 8, kRing = 4, kRingBytes = kFewWaves * kRing * 2048;
constexpr int kFewLds = 90 * 1024;                       // most bytes of a
// bytes between the rows of a in LDS: 16 rows in different banks, nothing behind a row that is not zero
__host__ __device__ constexpr int few_stride(int k) { return (k + 127) / 128 * 128 + 16; }

// Where the parts begin: rings of kRingBytes, m rows of a, 16 zeros, the scales of the rows of a and their largest magnitudes, and sums of
// all waves but one where several share rows of b.  The kernel has no LDS besides.
__host__ __device__ constexpr int few_zeros(int m, int k) { return kRingBytes + m * few_stride(k); }
__host__ __device__ constexpr int few_scales(int m, int k) { return few_zeros(m, k) + 16; }
__host__ __device__ constexpr int few_sums(int m, int k) { return few_scales(m, k) + 2 * kFewRows * 4; }
constexpr int few_lds(int m, int k, int share) { return few_sums(m, k) + (share > 1 ? (kFewWaves - 1) * 1024 : 0); }

// waves that take parts of k of the same 16 rows of b: enough for the chip to be busy, four blocks of 128 bytes of k each at least
constexpr int few_share(int64_t n, int k)
{
    const int blocks = (k + 127) / 128;
    const int64_t groups = (n + 15) / 16;
    int share = 1;
    while (share < kFewWaves && groups * share < 2 * kFewWaves * kCus && blocks >= 4 * share) share *= 2;
    return share;
}

// Whether k_i8_few takes this product: what it needs of LDS is there.  Longer rows are work for tiles, which take as long there (us against 4096 rows b:
// 16 rows of 5504 here 13.3, of 5632 in tiles 13.0; 11 of 8064 16.1, of 8192 16.8).
constexpr bool few_rows(int64_t m, int64_t n, int64_t k)
{
    return m <= kFewRows && m * few_stride((int)k) <= kFewLds && few_lds((int)m, (int)k, few_share(n, (int)k)) <= kWorkgroupLds;
}

}  // namespace hr
