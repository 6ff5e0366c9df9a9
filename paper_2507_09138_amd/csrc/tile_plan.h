// Which tiles the products of gated blocks take, and in how many parts of k (host arithmetic).
#pragma once
#include <algorithm>

#include "entry.h"
#include "tile.h"

namespace hr {

constexpr int64_t kMostParts = 64, kMostSums = 1 << 28;              // of k, and bytes of their sums

// Blocks of k that a place for a workgroup multiplies one after the other until all workgroups are done: first those of `long_` blocks, then the
// shorter ones, each on the first of `places` that is free.
inline double rounds(int64_t places, int64_t longs, int64_t long_, int64_t shorts, int64_t short_)
{
    const int64_t later = longs % places;                // places that take one of the long ones more
    int64_t early_free = longs / places * long_, late_free = early_free + long_, last = later ? late_free : early_free;
    while (shorts > 0) {
        const bool early = later == 0 || early_free <= late_free;
        shorts -= early ? places - later : later;
        int64_t& free = early ? early_free : late_free;
        free += short_;
        last = std::max(last, free);
    }
    return (double)last;
}

// Tiles (rows x columns of both matrices): 256 x 256, 128 x 128 or, for up to 64 rows of a gated block, 64 x 256, in parts of k or not: what takes
// least by this count of microseconds.  A compute unit takes one workgroup with a large tile at a time, two with small ones; a block of 128 bytes of k
// takes a large tile 1.6 (16 bits), two small ones 0.96, and one alone, where up to 256 are left or there are no more, 0.5; in float32 3.8 and 2.0
// (large tiles are no faster there).  Start and end take 6 to 8, parts are written and read at 4 MB/us, by another launch.  Parts of two products in one
// launch are about as long as each other.
// Measured, here (the other choices): 4096 x 4096 x 4096 bfloat16 102 .. 112 (128 x 128 118), 2048 x 4096 x 4096 61 (256 x 256 86, two parts 84),
// 512 x 512 x 4096 in eight parts 15.4 (one 32.6), float32 2048 x 768 x 4096 in five 113 (one 260, two 148), that and 4096 x 768 x 2048 in one launch
// 219 (one after the other 228; in six parts and one, unlike lengths, 325).
// Where large tiles leave much of a last round empty, the rows of that round are left to small ones, in a second launch: 8192 x 4096 x 21504 and
// 21504 x 4096 x 8192, 2 and 5.25 rounds, 2283 -> 2150.
// m, n and k of the products are there; parts, part_k and large are set.
inline Tiling plan_tiles(bool gated, size_t es, TileArgs* p, int count)
{
    const double pair = es == 4 ? 3.8 : 0.96, one = es == 4 ? 2.0 : 0.5;             // of small tiles
    Tiling best{};
    double least = 0;
    const int64_t rows[2] = {p[0].m, count > 1 ? p[1].m : 0};
    int64_t longest_k = 0, chosen = 0, large[2] = {};    // of the best so far: blocks of its longest part, rows in large tiles
    for (int i = 0; i < count; ++i) longest_k = std::max<int64_t>(longest_k, p[i].k / 128);
    // small tiles of so many blocks each: rounds of two on every compute unit, the last one half as long where it has one at most for each
    auto small = [&](int64_t tiles, int64_t of) {
        const int64_t at_once = 2 * kComputeUnits, left = tiles % at_once;
        return (double)(tiles / at_once * of) * pair + (left == 0 ? 0 : left <= kComputeUnits ? of * one : of * pair);
    };
    auto consider = [&](int bm, int bn) {
        const int64_t cols = bn / (gated ? 2 : 1);
        int64_t last = 0;
        for (int64_t n = 1; n <= kMostParts; ++n) {
            const int64_t length = (longest_k + n - 1) / n;                  // blocks of the longest part
            if (n > 1 && (length < 2 || length == last)) continue;
            last = length;
            int64_t groups[2] = {0, 0}, of[2] = {0, 0};
            double work = 0, joins = 0;
            bool fits = true;
            for (int i = 0; i < count; ++i) {
                const int64_t blocks = p[i].k / 128, parts = (blocks + length - 1) / length;
                const double sums = (double)parts * p[i].m * p[i].n * (gated ? 8 : 4);
                of[i] = (blocks + parts - 1) / parts;
                groups[i] = (p[i].m + bm - 1) / bm * ((p[i].n + cols - 1) / cols) * parts;
                work += (double)groups[i] * of[i];
                if (parts > 1) {
                    joins += 2 * sums / 4e6;
                    fits &= groups[i] <= 8 * kComputeUnits && sums <= kMostSums;
                }
            }
            if (!fits) break;
            if (joins > 0) joins += 4;
            const int l = of[1] > of[0];                 // the product of the longer parts
            const int64_t all = groups[0] + groups[1];
            auto try_one = [&](double t, const int64_t* in_large) {
                if (!best.bm || t < least) {
                    least = t;
                    best = {bm, bn};
                    chosen = length;
                    std::copy_n(in_large, 2, large);
                }
            };
            if (bm < 256) {
                if (all <= kComputeUnits) try_one(std::max(of[0], of[1]) * one + 6 + joins, rows);
                else if (count > 1 && of[0] != of[1]) try_one(rounds(2 * kComputeUnits, groups[l], of[l], groups[1 - l], of[1 - l]) * pair + 6 + joins, rows);
                else try_one(small(all, of[0]) + 6 + joins, rows);
                continue;
            }
            double t = rounds(kComputeUnits, groups[l], of[l], groups[1 - l], of[1 - l]) * 1.6;
            t = std::max(std::max(of[0], of[1]) * 1.2, (t + work / kComputeUnits * 1.6) / 2) + 8 + joins;
            if (n == 1) {                                // rows that fill whole rounds, the others in small tiles
                double mixed = 14;
                int64_t kept[2] = {0, 0};
                for (int i = 0; i < count; ++i) {
                    const int64_t across = (p[i].n + cols - 1) / cols, down = (p[i].m + bm - 1) / bm, full = across * down / kComputeUnits * kComputeUnits / across,
                                  left = p[i].m - full * bm;
                    kept[i] = left > 0 ? full * bm : p[i].m;
                    mixed += (double)((std::min(full, down) * across + kComputeUnits - 1) / kComputeUnits * of[i]) * 1.6;
                    if (left > 0) mixed += small((left + 127) / 128 * ((p[i].n + cols / 2 - 1) / (cols / 2)), of[i]);
                }
                try_one(mixed, kept);
            }
            try_one(t, rows);
        }
    };
    if (gated && p[0].m <= 64) {
        consider(64, 256);
    } else {
        consider(128, 128);
        if (es < 4) consider(256, 256);
    }
    for (int i = 0; i < count; ++i) {
        const int64_t blocks = p[i].k / 128, parts = (blocks + chosen - 1) / chosen, of = (blocks + parts - 1) / parts;
        p[i].parts = (int)((blocks + of - 1) / of);
        p[i].part_k = (int)of * 128;
        p[i].large = large[i];
    }
    return best;
}
// room for the sums of parts of k
inline size_t sums_bytes(bool gated, const TileArgs& p) { return p.parts > 1 ? aligned((size_t)(p.parts * p.m * p.n * (gated ? 2 : 1)) * 4) : 0; }

inline int64_t padded(int64_t n, size_t es) { return (n * (int64_t)es + 127) / 128 * 128; }             // bytes of a row

// Waves that take parts of k of the same columns: enough for the chip to be busy (4 a SIMD), eight steps of 64 bytes each at least.  us, against up to 1024 waves:
// 1 x 4096 x 10752 bfloat16 36 (43), 4 x 4097 x 1024 14.9 (16.1); with 8192 the same.  At least 16 steps: 16 x 768 x 2048 binary16 4.4 (6.0).
inline int few_share(int64_t groups, int64_t k_bytes, int most)
{
    int share = 1;
    while (share < most && groups * share < 4096 && k_bytes / 64 >= 16 * share) share *= 2;
    return share;
}

}  // namespace hr
