// Launches of k_tiles for one type of elements: the body of gated_f16.hip, gated_bf16.hip and gated_f32.hip.
#pragma once
#include <algorithm>
#include <type_traits>
#include <utility>

#include "tile.h"

namespace hr {

template <typename T, bool GATED>
static hipError_t launch_one_size(const Tiling& t, TilePair pair, int count, hipStream_t s)
{
    hipError_t e = hipSuccess;
    const int64_t cols = GATED ? t.bn / 2 : t.bn;
    auto tiles = [&](const TileArgs& p) { return (p.m + t.bm - 1) / t.bm * ((p.n + cols - 1) / cols); };
    int64_t all = 0;
    for (int i = 0; i < count; ++i) all += tiles(pair.p[i]) * pair.p[i].parts;
    const bool deep = all <= kComputeUnits;              // (nothing but requests of its own hides the time that a workgroup's loads take)
    if (count > 1 && pair.p[1].part_k > pair.p[0].part_k) std::swap(pair.p[0], pair.p[1]);               // (long parts first)
    auto go = [&](auto kernel, int buffers) {
        const size_t lds = (size_t)(t.bm + t.bn) * 128 * buffers;
        unsigned groups[2] = {0, 0};
        for (int i = 0; i < count; ++i) {
            // (where there are more than two buffers every part of a tile has a workgroup of its own)
            const int64_t of_eight = (tiles(pair.p[i]) * pair.p[i].parts + 7) / 8;
            pair.p[i].slots = (int)(buffers > 2 ? of_eight : std::min(of_eight, (int64_t)kComputeUnits / 8 * (lds <= 80 * 1024 ? 2 : 1))) * 8;
            groups[i] = (unsigned)pair.p[i].slots;
        }
        pair.first = groups[0];
        if (lds > 64 * 1024) e = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (e == hipSuccess) hipLaunchKernelGGL(kernel, dim3(groups[0] + groups[1]), dim3(512), lds, s, pair);
    };
    auto of_size = [&](auto tail) {
        constexpr bool TAIL = decltype(tail)::value;
        if (t.bm == 256) {
            if constexpr (sizeof(T) == 2) go(k_tiles<T, GATED, 256, 256, 128, 2, TAIL>, 2);
        } else if (t.bm == 128) {
            deep ? go(k_tiles<T, GATED, 128, 128, 32, 4, TAIL>, 4) : go(k_tiles<T, GATED, 128, 128, 32, 2, TAIL>, 2);
        } else if constexpr (GATED) {
            deep ? go(k_tiles<T, GATED, 64, 256, 32, 3, TAIL>, 3) : go(k_tiles<T, GATED, 64, 256, 32, 2, TAIL>, 2);
        }
    };
    if constexpr (GATED) {                               // (operands of the gradients are laid out in whole blocks)
        pair.p[0].end < pair.p[0].k ? of_size(std::true_type{}) : of_size(std::false_type{});
    } else {
        of_size(std::false_type{});
    }
    const int most = std::max(pair.p[0].parts, count > 1 ? pair.p[1].parts : 1);
    if (e == hipSuccess && most > 1) {
        auto join = [&](auto kernel, int shares) {
            unsigned groups[2] = {0, 0};
            for (int i = 0; i < count; ++i)
                if (pair.p[i].parts > 1) groups[i] = (unsigned)std::min<int64_t>((pair.p[i].m * ((pair.p[i].n + 3) / 4) + 256 / shares - 1) / (256 / shares), 1 << 20);
            pair.first = groups[0];
            hipLaunchKernelGGL(kernel, dim3(groups[0] + groups[1]), dim3(256), 0, s, pair);
        };
        if (most >= 12) join(k_tiles_join<T, GATED, 16>, 16);
        else if (most >= 4) join(k_tiles_join<T, GATED, 4>, 4);
        else join(k_tiles_join<T, GATED, 1>, 1);
    }
    return e == hipSuccess ? hipGetLastError() : e;
}

template <typename T, bool GATED>
hipError_t launch_tiles(const Tiling& t, const TilePair& pair, int count, hipStream_t s)
{
    TilePair first{}, rest{};
    int firsts = 0, rests = 0;
    for (int i = 0; i < count; ++i) {
        const TileArgs& p = pair.p[i];
        if (p.large > 0) {
            first.p[firsts] = p;
            first.p[firsts++].m = p.large;
        }
        if (p.large < p.m) {
            TileArgs& r = rest.p[rests++] = p;
            r.row0 = p.large;
            r.a += p.large * p.lda;
            r.m -= p.large;
        }
    }
    if (firsts)
        if (hipError_t e = launch_one_size<T, GATED>(t, first, firsts, s)) return e;
    return rests ? launch_one_size<T, GATED>(Tiling{128, 128}, rest, rests, s) : hipSuccess;
}

}  // namespace hr
