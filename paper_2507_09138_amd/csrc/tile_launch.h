// Launches of k_tiles for one type of elements: the body of gated_f16.hip, gated_bf16.hip and gated_f32.hip.
#pragma once
#include <algorithm>

#include "tile.h"

namespace hr {

template <typename T, bool GATED>
hipError_t launch_tiles(const Tiling& t, TileArgs p, hipStream_t s)
{
    hipError_t e = hipSuccess;
    const int64_t cols = GATED ? t.bn / 2 : t.bn, tiles = (p.m + t.bm - 1) / t.bm * ((p.n + cols - 1) / cols);
    const bool deep = t.bm < 256 && tiles * t.parts <= kComputeUnits;
    auto go = [&](auto kernel, int buffers) {
        const size_t lds = (size_t)(t.bm + t.bn) * 128 * buffers;
        if (lds > 64 * 1024) e = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (e == hipSuccess) hipLaunchKernelGGL(kernel, dim3((unsigned)(std::min((tiles + 7) / 8, (int64_t)kComputeUnits / 8 * (lds <= 80 * 1024 ? 2 : 1)) * 8), t.parts), dim3(512), lds, s, p);
    };
    p.parts = t.parts;
    p.part_k = t.part_k;
    if (t.bm == 256) go(k_tiles<T, GATED, 256, 256, 128, 2>, 2);
    else if (t.bm == 128) deep ? go(k_tiles<T, GATED, 128, 128, 32, 4>, 4) : go(k_tiles<T, GATED, 128, 128, 32, 2>, 2);
    else deep ? go(k_tiles<T, GATED, 64, 256, 32, 3>, 3) : go(k_tiles<T, GATED, 64, 256, 32, 2>, 2);
    if (e == hipSuccess && t.parts > 1) {
        auto join = [&](auto kernel, int shares) {
            const int64_t want = (p.m * ((p.n + 3) / 4) + 256 / shares - 1) / (256 / shares);
            hipLaunchKernelGGL(kernel, dim3((unsigned)std::min<int64_t>(want, 1 << 20)), dim3(256), 0, s, p);
        };
        if (t.parts >= 12) join(k_tiles_join<T, GATED, 16>, 16);
        else if (t.parts >= 4) join(k_tiles_join<T, GATED, 4>, 4);
        else join(k_tiles_join<T, GATED, 1>, 1);
    }
    return e == hipSuccess ? hipGetLastError() : e;
}

}  // namespace hr
