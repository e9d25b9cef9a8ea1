// block_units.hpp -- attention over the uniform cache: the tiles of 32 positions that rows see, and how the work of many rows is
// counted.  For device and host.
#pragma once

#include <hip/hip_runtime.h>

#include "internal.hpp"

namespace dkv {

constexpr int kBT = 32;         // positions per block, and of a tile
constexpr int kTileRows = 128;  // rows of a workgroup of the many-row kernel
constexpr int kTileStart = 4;   // a 128-row block's start, in tiles

// The tiles that a sequence's new tokens see, in order: [0, sb) and [w0, last].
struct Tiles {
    int sb, w0, last;
    __host__ __device__ __forceinline__ int count() const { return sb + last + 1 - w0; }
    __host__ __device__ __forceinline__ int at(int step) const { return step < sb ? step : w0 + step - sb; }
};
__host__ __device__ __forceinline__ Tiles tiles_of(const BlockAttnArgs& a, int n, int L)
{
    Tiles t;
    t.last = (L + n - 1) / kBT;
    const int sb = a.sinks / kBT + (a.sinks % kBT != 0);
    t.sb = min(sb, t.last + 1);
    t.w0 = max(t.sb, max(0, L + 1 - a.window) / kBT);
    return t;
}

// Units of a sequence's 128-row blocks up to block t: each counts about as many as it has tiles.  They grow with the rows'
// positions, a tile for 32, until the window has left the tiles of the first tokens behind; up to there a sum along a line in closed
// form stands for them, from there on each has as many.
struct TileUnits {
    int blocks, full;        // 128-row blocks; from `full` on all have as many tiles
    long long first, most;   // units of block 0, of those from `full` on
    __host__ __device__ __forceinline__ long long upto(long long t) const
    {
        // (up to 2^23 tokens of up to 64 heads: g <= 2^22, and most - first <= 2^18, so the product is below 2^62)
        const long long g = t < full ? t : full;
        return first * g + (most - first) * g * (g - 1) / (2 * (long long)max(full, 1)) + most * (t - g);
    }
};
__host__ __device__ __forceinline__ TileUnits tile_units(const BlockAttnArgs& a, int n, int L)
{
    TileUnits u;
    u.blocks = (n * a.G + kTileRows - 1) / kTileRows;
    const int step = (kTileRows + a.G - 1) / a.G;  // tokens of a block, about
    u.first = tiles_of(a, min(n, step), L).count() + kTileStart;
    const int last = max(0, n - step);
    const long long end = (long long)a.window + (long long)(a.sinks / kBT + (a.sinks % kBT != 0)) * kBT;  // the line's
    const int late = end < L + last ? (int)max(0LL, min((long long)last, end - L)) : last;
    u.full = late / step;
    u.most = max((long long)tiles_of(a, min(n - late, step), L + late).count() + kTileStart, u.first);
    return u;
}

}  // namespace dkv
