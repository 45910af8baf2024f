// A block's tile of a row-grouped product, from the experts' offsets alone: for launches that are too short to wait for a
// kernel that makes a list of them first.
#pragma once

#include "common.h"

namespace moe {

// Tiles of BM rows by one of `tiles` columns: an expert's row by row inside a column, experts one after the other, an eighth of
// all for each XCD (the blocks go round the eight).  A grid of block_tile_grid() holds all of them; false: no tile is left for
// this block.  Every lane of the wavefront calls it.
template <int BM>
__device__ __forceinline__ bool block_tile(const int32_t *__restrict__ offsets, int E, int tiles, int block, int &expert,
                                           int &row0, int &row1, int &column)
{
    const int lane = lane_id();
    const int e = min(lane, E - 1), first = offsets[e], end = lane < E ? offsets[e + 1] : first;
    const int mt = end > first ? (end - first + BM - 1) / BM : 0;
    int sum = mt * tiles;
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) {
        const int v = __shfl_up(sum, d);
        if (lane >= d) sum += v;
    }
    const int total = __builtin_amdgcn_readlane(sum, kWave - 1), per_xcd = (total + 7) / 8;
    const int slot = block / 8, index = block % 8 * per_xcd + slot;
    if (slot >= per_xcd || index >= total) return false;
    expert = __builtin_amdgcn_readfirstlane(__popcll(__ballot(sum <= index)));
    const int row_tiles = __builtin_amdgcn_readlane(mt, expert);
    const int within = index - (__builtin_amdgcn_readlane(sum, expert) - row_tiles * tiles);
    row0 = __builtin_amdgcn_readlane(first, expert) + within % row_tiles * BM;
    row1 = min(row0 + BM, __builtin_amdgcn_readlane(end, expert));
    column = within / row_tiles;
    return true;
}
inline unsigned block_tile_grid(int64_t rows, int E, int bm, int tiles)
{
    return static_cast<unsigned>(align_up((static_cast<size_t>(rows) / bm + (rows < E ? rows : E)) * tiles, 8));
}

}  // namespace moe
