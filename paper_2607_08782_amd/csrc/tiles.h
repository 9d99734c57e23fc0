// Pieces that the tiled grouped products share: direct loads into LDS, ragged groups as
// lists of tiles, tiles in an order that keeps operands in an XCD's L2.
#pragma once

#include "common.h"

namespace moe {
namespace {

constexpr int NUM_XCD = 8;
constexpr uint32_t RSRC_WORD3 = 0x00020000;        // raw buffer: 32-bit data format
constexpr int A_OOB = 0x7fffff00;                  // offset past any descriptor: reads zero

typedef __attribute__((address_space(3))) void lds_void;

// wait until at most N of this wave's vector-memory operations are outstanding
// (they complete in issue order); no memory access moves across it
template <int N>
__device__ __forceinline__ void wait_vm() {
    static_assert(N >= 0 && N < 64, "vmcnt range");
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

// First row of group g.  The first `lead` groups hold lead_rows rows each (the
// shared experts' groups of moe_grouped_ffn_rows_shared, every token once); the
// offsets array gives the row ranges of the groups after them, counted from
// row lead * lead_rows, as moe_permute writes them.
__device__ __forceinline__ int group_start(const int32_t* offsets, int lead, int lead_rows, int g) {
    return g < lead ? g * lead_rows : lead * lead_rows + offsets[g - lead];
}

// s_tstart[g] = tiles of the groups before g, for g = 0..n_groups (a group of
// more than small_rows rows has ceil(rows / BM) * n_tiles tiles, others none);
// run by one whole wave.
template <int BM>
__device__ __forceinline__ void tile_starts(const int* s_off, int n_groups, int small_rows,
                                            int n_tiles, int* s_tstart, int lane) {
    int carry = 0;
    for (int g0 = 0; g0 < n_groups; g0 += 64) {
        const int g = g0 + lane;
        const int rows = g < n_groups ? s_off[g + 1] - s_off[g] : 0;
        const int v = rows > small_rows ? (int)ceil_div(rows, BM) * n_tiles : 0;
        const int incl = wave_incl_scan(v);
        if (g < n_groups) s_tstart[g + 1] = carry + incl;
        carry += __shfl(incl, 63, 64);
    }
    if (lane == 0) s_tstart[0] = 0;
}

// Tile `local` of a group of mt x n_tiles tiles: the row tiles in blocks of at most
// 8 (of equal size, give or take one), each block running through all column tiles,
// rows first.  The 32 tiles an XCD works on at once then span about 8 row and 4
// column slabs of operands, whatever the group's height (rows first over a whole
// group of 32 row tiles, they span 32 + 1: an 8192-row expert's gate/up product at
// d = f = 2048 x 2816 fetched twice the bytes).
struct TilePos {
    int m, n;
};

__device__ __forceinline__ TilePos tile_pos(int local, int mt, int n_tiles) {
    const int nb = (mt + 7) >> 3;
    const int base = mt / nb, extra = mt - base * nb;      // the first `extra` blocks have one more
    const int big = extra * (base + 1) * n_tiles;
    TilePos p;
    if (local < big) {
        const int b = local / ((base + 1) * n_tiles), l = local - b * (base + 1) * n_tiles;
        p.n = l / (base + 1);
        p.m = b * (base + 1) + l - p.n * (base + 1);
    } else {
        const int l0 = local - big, b = l0 / (base * n_tiles), l = l0 - b * base * n_tiles;
        p.n = l / base;
        p.m = extra * (base + 1) + b * base + l - p.n * base;
    }
    return p;
}

}  // namespace
}  // namespace moe
