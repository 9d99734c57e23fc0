// Pieces that the grouped products of quantized operands share: groups of few rows as weight
// strips, groups of many as a workgroup's list of tiles.
#pragma once

#include "tiles.h"

namespace moe {
namespace {

// First row of group g of a product's arguments.
template <typename Args>
__device__ __forceinline__ int first_row(const Args& p, int g) {
    return group_start(p.offsets, p.lead, p.lead_rows, g);
}

// The n-th group that holds rows, its first row and their number (a call of fewer rows than
// groups launches strips for as many groups as it has rows: a single token's step over 64
// experts of which it takes 6 starts 264 workgroups, not 2816).
struct Group {
    int g, row0, rows;
};

template <typename Args>
__device__ __forceinline__ Group nth_group(const Args& p, int n) {
    const int lane = threadIdx.x & 63;
    for (int g0 = 0; g0 < p.n_groups; g0 += 64) {
        const int g = min(g0 + lane, p.n_groups - 1);
        const int row0 = first_row(p, g), rows = first_row(p, g + 1) - row0;
        uint64_t mask = __ballot(g0 + lane < p.n_groups && rows > 0);
        const int here = __popcll(mask);
        if (n < here) {
            for (; n > 0; --n) mask &= mask - 1;
            const int l = __builtin_ctzll(mask);
            return {g0 + l, __builtin_amdgcn_readlane(row0, l), __builtin_amdgcn_readlane(rows, l)};
        }
        n -= here;
    }
    return {0, 0, 0};
}

__device__ __forceinline__ uint64_t uniform(uint64_t v) {
    return (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(v >> 32)) << 32 |
           (uint32_t)__builtin_amdgcn_readfirstlane((int)v);
}

// weight row, within its 32-row block, of LDS row r: the instruction's row 8 a + 4 h + b is
// accumulator 4 a + b of half h of the wave, which holds columns 16 h + 0 .. 15
__device__ __forceinline__ int w_order(int r) {
    return (r & ~31) + 16 * ((r >> 2) & 1) + 4 * ((r >> 3) & 3) + (r & 3);
}

// Tiles of 256 rows come in two kinds: high ones, and those of at most half the rows (a
// group's last), whose upper waves have nothing to multiply.  These come last, where a round
// is partly filled (4096 Mixtral-shaped tokens, 5.7 rounds of the one and 0.4 of the other:
// gate/up 220 us in 7 rounds, 206 so).  The smaller tiles stay in order: a group's tiles apart
// read its weights twice (1024 tokens of DeepSeek-V2-Lite 106 and 112 us).
template <int BM>
__device__ __forceinline__ int high_tiles(int rows) {
    return BM > 128 ? (rows + BM / 2 - 1) / BM : (int)ceil_div(rows, BM);
}

// start[g] = tiles of the groups before g, by count(rows) row tiles each; by one wave
template <typename Count>
__device__ __forceinline__ void starts(const int* s_off, int n_groups, int n_tiles, int* start, int lane,
                                       Count count) {
    int carry = 0;
    for (int g0 = 0; g0 < n_groups; g0 += 64) {
        const int g = g0 + lane;
        const int incl = wave_incl_scan(g < n_groups ? count(s_off[g + 1] - s_off[g]) * n_tiles : 0);
        if (g < n_groups) start[g + 1] = carry + incl;
        carry += __shfl(incl, 63, 64);
    }
    if (lane == 0) start[0] = 0;
}

constexpr int TILE_LIST = 32;                            // tile records kept, in two halves

// A workgroup's tiles of a product over ragged groups, of BM rows x one of n_tiles column tiles
// each.  Each XCD takes a contiguous chunk of the high tiles, then one of the low; its workgroups
// every nper-th of it, those from the end what is left after whole rounds, of which the high
// ones come as two halves if there are workgroups for all.
template <int BM>
struct TileShare {
    const int *off, *high_start, *low_start;             // row offsets, starts of both kinds (LDS)
    int n_groups, n_tiles, nper, widx;
    int high, high0, low0, rounds, whole, last_high, n_list;
    bool halves;

    __device__ __forceinline__ TileShare(const int* s_off, const int* s_high, const int* s_low, int groups,
                                         int tiles)
        : off(s_off), high_start(s_high), low_start(s_low), n_groups(groups), n_tiles(tiles) {
        nper = gridDim.x / NUM_XCD;
        widx = blockIdx.x / NUM_XCD;
        const int xcd = blockIdx.x % NUM_XCD;
        high = share(s_high, xcd, high0);
        const int all = high + share(s_low, NUM_XCD - 1 - xcd, low0);
        rounds = all / nper;
        whole = rounds * nper;
        last_high = max(high - whole, 0);
        halves = BM > 128 && all - whole + last_high <= nper;
        const int left = all - whole + (halves ? last_high : 0);
        n_list = rounds + (nper - 1 - widx < left ? 1 : 0);
    }

    __device__ __forceinline__ int share(const int* start, int xcd, int& begin) const {
        const int total = __builtin_amdgcn_readfirstlane(start[n_groups]);
        const int chunk = (total + NUM_XCD - 1) / NUM_XCD;
        begin = min(xcd * chunk, total);
        return min(chunk, total - begin);
    }

    // Tile q of the workgroup's n_list: its group, first row, rows and column tile.
    struct Tile {
        int g, row0, valid, n;
    };
    __device__ __forceinline__ Tile at(int q) const {
        int i = q * nper + (q < rounds ? widx : nper - 1 - widx), part = 0, parts = 1;
        if (halves && i >= whole) {
            if (i < whole + 2 * last_high) {
                part = (i - whole) & 1;
                parts = 2;
                i = whole + (i - whole) / 2;
            } else {
                i -= last_high;
            }
        }
        TilePos pos;
        int g;
        if (i < high) {
            const int L = high0 + i;
            g = last_le(high_start, n_groups, L);
            pos = tile_pos(L - high_start[g], high_tiles<BM>(off[g + 1] - off[g]), n_tiles);
        } else {
            const int L = low0 + i - high;
            g = last_le(low_start, n_groups, L);
            pos = {high_tiles<BM>(off[g + 1] - off[g]), L - low_start[g]};
        }
        const int rows = off[g + 1] - off[g], m0 = pos.m * BM + part * (BM / 2);
        return {g, off[g] + m0, min(BM / parts, rows - m0), pos.n};
    }
};

}  // namespace
}  // namespace moe
