// Rows sorted by expert in tiles, found by each workgroup from the experts' offsets.
#pragma once

#include "common.h"

namespace pr2 {

constexpr int kXcds = 8;

struct RowTile {
    int expert;         // N: rows that belong to no expert (from offsets[N] on)
    int row0, rows;
    int panel;
};

// inclusive sum over the wavefront's lanes
__device__ __forceinline__ int lane_scan(int v) {
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);     // from 1, 2, 4, 8 lanes below in a row of 16
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);     // a row's last lane to the next row
    v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);     // lane 31 to the upper half
    return v;
}

// The work items are (tile, panel) pairs, an expert's tiles in row order, every panel of a tile in
// turn, or (BY_PANEL) every tile of an expert's panel in turn; workgroup b runs on XCD b % 8 and
// each XCD takes a contiguous range of them.  Every wavefront of a workgroup finds the workgroup's
// item by itself: a lane counts the tiles of a few consecutive experts, a scan over the lanes
// gives their places, and the lane that holds the item's tile hands it to the others.  That takes one
// load's latency and no launch or workspace.  False: no item is left for this workgroup.  Offsets are
// clamped into [0, R] and to rise, whatever they hold.  (N <= 1024; offsets null: one expert, all rows.)
template <bool BY_PANEL = false>
__device__ __forceinline__ bool find_tile(const int* offsets, int N, int R, int tile_rows, int panels,
                                          uint32_t block, RowTile* t) {
    const int lane = threadIdx.x & 63;
    constexpr int kHeld = 4;                    // experts a lane holds in registers
    const int per = offsets ? (N + 64) / 64 : 1;        // of N + 1, the rows of no expert last
    int at[kHeld + 1];                          // where each expert's rows begin
    auto offset = [&](int e) __attribute__((always_inline)) {
        return min(max(offsets[min(e, N)], 0), R);
    };
    auto tiles_of = [&](int first, int last) __attribute__((always_inline)) {
        return (max(last - first, 0) + tile_rows - 1) / tile_rows;
    };
    // rows of expert e, whose offsets are first and next
    auto end_of = [&](int e, int first, int next) __attribute__((always_inline)) {
        return e < N ? max(next, first) : (e == N ? R : first);
    };
    const int e0 = lane * per;
    int own = 0;
    if (!offsets) {
        at[0] = lane == 0 ? 0 : R;
        at[1] = R;
        own = tiles_of(at[0], R);
    } else if (per <= kHeld) {
#pragma unroll
        for (int i = 0; i <= kHeld; ++i) at[i] = i <= per ? offset(e0 + i) : 0;
#pragma unroll
        for (int i = 0; i < kHeld; ++i)
            if (i < per) own += tiles_of(at[i], end_of(e0 + i, at[i], at[i + 1]));
    } else {
        for (int i = 0; i < per && e0 + i <= N; ++i) {
            const int first = offset(e0 + i);
            own += tiles_of(first, end_of(e0 + i, first, offset(e0 + i + 1)));
        }
    }
    const int upto = lane_scan(own);
    const uint32_t items = (uint32_t)__builtin_amdgcn_readlane(upto, 63) * (uint32_t)panels;
    const uint32_t per_xcd = (items + kXcds - 1) / kXcds;
    const uint32_t local = block / kXcds;
    const uint32_t item = block % kXcds * per_xcd + local;
    if (local >= per_xcd || item >= items) return false;
    const int tile = (int)(item / (uint32_t)panels);
    const uint64_t above = __ballot(upto > tile);
    if (!above) return false;                   // (offsets that fall can count more tiles than an int holds)
    const int holder = __builtin_ctzll(above);
    // in the lane that holds the tile: its expert, that one's rows and the tiles before them
    int before = upto - own, expert = e0, first = 0, last = 0;
    if (!offsets) {
        first = at[0];
        last = R;
    } else if (per <= kHeld) {
        bool found = false;
#pragma unroll
        for (int i = 0; i < kHeld; ++i) {
            if (i >= per || found) continue;
            expert = e0 + i;
            first = at[i];
            last = end_of(expert, first, at[i + 1]);
            const int n = tiles_of(first, last);
            found = tile - before < n;
            before += found ? 0 : n;
        }
    } else if (lane == holder) {
        for (int i = 0; i < per; ++i) {
            expert = e0 + i;
            first = offset(expert);
            last = end_of(expert, first, offset(expert + 1));
            const int n = tiles_of(first, last);
            if (tile - before < n) break;
            before += n;
        }
    }
    before = __builtin_amdgcn_readlane(before, holder);
    first = __builtin_amdgcn_readlane(first, holder);
    last = __builtin_amdgcn_readlane(last, holder);
    t->expert = __builtin_amdgcn_readlane(expert, holder);
    const int n = tiles_of(first, last);
    if (n < 1) return false;                    // (the same)
    const uint32_t in = item - (uint32_t)before * (uint32_t)panels;       // item of the expert's
    int which;
    if (BY_PANEL) {
        which = (int)(in % (uint32_t)n);
        t->panel = (int)(in / (uint32_t)n);
    } else {
        which = tile - before;
        t->panel = (int)(in - (uint32_t)which * (uint32_t)panels);
    }
    // (the same; a panel may be below 0 then, too)
    if (which < 0 || which >= n || (uint32_t)t->panel >= (uint32_t)panels) return false;
    t->row0 = first + which * tile_rows;
    t->rows = min(tile_rows, last - t->row0);
    return true;
}

// Workgroups that are enough for any offsets, and as the eight XCDs take their ranges: at most N + 1
// tiles are not full.
inline int64_t tile_groups(int64_t R, int N, int tile_rows, int64_t panels) {
    const int64_t experts = R < N + 1 ? R : N + 1;
    const int64_t tiles = (R + experts * (tile_rows - 1)) / tile_rows;
    return (tiles * panels + kXcds - 1) / kXcds * kXcds;
}

}  // namespace pr2
