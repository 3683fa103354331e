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

// The work items are (tile, panel) pairs, an expert's tiles in row order, every panel of a tile in
// turn; workgroup b runs on XCD b % 8 and each XCD takes a contiguous range of them.  Every
// wavefront of a workgroup finds the workgroup's item by itself: a lane counts the tiles of a
// few consecutive experts, a scan over the lanes gives their places.  False: no item is left for
// this workgroup.  Offsets are clamped into [0, R] and to rise, whatever they hold.  (N <= 1024;
// offsets null: one expert, all rows.)
__device__ __forceinline__ bool find_tile(const int* offsets, int N, int R, int tile_rows, int panels,
                                          uint32_t block, RowTile* t) {
    const int lane = threadIdx.x & 63;
    const int per = (N + 64) / 64;              // of N + 1, the rows of no expert last
    auto bounds = [&](int e, int* first, int* last) __attribute__((always_inline)) {
        if (!offsets) {
            *first = e == 0 ? 0 : R;
            *last = R;
            return;
        }
        *first = min(max(offsets[min(e, N)], 0), R);
        *last = e < N ? max(min(offsets[e + 1], R), *first) : R;
    };
    int own = 0;
    for (int i = 0; i < per; ++i) {
        const int e = lane * per + i;
        if (e > N) break;
        int first, last;
        bounds(e, &first, &last);
        own += (last - first + tile_rows - 1) / tile_rows;
    }
    int upto = own;
#pragma unroll
    for (int n = 1; n < 64; n *= 2) {
        const int v = __shfl_up(upto, n);
        upto += lane >= n ? v : 0;
    }
    const int64_t items = (int64_t)__builtin_amdgcn_readlane(upto, 63) * panels;
    const int64_t per_xcd = (items + kXcds - 1) / kXcds;
    const int64_t local = block / kXcds;
    const int64_t item = (int64_t)(block % kXcds) * per_xcd + local;
    if (local >= per_xcd || item >= items) return false;
    int tile = (int)(item / panels);
    t->panel = (int)(item - (int64_t)tile * panels);
    const int holder = __builtin_ctzll(__ballot(upto > tile));
    tile -= __builtin_amdgcn_readlane(upto - own, holder);
    for (int e = holder * per;; ++e) {
        int first, last;
        bounds(e, &first, &last);
        const int n = (last - first + tile_rows - 1) / tile_rows;
        if (tile < n || e >= N) {
            t->expert = __builtin_amdgcn_readfirstlane(e);
            t->row0 = __builtin_amdgcn_readfirstlane(first + tile * tile_rows);
            t->rows = __builtin_amdgcn_readfirstlane(min(tile_rows, last - first - tile * tile_rows));
            return true;
        }
        tile -= n;
    }
}

// Workgroups that are enough for any offsets, and as the eight XCDs take their ranges: at most N + 1
// tiles are not full.
inline int64_t tile_groups(int64_t R, int N, int tile_rows, int64_t panels) {
    const int64_t experts = R < N + 1 ? R : N + 1;
    const int64_t tiles = (R + experts * (tile_rows - 1)) / tile_rows;
    return (tiles * panels + kXcds - 1) / kXcds * kXcds;
}

}  // namespace pr2
