// Where the rows of a product grouped by expert lie: group e is rows offsets[e] .. offsets[e + 1] - 1 of the output, and its row tiles
// follow those of group e - 1.  The offsets are the device's, so every workgroup finds its tile for itself: each lane holds the
// last tile of every 64th group, and a ballot finds the first group that ends behind the tile.  Offsets are clamped to 0 .. rows and taken as not falling,
// whatever they hold, so that no tile lies outside the output.
#pragma once

#include "tbik_device.hpp"
#include "tbik_internal.hpp"

namespace tbik {

constexpr int kGroupsPerLane = kMaxGroups / 64;
constexpr int GROUP_PANEL = 8;             // row tiles

struct GroupRows {
    int group, first, end;                 // rows first .. end - 1 of this tile's group, from the tile on
    int row, high;                         // which of the group's row tiles it is, of how many
};

template <int TILE_ROWS>
struct GroupMap {
    int tiles_end[kGroupsPerLane];         // of group 64 j + lane: row tiles of all groups up to and with it
    int begin[kGroupsPerLane], end[kGroupsPerLane];
    int tiles;

    // All 64 lanes of the wavefront.
    __device__ __forceinline__ void read(const int32_t *offsets, int groups, int rows, int lane) {
        int before = 0, floor = min(max(offsets[0], 0), rows);
#pragma unroll
        for (int j = 0; j < kGroupsPerLane; ++j) {
            tiles_end[j] = before;
            begin[j] = end[j] = floor;
            if (j * 64 >= groups) continue;                                      // uniform
            const int e = j * 64 + lane;
            int n = e < groups ? max(min(offsets[e + 1], rows), floor) : floor;  // not falling: the largest so far
#pragma unroll
            for (int d = 1; d < 64; d *= 2) {
                const int up = __shfl_up(n, d);
                if (lane >= d) n = max(n, up);
            }
            const int left = __shfl_up(n, 1), b = lane > 0 ? left : floor;
            int sum = (n - b + TILE_ROWS - 1) / TILE_ROWS;
#pragma unroll
            for (int d = 1; d < 64; d *= 2) {
                const int up = __shfl_up(sum, d);
                if (lane >= d) sum += up;
            }
            begin[j] = b;
            end[j] = n;
            tiles_end[j] = before + sum;
            before = __builtin_amdgcn_readlane(tiles_end[j], 63);
            floor = __builtin_amdgcn_readlane(n, 63);
        }
        tiles = before;
    }

    // Row tile `tile` (uniform, below `tiles`).
    __device__ __forceinline__ GroupRows at(int tile) const {
        GroupRows g{0, 0, 0, 0, 1};
        bool found = false;
#pragma unroll
        for (int j = 0; j < kGroupsPerLane; ++j) {
            const uint64_t behind = __builtin_amdgcn_ballot_w64(tiles_end[j] > tile);
            if (!found && behind) {                                              // uniform
                found = true;
                const int l = __builtin_ctzll(behind);
                const int b = __builtin_amdgcn_readlane(begin[j], l), n = __builtin_amdgcn_readlane(end[j], l);
                const int last = __builtin_amdgcn_readlane(tiles_end[j], l);
                const int high = (n - b + TILE_ROWS - 1) / TILE_ROWS, row = tile - (last - high);
                g = {j * 64 + l, b + row * TILE_ROWS, n, row, high};
            }
        }
        return g;
    }

    // Tile `t` (uniform, below tiles * columns) of a product whose rows have `columns` tiles each: a group's tiles follow those of the group before, row tile by row
    // tile, or (`panels`) in panels of up to GROUP_PANEL of its row tiles, column by column in a panel, so that consecutive tiles share rows of X and columns of the
    // weight.  A division is some 30 instructions, ahead of which the next tile's loads cannot start: the common case takes two.
    __device__ __forceinline__ GroupRows at(int t, int columns, bool panels, int &column) const {
        const int row_tile = t / columns;
        GroupRows g = at(row_tile);
        if (!panels) {
            column = t - row_tile * columns;
            return g;
        }
        return in_panels(g, t, columns, row_tile, column);
    }

private:
    __device__ __forceinline__ GroupRows in_panels(GroupRows g, int t, int columns, int row_tile, int &column) const {
        int row = g.row, rows = g.high, first = 0;                               // of the panel: how many, the first one
        int v = (t - row_tile * columns) + row * columns;                        // the tile's number in its group
        if (rows > GROUP_PANEL) {                                                // panels of about the same height
            const int n = (rows + GROUP_PANEL - 1) / GROUP_PANEL, most = (rows + n - 1) / n, k = v / (most * columns);
            first = k * most;
            v -= first * columns;
            rows = min(most, rows - first);
        }
        column = v / rows;
        g.first += (first + v - column * rows - row) * TILE_ROWS;
        return g;
    }
};

// Row of X for row i of the output.  `tokens`: rows of X; an index outside is taken as the nearest row.
__device__ __forceinline__ int source_row(const int32_t *rows, int i, int tokens) {
    return rows ? min(max(rows[i], 0), tokens - 1) : i;
}

}  // namespace tbik
