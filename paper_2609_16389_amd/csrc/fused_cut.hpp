// How the products whose ends are fused are cut into workgroups: tiles, ranges of k,
// bands of columns and pieces of a vocabulary.  Host code without HIP.
#pragma once

#include <math.h>
#include <stddef.h>
#include <stdint.h>

#include <algorithm>

namespace xfused_host {

inline int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline int64_t up_to(int64_t a, int64_t b) { return cdiv(a, b) * b; }

// Inner sizes, columns and vocabularies: a wave's rows of an operand lie within
// the 2^31 bytes that its loads address.
constexpr int64_t kMaxSide = (int64_t)1 << 22;
constexpr int64_t kMaxRows = (int64_t)1 << 30;
constexpr int64_t kMaxStep = (int64_t)1 << 26;   // bytes between rows read in place
constexpr int64_t kRowsLaunch = 65536;           // rows of a result in one launch

// How a product is cut: into tiles, and ranges of k whose sums are joined by a
// second launch.  (Joined by the last workgroup of a tile instead, 3 ranges of 129
// tiles took 29 us in place of 15 and 7: one workgroup reads them too slowly.)
enum TileKind { kTile256, kTile128, kTile64 };   // 256 x 256, 128 x 128, 64 x 128
constexpr int kTileRows[] = {256, 128, 64}, kTileCols[] = {256, 128, 128};
struct Cut {
    TileKind tile;
    bool staged;        // its operands may have any address (kTile64)
    double cost;        // microseconds
    int split, chunk;   // steps of a range
    int64_t ld;         // of the parts
    int halves = 1;     // 2: the rows come twice, as two parts of their values, and are joined too
};

// Rows up to which slopes are kept in two parts (fused_ends.hpp).
constexpr int64_t kTwoParts = 128;

// The least of the rounds of workgroups that the CUs take times the time of one
// (microseconds: its beginning and end, and each step, longer where two share a
// CU), and for a split the parts written and read again.  Fitted to 37 products (8-bit
// and 16-bit, 37 to 8192 rows), each with all tiles and splits.  Microseconds, 256 /
// 128 / 64 rows a tile, split where that is faster: 64 x 8192 x 8192 8-bit 24.3 / 20.0 /
// 16.9; 333 x 5120 x 2048 8-bit 28 / 19.2 / 11.7; 1000 x 8192 x 4096 8-bit 54 / 45.2 / 50.0;
// 2048 x 14336 x 4096 8-bit 121 / 151 / 172; gated 512 x 4096 x 4096 48 / 45.5 / 40.4;
// d_x of 2048 x 2048 x 5632 112 (4 ranges; not split 242) / 123 / 128.
// What it leaves out: what an end stores, and rows across k, which take 1.5 to 1.6 us a
// step of the largest tile (the three products of a head's gradient, 333 x 32001 x 1001:
// 29 / 47 / 29 us by this, 41 / 46 / 49 measured); and of the staged tile three fit on a CU
// (48 KB of LDS, 108 registers) where two are counted.
// across: A's rows are its k (a transposed product), which the smallest tile does
// not take.  Staged products have only that tile: of too many rows and columns
// they have no cut, and its cost is infinite.
struct TileCost {
    double ends, step, shared;
    int per_cu;
};
constexpr TileCost kCost[] = {{6.0, 1.45, 1.45, 1}, {3.0, 0.82, 1.1, 2}, {2.5, 0.43, 0.67, 2}};
inline Cut cut_of(int64_t M, int64_t N, int64_t steps, bool gated, bool across, bool may_split, bool staged, int cu_count)
{
    const int64_t cols = gated ? 2 * N : N, cus = std::max(cu_count, 1);
    M = std::min(M, kRowsLaunch);
    steps = std::max<int64_t>(steps, 1);
    Cut best{};
    best.cost = HUGE_VAL;   // (of no cut: more workgroups of the smallest tile than a launch has)
    for (const TileKind t : {kTile256, kTile128, kTile64}) {
        if ((t == kTile64 && across) || (staged && t != kTile64))
            continue;
        const int64_t tiles = cdiv(M, kTileRows[t]) * cdiv(cols, kTileCols[t]);
        for (int64_t split = 1; split <= 32; ++split) {
            const int64_t chunk = cdiv(steps, split);
            if (split > 1 && (!may_split || chunk < 3 || cdiv(steps, chunk) != split))
                continue;
            const int64_t groups = tiles * split;
            if (t != kTile256 && groups > (int64_t)1 << 22)   // (a launch has at most 2^32 threads)
                break;
            const int64_t rounds = cdiv(groups, cus * kCost[t].per_cu);
            const double step = (groups > cus ? kCost[t].shared : kCost[t].step) * (staged ? 1.5 : 1.0);
            const double join = split > 1 ? 3.0 + (double)split * (double)M * (double)cols * 8.0 / 3.5e6 : 0.0;
            const double cost = (double)rounds * (kCost[t].ends + step * (double)chunk) + join;
            if (cost < best.cost)
                best = Cut{t, staged, cost, (int)split, (int)chunk, gated ? 2 * up_to(N, 4) : up_to(N, 4)};
        }
    }
    return best;
}

// Whether the staged tiles take less than a product that needs copies first
// (microseconds).
inline bool takes_less(const Cut &staged, const Cut &copied, double copies)
{
    return staged.cost < copied.cost + copies;
}

// Where the last round of large tiles would leave CUs idle: the columns of the whole
// rounds (`body`), and the cut of those after them, which are a launch of their own.
// (8-bit 4096 x 5120 x 4096, one round and a quarter: 93 us in place of 115; 4096 x
// 14336 x 4096, three and a half: 250 in place of 264, with x's 8-bit rows; gated 2048 x
// 2048 x 5632, one and three eighths: 96 in place of 108.)
struct Band {
    int64_t body;   // all columns: no band
    Cut rest;
};
inline Band band_of(const Cut &c, int64_t M, int64_t N, int64_t steps, bool gated, int cu_count)
{
    const int64_t cus = std::max(cu_count, 1), width = gated ? 128 : 256, rows = cdiv(M, 256);
    const int64_t whole = c.tile == kTile256 && c.split == 1 && M <= kRowsLaunch ? rows * cdiv(N, width) / cus : 0;
    const int64_t body = whole * cus / rows * width;
    if (body <= 0 || body >= N)
        return Band{N, c};
    const Cut rest = cut_of(M, N - body, steps, gated, false, false, false, cu_count);
    const double cost = (double)whole * (kCost[kTile256].ends + kCost[kTile256].step * (double)c.chunk) + rest.cost + 3.0;
    return cost < 0.97 * c.cost ? Band{body, rest} : Band{N, c};
}

inline size_t part_bytes(const Cut &c, int64_t M)
{
    return c.split * c.halves > 1 ? (size_t)c.split * (size_t)std::min(M, kRowsLaunch) * c.ld * 4 : 0;
}

// Distance of rows of slopes: a line more than whole 4 KB, where rows that many
// apart would share a few of memory's channels.
inline int64_t slope_ld(int64_t n) { return up_to(n, 8) + (n * 2 % 4096 == 0 ? 64 : 0); }

// Columns of the vocabulary at a time: what holds the slopes of a piece (16 bits
// each) stays near 256 MB.
inline int64_t head_piece(int64_t T, int64_t V)
{
    const int64_t some = ((int64_t)1 << 27) / std::max<int64_t>(T, 1);
    return std::min(up_to(V, 8), std::max<int64_t>(some / 2048 * 2048, 2048));
}

}  // namespace xfused_host
