// Cuts of the products whose ends are fused, at sizes up to the ends of the
// documented ranges: `sizes` checks that each is a launch that can run, and one
// line is printed for each that cannot.
#include "fused_cut.hpp"

#include <cstdio>
#include <vector>

using namespace xfused_host;

namespace {

int faults = 0;

const char *const kTiles[] = {"256 x 256", "128 x 128", "64 x 128"};

// Of a cut that is launched.
void check(const char *what, const Cut &c, int64_t M, int64_t N, int64_t steps, bool gated, bool across, bool may_split)
{
    const int threads = c.tile == kTile256 ? 512 : 256;
    const int64_t rows = std::min(M, kRowsLaunch), cols = gated ? 2 * N : N;
    const int64_t tiles = cdiv(rows, kTileRows[c.tile]) * cdiv(cols, kTileCols[c.tile]);
    const char *why = nullptr;
    if (c.split < 1 || c.chunk < 1)
        why = "nothing is launched";
    else if ((int64_t)c.split * c.chunk < steps || (int64_t)(c.split - 1) * c.chunk >= steps)
        why = "ranges of k";
    else if (!may_split && c.split > 1)
        why = "split";
    else if ((across && c.tile == kTile64) || (c.staged && c.tile != kTile64))
        why = "a tile that there is not";
    else if ((double)tiles * c.split * threads > 4294967296.0)
        why = "more than 2^32 threads";
    else if (!(c.cost > 0.0))
        why = "cost";
    else if (c.split > 1 && ((double)rows * cdiv(N, 4) > 4294967296.0 || c.ld < cols || c.ld % (gated ? 8 : 4)))
        why = "join";
    if (!why)
        return;
    ++faults;
    std::printf("%s M %lld N %lld steps %lld gated %d across %d split %d staged %d: %s (tile %s, %d ranges of %d)\n", what,
                (long long)M, (long long)N, (long long)steps, gated, across, may_split, c.staged, why, kTiles[c.tile], c.split,
                c.chunk);
}

}  // namespace

int main()
{
    // (both sides of each power of two, of the tiles, and the ends)
    std::vector<int64_t> sides, rows;
    for (int k = 0; k <= 22; ++k)
        for (const int64_t d : {-1, 0, 1}) {
            const int64_t n = ((int64_t)1 << k) + d;
            if (n >= 1 && n <= kMaxSide)
                sides.push_back(n);
        }
    for (const int64_t n : {77, 333, 2200000, 2200001, 524289, 262145, 50001})
        sides.push_back(n);
    rows = sides;
    for (const int64_t n : {kMaxRows - 1, kMaxRows, kRowsLaunch + 1})
        rows.push_back(n);
    for (const int cus : {1, 64, 256, 304})
        for (const int64_t M : rows)
            for (const int64_t N : sides)
                for (const int64_t steps : {1, 2, 3, 9, 64, 224, 1024, 65536})
                    for (const bool gated : {false, true}) {
                        if (gated && N > kMaxSide / 2)
                            continue;
                        for (const bool may_split : {false, true}) {
                            // what has k along both rows: copied or staged, whichever takes less
                            const Cut copied = cut_of(M, N, steps, gated, false, may_split, false, cus);
                            const Cut staged = cut_of(M, N, steps, gated, false, may_split, true, cus);
                            check("copied", copied, M, N, steps, gated, false, may_split);
                            for (const double copies : {4.0, 1e3, 1e9}) {
                                const Cut c = takes_less(staged, copied, copies) ? staged : copied;
                                check("taken", c, M, N, steps, gated, false, may_split);
                            }
                            if (!gated)
                                check("across", cut_of(M, N, steps, false, true, may_split, false, cus), M, N, steps, false, true,
                                      may_split);
                        }
                        const Cut c = cut_of(M, N, steps, gated, false, true, false, cus);
                        const Band b = band_of(c, M, N, steps, gated, cus);
                        if (b.body < N)
                            check("band", b.rest, M, N - b.body, steps, gated, false, false);
                    }
    return faults ? 1 : 0;
}
