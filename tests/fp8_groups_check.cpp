// Host check of where the weight gradient finds the scales of a tile's columns
// (fp8_plan.h), in the plans of its own tiles and of others, as another fit of their
// costs would give them: where a rest starts inside a group of 128 columns, and its tiles
// are wider than that.
#include <cstdio>

#define __host__
#define __device__
#include "fp8_plan.h"

using namespace compass;

// The narrow tiles cheap in whole rounds, the wide ones where most CUs are idle.
static const Tile8 kNarrow[2] = {{64, 64, 3, 2.0f, 0.1f, 0.1f}, {128, 128, 2, 0.2f, 2.0f, 0.3f}};
static const Tile8 kWide[2] = {{128, 64, 2, 2.0f, 0.1f, 0.1f}, {256, 256, 1, 0.3f, 3.0f, 0.2f}};

int main() {
    long inside = 0, columns = 0;
    const struct { const Tile8 *tiles; int count; } sets[] = {{kGradTiles, kGradTileCount}, {kNarrow, 2}, {kWide, 2}};
    for (auto &set : sets)
        for (int M : {1, 64, 777, 4096})
            for (int N : {8, 64, 200, 1000, 1536, 3000})
                for (int K = 144; K < 60000; K += K / 3 / 16 * 16 + 16) {
                    const Cut cut = plan_cut(set.tiles, set.count, N, K, (M + 63) / 64, 1, 4);
                    for (int i = 0; i < 2 && cut.part[i].tiles_m; ++i) {
                        const int width = set.tiles[cut.part[i].cfg].cols;
                        for (int t = 0; t < cut.part[i].tiles_n; ++t) {
                            const int k0 = cut.col0(i) + t * width;
                            inside += k0 % 128 && width > 64;
                            for (int c = 0; c < width && k0 + c < K; c += 16, ++columns)
                                if (k0 / 128 + groups_from(k0, c) != (k0 + c) / 128)
                                    return std::printf("tile at column %d: the scale of column %d is taken from group %d\n", k0,
                                                       k0 + c, k0 / 128 + groups_from(k0, c)), 1;
                        }
                    }
                }
    std::printf("ok %ld %ld\n", columns, inside);
    return inside == 0;   // (such tiles have to be among them)
}
