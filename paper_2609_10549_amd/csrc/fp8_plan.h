// How the products of 8-bit rows are cut: output tiles and slices of the depth.
#pragma once
#include <stddef.h>

#include <algorithm>

#include "xent_plan.h"

namespace compass {

// Tiles of the 8-bit product: rows, columns, workgroups per CU, and what they
// cost in microseconds on MI355X (codes of both signs, unit scales): a stage of
// 128 of the depth on a workgroup with most of the card idle (`alone`: 16 tiles) and
// with all CUs full (`full`), a tile's prologue and epilogue. Fitted to depths of
// 512, 2048 and 8192.
struct Tile8 {
    int rows, cols, wg_per_cu;
    float alone, full, edge;
};
constexpr int kTile8Count = 6;
constexpr int kFewRows = kTile8Count;   // cfg of the kernel for few rows
constexpr Tile8 kTiles8[kTile8Count] = {
    {256, 256, 1, 1.10f, 1.33f, 8.0f}, {256, 128, 1, 0.66f, 0.80f, 5.8f}, {128, 128, 2, 0.50f, 0.88f, 3.7f},
    {128, 128, 1, 0.44f, 0.52f, 3.0f}, {128, 64, 2, 0.47f, 0.62f, 2.4f},  {64, 64, 2, 0.30f, 0.43f, 1.8f},
};
constexpr int kFewMaxRows = 48, kFewMaxDepth = 1 << 15;

// Partial sums of a split output (rows x cols of one launch): floats of a row, whole
// 16-byte vectors, and bytes of all slices.
__host__ __device__ inline int part_ld(int cols) { return (cols + 3) / 4 * 4; }
inline size_t part_bytes(int slices, int rows, int cols) {
    return slices > 1 ? (size_t)slices * (size_t)rows * (size_t)part_ld(cols) * 4 : 0;
}

// The cheapest of `count` tiles for a rows x cols output over `stages` stages, and,
// where tiles are fewer than the card's slots, slices of the reduction: whole units of
// `unit` stages, at least `least` units each.
inline TilePlan plan_single(const Tile8 *tiles, int count, int rows, int cols, int stages, int unit, int least) {
    TilePlan best{};
    const int units = (stages + unit - 1) / unit;
    for (int cfg = 0; cfg < count; ++cfg) {
        const Tile8 &ts = tiles[cfg];
        const int tm = (rows + ts.rows - 1) / ts.rows, tn = (cols + ts.cols - 1) / ts.cols;
        const double slots = (double)kCUs * ts.wg_per_cu;
        for (int k = 1; k <= kMaxSlices && (k == 1 || (units / k >= least && (double)tm * tn * k <= 2 * slots)); ++k) {
            const int per = (units + k - 1) / k, ns = (units + per - 1) / per;
            const double rounds = (double)tm * tn * ns / slots, whole = (double)(long)rounds, rest = rounds - whole;
            const double n = std::min(unit * per, stages);
            double us = 3.0 + whole * (n * ts.full + ts.edge);
            // (the power that the busy CUs draw sets the clock of all)
            if (rest > 0) us += n * (ts.alone + (ts.full - ts.alone) * rest * rest) + ts.edge;
            // fp32 slices out and in, and the launch that joins them
            if (ns > 1) us += 3.0 + (double)rows * cols * (8.0 * ns + 2.0) / 4.5e6;
            if (best.tiles_m == 0 || us < best.us) best = {cfg, tm, tn, ns, per * unit, us};
        }
    }
    return best;
}

// The same, or two launches along the longer axis: tiles that fill whole rounds of
// workgroups, then the rest in tiles (and slices) of its own, where the last round of
// one shape would leave most of the card idle.
struct Cut {
    TilePlan part[2];
    int rows, cols;   // of the output
    bool along_m;
    int first;        // length of the long axis in part[0] (the whole of it: one launch)
    int row0(int i) const { return i && along_m ? first : 0; }
    int col0(int i) const { return i && !along_m ? first : 0; }
    int rows_of(int i) const { return !along_m ? rows : i ? rows - first : first; }
    int cols_of(int i) const { return along_m ? cols : i ? cols - first : first; }
    size_t workspace() const {   // (one launch's sums are joined before the next one's)
        size_t most = 0;
        for (int i = 0; i < 2 && part[i].tiles_m; ++i)
            most = std::max(most, part_bytes(part[i].slices, rows_of(i), cols_of(i)));
        return most;
    }
};
inline Cut plan_cut(const Tile8 *tiles, int count, int rows, int cols, int stages, int unit, int least) {
    const bool along_m = rows >= cols;
    const int length = along_m ? rows : cols;
    Cut best{{plan_single(tiles, count, rows, cols, stages, unit, least), {}}, rows, cols, along_m, length};
    double best_us = best.part[0].us;
    for (int cfg = 0; cfg < count; ++cfg) {
        const Tile8 &ts = tiles[cfg];
        const int tm = (rows + ts.rows - 1) / ts.rows, tn = (cols + ts.cols - 1) / ts.cols;
        const int across = along_m ? tn : tm, lines_all = along_m ? tm : tn;
        const long slots = (long)kCUs * ts.wg_per_cu, rounds = (long)tm * tn / slots;
        for (long r = rounds; r >= 1 && r >= rounds - 1; --r) {
            const int lines = (int)(r * slots / across), done = lines * (along_m ? ts.rows : ts.cols);
            const double us = 3.0 + r * ((double)stages * ts.full + ts.edge);
            if (lines < 1 || lines >= lines_all || us >= best_us) continue;
            const TilePlan q = along_m ? plan_single(tiles, count, rows - done, cols, stages, unit, least)
                                       : plan_single(tiles, count, rows, cols - done, stages, unit, least);
            if (us + q.us < best_us) {
                best_us = us + q.us;
                best.part[0] = {cfg, along_m ? lines : tm, along_m ? tn : lines, 1, (stages + unit - 1) / unit * unit, us};
                best.part[1] = q;
                best.first = done;
            }
        }
    }
    return best;
}

// The 8-bit product: slices are whole blocks of 512 (a word of scales), at least two;
// few rows have a kernel of their own, bound by the weight's way from memory, by all
// operands' way from the caches (A once per 16 columns), or by a workgroup's depth (two
// on a CU with up to 16 rows, else one). 48 x 4096 x 4096 7.6 us, in slices of tiles
// 10.1; 32 x 6144 x 12288 20.6, in slices 18.6.
inline Cut plan_product(int M, int N, int K) {
    Cut best = plan_cut(kTiles8, kTile8Count, M, N, (K + 127) / 128, 4, 2);
    if (M <= kFewMaxRows && K <= kFewMaxDepth) {
        const int blocks = (M + 15) / 16, wgs = (N + 15) / 16, slots = blocks == 1 ? 2 * kCUs : kCUs;
        const int rounds = (wgs + slots - 1) / slots;
        const double way = K * 16.0 * (blocks + 1);   // bytes of a workgroup
        const double us = 3.0 + std::max({(double)N * K / 5.6e6, wgs * way / 13e6, rounds * (1.5 + way / 80e3)});
        if (us < best.part[0].us + best.part[1].us) best = {{{kFewRows, 1, wgs, 1, (K + 127) / 128, us}, {}}, M, N, true, M};
    }
    return best;
}

// The weight gradient's tiles (rows of dW, columns), a stage being 64 rows of the
// reduction (`alone`: 16 to 256 tiles of 128 stages).
constexpr int kGradTileCount = 5;
constexpr Tile8 kGradTiles[kGradTileCount] = {
    {256, 256, 1, 1.43f, 1.50f, 9.5f}, {256, 128, 1, 0.90f, 0.94f, 5.3f}, {128, 128, 2, 0.64f, 1.04f, 3.9f},
    {128, 64, 2, 0.56f, 0.80f, 2.6f},  {64, 64, 3, 0.50f, 0.85f, 2.3f},
};
// Groups of 128 columns from the one that holds column k0 to the one that holds column
// k0 + c. (A tile may start inside a group: behind an odd number of tiles of 64 columns.)
__host__ __device__ inline int groups_from(int k0, int c) { return (k0 % 128 + c) / 128; }
inline Cut plan_grad(int M, int N, int K) {
    return plan_cut(kGradTiles, kGradTileCount, N, K, (M + 63) / 64, 1, 4);
}

}  // namespace compass
