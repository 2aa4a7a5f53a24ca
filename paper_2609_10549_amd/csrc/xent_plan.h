// How the products of the vocabulary cross entropy are cut: output tiles,
// slices of the reduction, pieces of the vocabulary. Host only.
#pragma once
#include <stddef.h>

#include <algorithm>

#include "plan.h"

namespace compass {

constexpr int kCUs = 256;   // the card this library is built for; sizes of workspaces follow from it
constexpr int kMaxSlices = 16;
constexpr size_t kPieceBytes = (size_t)512 << 20;   // dz of a default piece

struct TilePlan {
    int cfg;                // TileCfg
    int tiles_m, tiles_n;
    int slices, kslice;     // slices of the reduction
    double us;              // estimate
};

// Stages' and edges' time of `items` tiles of `per` stages each, by rounds of
// workgroups, from the costs that the plain GEMM's plan is fitted to (plan.h).
inline double rounds_us(int cfg, double items, int per) {
    const TileCost &tc = kTileCosts[cfg];
    const double rounds = items / ((double)kCUs * kTileShapes[cfg].wg_per_cu);
    const double whole = (double)(long)rounds, rest = rounds - whole;
    double t = whole * (per * tc.full + tc.edge);
    if (rest > 0) t += per * (tc.alone + (tc.full - tc.alone) * rest * rest) + tc.edge;
    return t;
}

// (as large as its deep form in everything but LDS)
inline bool tile_used(int cfg) { return cfg != kTile128x64; }

// The cheapest tile, with at most max_slices slices of the reduction, each at
// least 8 stages deep.
inline TilePlan plan_tiles(int M, int N, int R, int max_slices) {
    TilePlan best{};
    const int stages = (R + 63) / 64;
    for (int cfg = 0; cfg < kTileCfgs; ++cfg) {
        if (!tile_used(cfg)) continue;
        const TileShape &ts = kTileShapes[cfg];
        const int tm = (M + ts.rows - 1) / ts.rows, tn = (N + ts.cols - 1) / ts.cols;
        for (int k = 1; k <= max_slices && (k == 1 || stages / k >= 8); ++k) {
            const int per = (stages + k - 1) / k, ns = (stages + per - 1) / per;
            double t = rounds_us(cfg, (double)tm * tn * ns, per);
            // fp32 slices out and in, and the launch that joins them
            if (ns > 1) t += 4.0 + (double)M * N * (8.0 * ns + 2.0) / 4.5e6;
            if (best.tiles_m == 0 || t < best.us) best = {cfg, tm, tn, ns, per * 64, t};
        }
    }
    return best;
}

// A product in one launch, or in two along its long axis (rows of C with
// along_m, else columns): tiles that fill whole rounds of workgroups, then the
// rest in tiles of its own, where the last round of one shape would leave most
// of the card idle.
struct PairPlan {
    TilePlan part[2];
    int first;   // length of the long axis in part[0] (the whole of it: one launch)
};
inline PairPlan plan_pair(int M, int N, int R, bool along_m) {
    const int length = along_m ? M : N;
    PairPlan best{{plan_tiles(M, N, R, 1), {}}, length};
    double best_us = best.part[0].us;
    const int per = (R + 63) / 64;
    for (int cfg = 0; cfg < kTileCfgs; ++cfg) {
        if (!tile_used(cfg)) continue;
        const TileShape &ts = kTileShapes[cfg];
        const int tm = (M + ts.rows - 1) / ts.rows, tn = (N + ts.cols - 1) / ts.cols;
        const int across = along_m ? tn : tm, lines_all = along_m ? tm : tn;
        const long slots = (long)kCUs * ts.wg_per_cu, rounds = (long)tm * tn / slots;
        for (long r = rounds; r >= 1 && r >= rounds - 1; --r) {
            const int lines = (int)(r * slots / across);
            const int done = lines * (along_m ? ts.rows : ts.cols);
            if (lines < 1 || lines >= lines_all) continue;
            const int rest = length - done;
            const TilePlan q = along_m ? plan_tiles(rest, N, R, 1) : plan_tiles(M, rest, R, 1);
            const TilePlan p{cfg, along_m ? lines : tm, along_m ? tn : lines, 1, per * 64,
                             rounds_us(cfg, (double)lines * across, per)};
            if (p.us + 3.0 + q.us < best_us) {
                best_us = p.us + 3.0 + q.us;
                best = {{p, q}, done};
            }
        }
    }
    return best;
}

// Pieces of the vocabulary of a backward pass, all but the last `cols` wide.
struct Pieces { int cols, count; };
inline Pieces plan_pieces(int M, int V, int K, int piece) {
    int cols = piece;
    if (cols == 0) {
        // as many columns of dz as kPieceBytes holds; where they are several
        // pieces, each a multiple of what fills whole rounds of 256 x 256 tiles
        // in dz (M rows) and dW (K columns)
        const int tiles = std::min((M + 255) / 256, (K + 255) / 256);
        const size_t fit = std::max<size_t>(kPieceBytes / ((size_t)M * 2), 256);
        if ((size_t)V <= fit) {
            cols = V;
        } else {
            size_t unit = 256 * (size_t)std::max(1, kCUs / tiles);
            if (unit > fit) unit = 256;
            const size_t most = fit / unit * unit, count = ((size_t)V + most - 1) / most;
            cols = (int)(((size_t)V + count * unit - 1) / (count * unit) * unit);
        }
    }
    cols = std::min(cols, V);
    return {cols, (V + cols - 1) / cols};
}

// dz's row length: whole stages of the reduction of dz W
inline int dz_columns(int cols) { return (cols + 63) / 64 * 64; }

struct BackwardPlan {
    Pieces pieces;
    TilePlan dh;      // of a whole piece
    int ldz;
    size_t dz_bytes, part_bytes;
};
inline BackwardPlan plan_backward(int M, int V, int K, int piece) {
    BackwardPlan b;
    b.pieces = plan_pieces(M, V, K, piece);
    b.ldz = dz_columns(b.pieces.cols);
    b.dh = plan_tiles(M, K, b.ldz, kMaxSlices);
    b.dz_bytes = ((size_t)M * (size_t)b.ldz * 2 + 255) / 256 * 256 + 256;   // and the peak
    b.part_bytes = b.pieces.count > 1 || b.dh.slices > 1 ? (size_t)b.dh.slices * (size_t)M * (size_t)K * 4 : 0;
    return b;
}

// Row statistics that the tiles of the forward pass leave: two per column tile.
inline int stat_parts(const PairPlan &pl) { return 2 * (pl.part[0].tiles_n + pl.part[1].tiles_n); }

}  // namespace compass
