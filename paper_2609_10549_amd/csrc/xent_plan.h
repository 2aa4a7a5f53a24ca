// How the products of the vocabulary cross entropy are cut: output tiles,
// slices of the reduction, pieces of the vocabulary, and who takes which tile.
#pragma once
#include <stddef.h>

#include <algorithm>


namespace compass {

constexpr int kCUs = 256;   // the card this library is built for; sizes of workspaces follow from it
constexpr int kMaxSlices = 32;
constexpr size_t kPieceBytes = (size_t)512 << 20;   // dz of a default piece

struct TilePlan {
    int cfg;                // row of kTiles
    int tiles_m, tiles_n;
    int slices, kslice;     // slices of the reduction
    double us;              // estimate
};

// The products: logits to statistics, logits to dz, dW = dz^T H, dH = dz W.
enum Product : int { kLogits = 0, kGradLogits = 1, kGradWeight = 2, kGradHidden = 3 };

// Tiles of the products: rows, columns, workgroups per CU, and what they cost
// in microseconds on MI355X (bf16, N(0, 1) data; fitted to 15 sizes from 8 to
// 8192 rows in every tile, four products each, 8 % off on average): a stage of
// 64 of the reduction on one workgroup with most of the card idle (`alone`) and
// with all CUs holding as many as they can (`full`), the factor when rows do not
// start on 128-byte lines (K no multiple of 64), and a tile's prologue and
// epilogue in each product.
struct Tile {
    int rows, cols, wg_per_cu;
    float alone, full, ragged, edge[4];
};
constexpr int kTileCount = 10;
constexpr Tile kTiles[kTileCount] = {
    {256, 256, 1, 1.098f, 1.471f, 1.05f, {11.1f, 13.7f, 8.2f, 11.0f}},
    {256, 192, 1, 0.883f, 1.147f, 1.06f, {6.8f, 10.4f, 6.5f, 6.1f}},
    {256, 128, 1, 0.659f, 0.866f, 1.08f, {4.9f, 8.3f, 4.5f, 3.0f}},
    {192, 192, 1, 0.720f, 0.951f, 1.04f, {4.6f, 7.5f, 4.7f, 3.5f}},
    {128, 192, 1, 0.542f, 0.718f, 1.08f, {4.0f, 5.6f, 4.0f, 3.1f}},
    {128, 128, 2, 0.435f, 0.931f, 1.08f, {2.8f, 4.5f, 3.1f, 1.1f}},
    {128, 128, 1, 0.415f, 0.550f, 1.07f, {3.1f, 4.8f, 3.2f, 1.1f}},   // (deeper stage buffers)
    {128, 64, 1, 0.284f, 0.346f, 1.16f, {2.4f, 3.3f, 2.1f, 0.3f}},
    {64, 64, 2, 0.197f, 0.427f, 1.18f, {1.1f, 2.0f, 1.9f, 0.3f}},
    {64, 256, 1, 0.483f, 0.595f, 1.14f, {2.7f, 4.1f, 3.2f, 1.5f}},
};

// Time of `items` tiles of `per` stages each, by rounds of workgroups. A
// partly filled card runs between the two stage times (the power that the busy
// CUs draw sets the clock of all).
inline double rounds_us(int cfg, Product what, bool ragged, double items, int per) {
    const Tile &t = kTiles[cfg];
    const double rounds = items / ((double)kCUs * t.wg_per_cu);
    const double whole = (double)(long)rounds, rest = rounds - whole;
    const double stages = per * (ragged ? t.ragged : 1.0f);
    double us = whole * (stages * t.full + t.edge[what]);
    if (rest > 0) us += stages * (t.alone + (t.full - t.alone) * rest * rest) + t.edge[what];
    return us;
}

// The cheapest tile for C (M x N) over a reduction of R, with at most
// max_slices slices of it, each at least 8 stages deep.
inline TilePlan plan_tiles(Product what, bool ragged, int M, int N, int R, int max_slices) {
    TilePlan best{};
    const int stages = (R + 63) / 64;
    for (int cfg = 0; cfg < kTileCount; ++cfg) {
        const Tile &ts = kTiles[cfg];
        const int tm = (M + ts.rows - 1) / ts.rows, tn = (N + ts.cols - 1) / ts.cols;
        for (int k = 1; k <= max_slices && (k == 1 || stages / k >= 8); ++k) {
            const int per = (stages + k - 1) / k, ns = (stages + per - 1) / per;
            double t = rounds_us(cfg, what, ragged, (double)tm * tn * ns, per);
            // fp32 slices out and in, and the launch that joins them
            if (ns > 1) t += 4.0 + (double)M * N * (8.0 * ns + 2.0) / 4.5e6;
            if (best.tiles_m == 0 || t < best.us) best = {cfg, tm, tn, ns, per * 64, t};
        }
    }
    return best;
}

// Work position of workgroup b of `grid` in its round j, of `total` positions,
// or -1. Each XCD (workgroups go round-robin over them) walks a run of its own,
// an eighth of the positions (so all have workgroups, or grid = total).
__host__ __device__ inline int round_position(int total, int grid, int b, int j) {
    const int v = b & 7, at = j * ((grid >> 3) + (v < (grid & 7) ? 1 : 0)) + (b >> 3);
    if (at >= (total >> 3) + (v < (total & 7) ? 1 : 0)) return -1;
    return v * (total >> 3) + (v < (total & 7) ? v : (total & 7)) + at;
}

// A product in one launch, or in two along its long axis (rows of C with
// along_m, else columns): tiles that fill whole rounds of workgroups, then the
// rest in tiles of its own, where the last round of one shape would leave most
// of the card idle.
struct PairPlan {
    TilePlan part[2];
    int first;   // length of the long axis in part[0] (the whole of it: one launch)
};
inline PairPlan plan_pair(Product what, bool ragged, int M, int N, int R, bool along_m) {
    const int length = along_m ? M : N;
    PairPlan best{{plan_tiles(what, ragged, M, N, R, 1), {}}, length};
    double best_us = best.part[0].us;
    const int per = (R + 63) / 64;
    for (int cfg = 0; cfg < kTileCount; ++cfg) {
        const Tile &ts = kTiles[cfg];
        const int tm = (M + ts.rows - 1) / ts.rows, tn = (N + ts.cols - 1) / ts.cols;
        const int across = along_m ? tn : tm, lines_all = along_m ? tm : tn;
        const long slots = (long)kCUs * ts.wg_per_cu, rounds = (long)tm * tn / slots;
        for (long r = rounds; r >= 1 && r >= rounds - 1; --r) {
            const int lines = (int)(r * slots / across);
            const int done = lines * (along_m ? ts.rows : ts.cols);
            if (lines < 1 || lines >= lines_all) continue;
            const int rest = length - done;
            const TilePlan q = along_m ? plan_tiles(what, ragged, rest, N, R, 1) : plan_tiles(what, ragged, M, rest, R, 1);
            const TilePlan p{cfg, along_m ? lines : tm, along_m ? tn : lines, 1, per * 64,
                             rounds_us(cfg, what, ragged, (double)lines * across, per)};
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
    b.dh = plan_tiles(kGradHidden, K % 64 != 0, M, K, b.ldz, kMaxSlices);
    b.dz_bytes = ((size_t)M * (size_t)b.ldz * 2 + 255) / 256 * 256 + 256;   // and the peak
    b.part_bytes = b.pieces.count > 1 || b.dh.slices > 1 ? (size_t)b.dh.slices * (size_t)M * (size_t)K * 4 : 0;
    return b;
}

// Row statistics that the tiles of the forward pass leave: two per column tile.
inline int stat_parts(const PairPlan &pl) { return 2 * (pl.part[0].tiles_n + pl.part[1].tiles_n); }

}  // namespace compass
