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
constexpr int kFewMaxRows = 16, kFewMaxDepth = 1 << 15;

// Partial sums of a split product: floats of a slice (whole 16-byte vectors), bytes.
inline size_t part_stride(int M, int N) { return ((size_t)M * (size_t)N + 3) / 4 * 4; }
inline size_t part_bytes(const TilePlan &pl, int M, int N) {
    return pl.slices > 1 ? (size_t)pl.slices * part_stride(M, N) * 4 : 0;
}

// The cheapest tile and, where tiles are fewer than the card's slots, slices of
// the depth (whole blocks of 512, a word of scales; at least two each); few rows
// their own kernel, by the weight's way from memory or a workgroup's depth.
inline TilePlan plan_product(int M, int N, int K) {
    TilePlan best{};
    const int stages = (K + 127) / 128, blocks = (K + 511) / 512;
    for (int cfg = 0; cfg < kTile8Count; ++cfg) {
        const Tile8 &ts = kTiles8[cfg];
        const int tm = (M + ts.rows - 1) / ts.rows, tn = (N + ts.cols - 1) / ts.cols;
        const double slots = (double)kCUs * ts.wg_per_cu;
        for (int k = 1; k <= kMaxSlices && (k == 1 || (blocks / k >= 2 && (double)tm * tn * k <= 2 * slots)); ++k) {
            const int per = (blocks + k - 1) / k, ns = (blocks + per - 1) / per;
            const double rounds = (double)tm * tn * ns / slots, whole = (double)(long)rounds, rest = rounds - whole;
            const double n = std::min(4 * per, stages);
            double us = 3.0 + whole * (n * ts.full + ts.edge);
            if (rest > 0) us += n * (ts.alone + (ts.full - ts.alone) * rest * rest) + ts.edge;
            // fp32 slices out and in, and the launch that joins them
            if (ns > 1) us += 3.0 + (double)M * N * (8.0 * ns + 2.0) / 4.5e6;
            if (best.tiles_m == 0 || us < best.us) best = {cfg, tm, tn, ns, per * 512, us};
        }
    }
    if (M <= kFewMaxRows && K <= kFewMaxDepth) {
        const int wgs = (N + 15) / 16, rounds = (wgs + 2 * kCUs - 1) / (2 * kCUs);
        const double us = 3.0 + std::max((double)N * K / 6.5e6, rounds * (1.5 + K * 32.0 / 58e3));
        if (us < best.us) best = {kFewRows, 1, wgs, 1, K, us};
    }
    return best;
}

// The weight gradient's tiles (rows of dW, columns) with costs as in kTiles8, a stage
// being 64 rows of the reduction.
constexpr int kGradTileCount = 5;
constexpr Tile8 kGradTiles[kGradTileCount] = {
    {256, 256, 1, 1.10f, 1.47f, 8.2f}, {256, 128, 1, 0.66f, 0.87f, 4.5f}, {128, 128, 2, 0.44f, 0.93f, 3.1f},
    {128, 64, 2, 0.35f, 0.60f, 2.1f},  {64, 64, 3, 0.25f, 0.55f, 1.9f},
};
inline TilePlan plan_grad(int M, int N, int K) {
    TilePlan best{};
    const int stages = (M + 63) / 64;
    for (int cfg = 0; cfg < kGradTileCount; ++cfg) {
        const Tile8 &ts = kGradTiles[cfg];
        const int tn = (N + ts.rows - 1) / ts.rows, tk = (K + ts.cols - 1) / ts.cols;
        const double slots = (double)kCUs * ts.wg_per_cu;
        for (int k = 1; k <= kMaxSlices && (k == 1 || (stages / k >= 4 && (double)tn * tk * k <= 2 * slots)); ++k) {
            const int per = (stages + k - 1) / k, ns = (stages + per - 1) / per;
            const double rounds = (double)tn * tk * ns / slots, whole = (double)(long)rounds, rest = rounds - whole;
            double us = 3.0 + whole * (per * ts.full + ts.edge);
            if (rest > 0) us += per * (ts.alone + (ts.full - ts.alone) * rest * rest) + ts.edge;
            if (ns > 1) us += 3.0 + (double)N * K * (8.0 * ns + 2.0) / 4.5e6;
            if (best.tiles_m == 0 || us < best.us) best = {cfg, tn, tk, ns, per * 64, us};
        }
    }
    return best;
}

}  // namespace compass
