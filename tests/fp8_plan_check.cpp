// Host check of the plans of the 8-bit product and the weight gradient (fp8_plan.h).
// Over a grid of sizes, odd ones among them: the launches cover the output once, no
// slice of a reduction is empty, slices start on whole units, partial sums fit the
// workspace. Then, for each size given as "op,M,N,K" (op 0: product, 1: gradient), prints the
// launches that it takes, "op tile split rest" one per line, and last of all those that any size of the
// grid reaches, as "any ...".
#include <cstdio>
#include <set>
#include <tuple>

#define __host__
#define __device__
#include "fp8_plan.h"

using namespace compass;
typedef std::set<std::tuple<int, int, int, int>> Reached;

static bool check(int op, int M, int N, int K, Reached &r) {
    const Cut c = op ? plan_grad(M, N, K) : plan_product(M, N, K);
    const int rows = op ? N : M, cols = op ? K : N;
    const int stages = op ? (M + 63) / 64 : (K + 127) / 128, unit = op ? 1 : 4;
    if (c.rows != rows || c.cols != cols) return false;
    if (c.part[0].cfg == kFewRows && !op) {
        r.insert({op, kFewRows, 0, (M - 1) / 16});   // (the blocks of rows in the place of the part)
        return M <= kFewMaxRows && K <= kFewMaxDepth && c.workspace() == 0 && c.part[1].tiles_m == 0;
    }
    const int length = c.along_m ? rows : cols;
    if (c.part[1].tiles_m == 0 ? c.first != length : c.first < 1 || c.first >= length) return false;
    for (int i = 0; i < 2 && c.part[i].tiles_m; ++i) {
        const TilePlan &p = c.part[i];
        if (p.cfg < 0 || p.cfg >= (op ? kGradTileCount : kTile8Count)) return false;
        const Tile8 &t = (op ? kGradTiles : kTiles8)[p.cfg];
        const int h = c.rows_of(i), w = c.cols_of(i);
        if ((long)p.tiles_m * t.rows < h || (long)(p.tiles_m - 1) * t.rows >= h || (long)p.tiles_n * t.cols < w ||
            (long)(p.tiles_n - 1) * t.cols >= w)
            return false;
        // the first part ends with whole tiles, so that none of it reaches into the rest
        if (i == 0 && c.part[1].tiles_m && (c.first % (c.along_m ? t.rows : t.cols) || p.slices != 1)) return false;
        if (p.slices < 1 || p.slices > kMaxSlices || p.kslice % unit || (long)p.slices * p.kslice < stages ||
            (long)(p.slices - 1) * p.kslice >= stages)
            return false;
        if (part_bytes(p.slices, h, w) > c.workspace() || (p.slices > 1 && (long)h * part_ld(w) / 4 >= (1l << 32))) return false;
        r.insert({op, p.cfg, p.slices > 1, i});
    }
    return true;
}

int main(int argc, char **argv) {
    Reached any, given;
    long sizes = 0;
    for (int op : {0, 1})
        for (int M : {1, 2, 8, 16, 17, 33, 48, 64, 65, 130, 300, 520, 777, 913, 1100, 2100, 3000, 3760, 4096, 5555, 8192, 16384, 70000, 1 << 20})
            for (int N : {8, 64, 72, 136, 600, 1160, 1536, 2600, 4096, 5003, 6144, 9352, 12000, 13170, 16384, 54001, 1 << 20})
                for (int K : {16, 144, 528, 1040, 1552, 2048, 3008, 4208, 6144, 8208, 12288, 16384, 32784, 131072}) {
                    if (!check(op, M, op ? N / 8 * 8 : N, K, any)) return std::printf("op %d M %d N %d K %d\n", op, M, N, K), 1;
                    ++sizes;
                }
    std::printf("ok %ld\n", sizes);
    for (int i = 1; i < argc; ++i) {
        int op, M, N, K;
        if (std::sscanf(argv[i], "%d,%d,%d,%d", &op, &M, &N, &K) != 4 || !check(op, M, N, K, given))
            return std::printf("argument %s\n", argv[i]), 1;
    }
    for (auto &x : given) std::printf("%d %d %d %d\n", std::get<0>(x), std::get<1>(x), std::get<2>(x), std::get<3>(x));
    for (auto &x : any) std::printf("any %d %d %d %d\n", std::get<0>(x), std::get<1>(x), std::get<2>(x), std::get<3>(x));
    return 0;
}
