// Host check of the cross entropy's plans (xent_plan.h). Over a grid of sizes,
// odd ones among them: the rounds of all workgroups take every work position
// once; the launches of a product cover it; no slice of a reduction is empty; the
// pieces cover the vocabulary and their dz and partial sums fit the workspace.
// Then, for each size given as "M,V,K,piece", prints the tiles that its
// products take, one "product tile" per line (4: dH by partial sums), and last of all the tiles that any
// size of the grid reaches, as "any product tile".
#include <cstdio>
#include <cstdlib>
#include <set>
#include <utility>
#include <vector>

#define __host__
#define __device__
#include "xent_plan.h"

using namespace compass;
typedef std::set<std::pair<int, int>> Reached;

static bool tiles_ok(const TilePlan &p, int M, int N, int R) {
    const Tile &t = kTiles[p.cfg];
    const int stages = (R + 63) / 64;
    return p.cfg >= 0 && p.cfg < kTileCount && (long)p.tiles_m * t.rows >= M && (long)(p.tiles_m - 1) * t.rows < M &&
           (long)p.tiles_n * t.cols >= N && (long)(p.tiles_n - 1) * t.cols < N && p.slices >= 1 && p.kslice % 64 == 0 &&
           (long)p.slices * p.kslice >= (long)stages * 64 && (long)(p.slices - 1) * p.kslice < R &&
           (long)p.tiles_m * p.tiles_n * p.slices < (1l << 31);
}

static bool pair_ok(Product what, const PairPlan &p, int M, int N, int R, bool along_m, Reached &r) {
    const int length = along_m ? M : N, rest = length - p.first;
    r.insert({what, p.part[0].cfg});
    if (p.part[0].slices != 1 || !tiles_ok(p.part[0], along_m ? p.first : M, along_m ? N : p.first, R)) return false;
    if (p.part[1].tiles_m == 0) return rest == 0;
    r.insert({what, p.part[1].cfg});
    const Tile &t = kTiles[p.part[0].cfg];
    return rest > 0 && p.first % (along_m ? t.rows : t.cols) == 0 && p.part[1].slices == 1 &&
           tiles_ok(p.part[1], along_m ? rest : M, along_m ? N : rest, R);
}

static bool check(int M, int V, int K, int piece, Reached &r) {
    const bool ragged = K % 64 != 0;
    if (!pair_ok(kLogits, plan_pair(kLogits, ragged, M, V, K, false), M, V, K, false, r)) return false;
    const BackwardPlan b = plan_backward(M, V, K, piece);
    if (b.pieces.cols < 1 || (long)b.pieces.cols * b.pieces.count < V || (long)b.pieces.cols * (b.pieces.count - 1) >= V)
        return false;
    if (piece == 0 && b.pieces.count > 1 && (size_t)M * 2 * b.pieces.cols > kPieceBytes && b.pieces.cols > 256) return false;
    r.insert({b.part_bytes ? kGradHidden + 1 : kGradHidden, b.dh.cfg});
    if (!tiles_ok(b.dh, M, K, b.ldz)) return false;
    for (int i = 0; i < b.pieces.count; i += b.pieces.count > 1 ? b.pieces.count - 1 : 1) {
        const int cols = i + 1 < b.pieces.count ? b.pieces.cols : V - i * b.pieces.cols, ldz = dz_columns(cols);
        if (ldz % 64 || ldz < cols || (size_t)M * ldz * 2 + 256 > b.dz_bytes) return false;
        if (!pair_ok(kGradLogits, plan_pair(kGradLogits, ragged, M, ldz, K, false), M, ldz, K, false, r)) return false;
        if (!pair_ok(kGradWeight, plan_pair(kGradWeight, ragged, cols, K, M, true), cols, K, M, true, r)) return false;
    }
    return b.pieces.count == 1 && b.dh.slices == 1 ? b.part_bytes == 0
                                                   : b.part_bytes == (size_t)b.dh.slices * M * K * 4;
}

int main(int argc, char **argv) {
    for (int total : {1, 7, 8, 9, 255, 256, 257, 511, 800, 6304})
        for (int grid : {1, 5, 8, 97, 256, 512}) {
            if (grid > total || (grid < 8 && grid < total)) continue;
            std::vector<int> seen(total, 0);
            for (int b = 0; b < grid; ++b)
                for (int j = 0, pos; (pos = round_position(total, grid, b, j)) >= 0; ++j) ++seen[pos];
            for (int n : seen)
                if (n != 1) return std::printf("positions of %d over %d workgroups\n", total, grid), 1;
        }
    Reached any;
    long sizes = 0;
    for (int M : {1, 2, 8, 17, 64, 65, 130, 200, 300, 520, 777, 1100, 1544, 2100, 3000, 4096, 5555, 8192, 16384})
        for (int V : {1, 63, 130, 600, 1161, 1536, 2600, 4099, 6283, 9001, 12000, 20011, 32000, 50257, 100003, 131072})
            for (int K : {8, 72, 136, 264, 520, 552, 1024, 1544, 2048, 4096, 6144, 8200, 12288, 16384})
                for (int piece : {0, 1000}) {
                    if (piece >= V) continue;
                    if (!check(M, V, K, piece, any)) return std::printf("M %d V %d K %d piece %d\n", M, V, K, piece), 1;
                    ++sizes;
                }
    std::printf("ok %ld\n", sizes);
    Reached given;
    for (int i = 1; i < argc; ++i) {
        int M, V, K, piece;
        if (std::sscanf(argv[i], "%d,%d,%d,%d", &M, &V, &K, &piece) != 4 || !check(M, V, K, piece, given))
            return std::printf("argument %s\n", argv[i]), 1;
    }
    for (auto &x : given) std::printf("%d %d\n", x.first, x.second);
    for (auto &x : any) std::printf("any %d %d\n", x.first, x.second);
    return 0;
}
