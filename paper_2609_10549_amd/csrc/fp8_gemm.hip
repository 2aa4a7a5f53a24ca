// Product of 8-bit rows (fp8.h; compass_fp8_gemm):
//
//   C[m][n] = sum_g 2^(sa[m][g] + sw[n][g]) sum_{k in g} A[m][k] W[n][k]
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "compass.h"
#include "fp8.h"
#include "gemm_core.h"
#include "fp8_plan.h"
#include "internal.h"

namespace compass {

namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));

struct ProductParams {
    const uint8_t *A, *W, *sA, *sW;
    uint16_t *C;
    float *part;                 // split: fp32 [slices][part_rows][part_ld], from the first tile on
    int part_rows, part_ld;
    int M, N, K, S;              // S: bytes of a row of scales
    int tiles_m, tiles_n, group_m;
    int m_base, n_base;          // the first tile's row and column
    int slices, kslice;          // slices of K (kslice a multiple of 512)
};

// One global -> LDS load of 16 bytes per lane as dma16, from rsrc + voff + soff: a
// stage's place is the scalar, so that nothing is added per lane and load.
__device__ __forceinline__ void dma16s(i32x4 rsrc, uint32_t voff, uint32_t soff, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds"
                 :
                 : "s"(lds), "v"(voff), "s"(rsrc), "s"(soff)
                 : "memory");
}

// Loads of one operand's stages: D rows of the tile, one group of 128 each, the
// 16-byte chunk c of LDS row `row` at chunk c ^ ((row >> 1) & 7).
// WAVES waves share a stage, 8 rows per load.
template <int D, int WAVES = 4>
struct RowLoader {
    static constexpr int L = D / (8 * WAVES);   // loads per wave and stage
    uint32_t off[L];
    i32x4 rsrc;
    // load q covers rows 8 (WAVES q + wave) + (lane >> 3)
    __device__ __forceinline__ static int row(int q, int lane, int wave) { return 8 * (WAVES * q + wave) + (lane >> 3); }
    __device__ __forceinline__ static int chunk(int q, int lane, int wave) { return (lane & 7) ^ ((row(q, lane, wave) >> 1) & 7); }
    __device__ __forceinline__ void init(const uint8_t *p, int d0, int dim, int K, int lane, int wave) {
        rsrc = tile_rsrc4(p, (uint64_t)dim * (uint64_t)K, (uint64_t)d0 * (uint64_t)K);
        // resource words that came out of vector registers need five wait
        // states before a load reads them
        asm volatile("s_nop 4" : "+s"(rsrc));
#pragma unroll
        for (int q = 0; q < L; ++q) {
            const int i = row(q, lane, wave);
            off[q] = d0 + i < dim ? (uint32_t)i * (uint32_t)K + (uint32_t)chunk(q, lane, wave) * 16u : kOOBRow;
        }
    }
    // The stage at k0 is cut by the end ke, or behind it: the lanes whose chunks lie
    // there load zeros from now on (16 bytes are inside or outside: K is a multiple
    // of 16), wherever the stages that follow are.
    __device__ __forceinline__ void cut(int k0, int ke, int lane, int wave) {
#pragma unroll
        for (int q = 0; q < L; ++q)
            if (k0 + chunk(q, lane, wave) * 16 >= ke) off[q] = kOOBRow;
    }
    __device__ __forceinline__ void load(int q, int k0, uint32_t buf, int wave) const {
        dma16s(rsrc, off[q], (uint32_t)k0, buf + (uint32_t)((q * WAVES + wave) * 1024));
    }
};

// One global -> LDS load of 4 bytes per lane, from an address of its own, to LDS
// byte address lds + 4 * lane; as dma16 of 16 through a resource.
__device__ __forceinline__ void dma4(const uint8_t *from, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" : : "s"(lds), "v"(from) : "memory");
}

// Of n operations spread over slots [lo, hi), those before slot `at`.
constexpr int loads_before(int at, int n, int lo, int hi) {
    int count = 0;
    for (int k = 0; k < n; ++k) count += slot_of(k, n, lo, hi) < at;
    return count;
}

template <int I, int I1, class Step>
__device__ __forceinline__ void each_slot(const Step &step) {
    if constexpr (I < I1) {
        step(std::integral_constant<int, I>{});
        each_slot<I + 1, I1>(step);
    }
}

// BM x BN tiles, 4 waves, WC of them along the columns, NB stage buffers of A and W, a
// group of 128 per stage: one scaled MFMA per block of 16 x 16 and stage, which
// multiplies by both scales itself (a lane's chunks kq and kq + 4 of a row's group lie
// the same way in both operands, and all lanes of a row hold its one scale). Workgroups
// stay and take a tile of every round; the next tile's first stages load under the
// epilogue.
//
// What bounds it: the large tiles, the matrix cores and what feeds them. 8192 x 6144 x
// 12288 445 to 462 us from card to card (2.7 PFLOP/s); MFMAs are busy in 0.59e6 of
// 0.874e6 cycles, at 1.87 GHz (the library's product with one scale for all: 0.759e6
// at 1.93; 455 us on N(0, 1) and 400 on these values). The rest is this kernel's own: where
// the whole took 487 us it took 449 with scales that were constant, 391 without the
// loads to LDS, 362 without either. On the way there: a barrier per stage, loads in its last
// column of blocks and its scales by bytes 514 us; two barriers, the loads over half of
// the stage 478; columns in pairs, scales by words of four stages, their addresses in
// vector registers 466; a stage's place as the loads' scalar offset 459. What did not
// help, beside 484 to 489: touching lines a stage earlier (596 to 601), groups of 2 row
// tiles in place of 4 (504 to 507) or of 8 (480 to 490), 192 x 256 tiles (575).
//
// Small products are bound by a tile's edges and, between one and two workgroups per
// CU, by the CUs that have two: 777 x 5003 x 1552 16 us (280 tiles, 40 of them for 9 rows),
// 768 x 5003 x 1552 13.5 (240), 768 x 5120 x 1536 11.6. Some rows against a long weight, by
// the CUs without a tile or the fp32 slices that fill them: 64 x 6144 x 12288 23 us, 128
// rows 26 (48 tiles in 5 slices), 256 rows 40 (96 in 2), 512 rows 59 (192 tiles), where
// bytes and operations take 16, 16, 17 and 28.
template <int BM, int BN, int WC, int NB, int WGS, bool PART>
__global__ __launch_bounds__(kThreads, WGS) void product_kernel(const ProductParams p) {
    constexpr int WM = BM * WC / 4, WN = BN / WC, FM = WM / 16, FN = WN / 16, NM = FM * FN;
    constexpr int LA = BM / 32, LW = BN / 32, L = LA + LW;
    constexpr int SA = BM * 128, SW = BN * 128;
    constexpr int Q = BN == 2 * BM || BM == 2 * BN ? 2 : 4;   // words of scales per row and block: 4 Q stages
    constexpr int RS = (BM + BN) * Q * 4;        // scales of such a block
    constexpr int RB = FN * 32;                  // epilogue: bytes of a wave's row
    constexpr int REGION = PART ? 0 : 16 * RB;   // 16 rows per wave
    constexpr int SCALES = NB * (SA + SW), EPI = SCALES + 2 * RS, LDS = EPI + 4 * REGION;
    constexpr bool kAcc = WGS == 1;              // accumulators in the other half of the registers
    // The MFMAs of a stage go over pairs of columns of blocks, and there row by row,
    // so that a block row of the last pair is free for the next stage's every other
    // slot: what a wave reads of a stage is spread over two thirds of it. From slot B2
    // on the next stage is read, first the leading half of its columns, then its rows
    // behind their last use (slots RA on); the other columns follow in its own first
    // LATE slots. From slot B1 on a stage is in registers, and its buffers take the
    // loads of the stage NB ahead, until slot DE.
    constexpr int P = FN / 2, RA = (P - 1) * 2 * FM, LATE = NM / 4;
    constexpr int B1 = NM * 6 / 16, B2 = FN == 8 ? NM * 9 / 16 : NM / 2, DE = NM * 12 / 16;
    constexpr int EARLY = RA > B2 ? RA : B2 + (FM + 1) / 2;
    static_assert(LDS * WGS <= (160 << 10), "LDS");
    static_assert(FN % 4 == 0 && LATE < B1 + (B1 == 1) && B1 < B2 && B2 >= FM * FN / 2, "columns free when they are read");
    __shared__ __attribute__((aligned(1024))) char smem[LDS];

    const int tid = threadIdx.x;
    const int lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm0 = wave / WC * WM, wn0 = wave % WC * WN;
    const int tiles = p.tiles_m * p.tiles_n, total = tiles * p.slices, grid = (int)gridDim.x;
    const uint32_t lds0 = (uint32_t)(uintptr_t)LDS_AS(smem);
    const uint32_t ldsW = lds0 + NB * SA, ldsS = lds0 + SCALES;

    struct Tile { int m0, n0, slice, kb, ke; };
    auto tile_of_round = [&](int j, Tile &t) {
        const int pos = round_position(total, grid, (int)blockIdx.x, j);
        if (pos < 0) return false;
        t.slice = pos / tiles;
        const int tpos = pos - t.slice * tiles, gsz = p.group_m * p.tiles_n;
        const int grp = tpos / gsz, rin = tpos - grp * gsz;
        const int rows_here = min(p.group_m, p.tiles_m - grp * p.group_m);
        const int tn = rin / rows_here;
        t.m0 = p.m_base + (grp * p.group_m + rin - tn * rows_here) * BM;
        t.n0 = p.n_base + tn * BN;
        t.kb = t.slice * p.kslice;
        t.ke = min(p.K, t.kb + p.kslice);
        return true;
    };
    // The lane's number, not known to the compiler to be the same at every call:
    // what is derived from it is computed where it is needed, not kept in
    // registers (and spilled) from one tile to the next.
    auto fresh_lane = [&]() {
        int l = lane;
        asm volatile("" : "+v"(l));
        return l;
    };

    RowLoader<BM> la;
    RowLoader<BN> lw;
    // Scales: 64 / Q rows of the tile's BM + BN, Q words each, per piece; a piece per
    // wave and turn (the last row and word stand for those past the ends).
    constexpr int PIECES = (BM + BN) * Q / 64, TURNS = (PIECES + 3) / 4;
    static_assert(TURNS <= 2 * Q, "a stage for each turn, and time to land");
    const int words = p.S / 4;
    // (the bases in vector registers: as scalars they would be loaded again, and
    // waited for, at each call)
    uint64_t baseA = (uint64_t)p.sA, baseW = (uint64_t)p.sW;
    asm volatile("" : "+v"(baseA), "+v"(baseW));
    auto load_scales = [&](const Tile &t, int turn, int block) __attribute__((always_inline)) {
        const int piece = turn * 4 + wave, row = piece * (64 / Q) + lane / Q;
        if (PIECES % 4 != 0 && piece >= PIECES) return;
        const bool ofA = piece * (64 / Q) < BM;
        const int d = ofA ? min(t.m0 + row, p.M - 1) : min(t.n0 + row - BM, p.N - 1);
        const int word = min(t.kb / (4 * kGroup) + block * Q + lane % Q, words - 1);
        const uint64_t at = (ofA ? baseA : baseW) + (uint64_t)(uint32_t)d * (uint32_t)p.S + (uint32_t)(4 * word);
        dma4((const uint8_t *)at,
             (uint32_t)__builtin_amdgcn_readfirstlane((int)(ldsS + (uint32_t)(block & 1) * (uint32_t)RS + (uint32_t)piece * 256u)));
    };
    auto begin = [&](const Tile &t) {   // the tile's first NB stages and its first scales
        const int l = fresh_lane();
        la.init(p.A, t.m0, p.M, p.K, l, wave);
        lw.init(p.W, t.n0, p.N, p.K, l, wave);
#pragma unroll
        for (int q = 0; q < TURNS; ++q) load_scales(t, q, 0);
#pragma unroll
        for (int i = 0; i < NB; ++i) {
            const int k0 = t.kb + i * kGroup;
            if (k0 + kGroup > t.ke) {
                la.cut(k0, t.ke, l, wave);
                lw.cut(k0, t.ke, l, wave);
            }
#pragma unroll
            for (int q = 0; q < LA; ++q) la.load(q, k0, lds0 + i * SA, wave);
#pragma unroll
            for (int q = 0; q < LW; ++q) lw.load(q, k0, ldsW + i * SW, wave);
        }
    };

    Tile cur, nxt;
    if (!tile_of_round(0, nxt)) return;
    begin(nxt);
    for (int round = 1;; ++round) {
        cur = nxt;
        f32x4 acc[FN][FM];
#pragma unroll
        for (int ni = 0; ni < FN; ++ni)
#pragma unroll
            for (int mi = 0; mi < FM; ++mi) acc[ni][mi] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        {
            const int l = fresh_lane(), r = l & 15, kq = l >> 4;
            uint32_t atA[2], atW[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint32_t c = (uint32_t)(((4 * h + kq) ^ ((r >> 1) & 7)) << 4);
                atA[h] = (uint32_t)(wm0 + r) * 128u + c;
                atW[h] = (uint32_t)(wn0 + r) * 128u + c;
            }
            const uint32_t atSA = ldsS + (uint32_t)(wm0 + r) * (4u * Q), atSW = ldsS + (uint32_t)(BM + wn0 + r) * (4u * Q);
            typedef const __attribute__((address_space(3))) i32x4 lds16;
            typedef const __attribute__((address_space(3))) int lds4;
            // block f of an operand whose two chunks of the lane start at `at` in the buffer
            auto read8 = [&](const uint32_t (&at)[2], uint32_t buf, int f) __attribute__((always_inline)) {
                lds16 *lo = (lds16 *)(uintptr_t)(buf + at[0]), *hi = (lds16 *)(uintptr_t)(buf + at[1]);
                return __builtin_shufflevector(lo[f * 128], hi[f * 128], 0, 1, 2, 3, 4, 5, 6, 7);
            };
            auto read_scales = [&](uint32_t at, uint32_t word, int f) __attribute__((always_inline)) {   // of four stages
                return *(lds4 *)(uintptr_t)(at + word + (uint32_t)f * (64u * Q));
            };
            const int KT = (cur.ke - cur.kb + kGroup - 1) / kGroup;
            if (round > 1) __builtin_amdgcn_s_waitcnt(0);
            else wait_vm_lgkm0<(NB - 1) * L>();
            lds_barrier();
            i32x8 a[FM], b[FN];
            int sa[FM], sb[FN], wa[FM], wb[FN];   // scales, and the words of four stages that hold them
#pragma unroll
            for (int ni = 0; ni < FN; ++ni) {
                if (ni < FN / 2) b[ni] = read8(atW, ldsW, ni);
                sb[ni] = wb[ni] = read_scales(atSW, 0u, ni);
            }
#pragma unroll
            for (int mi = 0; mi < FM; ++mi) {
                a[mi] = read8(atA, lds0, mi);
                sa[mi] = wa[mi] = read_scales(atSA, 0u, mi);
            }
            uint32_t bA = lds0, bW = ldsW, sc = 0u;   // this stage's buffers, the word of its scales
            // Every accumulator in a register of its own, here and at each call: without
            // it the compiler rotates them from the constant zero on, and moves a part's
            // MFMAs behind the barrier and the branch that follow it, where their results
            // are used next (19 of a stage's first 20).
            auto pin = [&]() __attribute__((always_inline)) {
#pragma unroll
                for (int i = 0; i < NM; ++i) {
                    if constexpr (kAcc) asm volatile("" : "+a"(acc[i / FM][i % FM]));
                    else asm volatile("" : "+v"(acc[i / FM][i % FM]));
                }
            };
            pin();
            for (int st = 0; st < KT; ++st) {
                pin();
                const uint32_t nA = bA + SA == ldsW ? lds0 : bA + SA, nW = bW + SW == ldsS ? ldsW : bW + SW;
                const int sh = 8 * (st & 3), nsh = 8 * ((st + 1) & 3);   // the stage's byte of its words, the next one's
                const int ahead = cur.kb + (st + NB) * kGroup;   // where the stage that is loaded starts
                auto slot = [&](auto ic) __attribute__((always_inline)) {
                    // down one pair of columns, up the next (the last down, as the first
                    // of the next stage), its two columns by turns: consecutive MFMAs
                    // share an operand
                    constexpr int I = decltype(ic)::value, pair = I / (2 * FM), t = I % (2 * FM);
                    constexpr int mi = pair % 2 == 0 || pair == P - 1 ? t / 2 : FM - 1 - t / 2;
                    constexpr int ni = 2 * pair + ((t ^ (t >> 1)) & 1);
                    acc[ni][mi] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b[ni], a[mi], acc[ni][mi], 0, 0, 0, sb[ni],
                                                                                   0, sa[mi]);
#pragma unroll
                    for (int f = 0; f < FN / 2; ++f) {
                        if (slot_of(f, FN / 2, 0, LATE) == I) {
                            b[FN / 2 + f] = read8(atW, bW, FN / 2 + f);
                            sb[FN / 2 + f] = (int)((uint32_t)wb[FN / 2 + f] >> sh);
                        }
                        if (slot_of(f, FN / 2, B2, EARLY) == I) {
                            b[f] = read8(atW, nW, f);
                            sb[f] = (int)((uint32_t)wb[f] >> nsh);
                        }
                    }
                    if constexpr (I >= RA && t % 2 == 1) {
                        a[mi] = read8(atA, nA, mi);
                        sa[mi] = (int)((uint32_t)wa[mi] >> nsh);
                    }
#pragma unroll
                    for (int j = 0; j < L; ++j)
                        if (slot_of(j, L, B1, DE) == I) {
                            if (j < LA) la.load(j, ahead, bA, wave);
                            else lw.load(j - LA, ahead, bW, wave);
                        }
                    __builtin_amdgcn_sched_barrier(0);
                };
                each_slot<0, B1>(slot);
                pin();
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                lds_barrier();
                // the next block of scales, a turn per stage from this one's first on
                if (const int turn = st & (4 * Q - 1); turn < TURNS && st - turn + 4 * Q < KT)
                    load_scales(cur, turn, st / (4 * Q) + 1);
                if (nsh == 0) {   // this stage's scales are out of their words: the next four stages'
                    sc = (sc & (4u * Q - 4u)) < 4u * Q - 4u ? sc + 4u : sc < (uint32_t)RS ? (uint32_t)RS : 0u;
#pragma unroll
                    for (int mi = 0; mi < FM; ++mi) wa[mi] = read_scales(atSA, sc, mi);
#pragma unroll
                    for (int ni = 0; ni < FN; ++ni) wb[ni] = read_scales(atSW, sc, ni);
                }
                if (ahead + kGroup > cur.ke) {
                    la.cut(ahead, cur.ke, l, wave);
                    lw.cut(ahead, cur.ke, l, wave);
                }
                each_slot<B1, B2>(slot);
                pin();
                // the next stage has landed (loads of scales among those in flight make
                // the count wait for more, not less)
                wait_vm_lgkm0<(NB - 2) * L + loads_before(B2, L, B1, DE)>();
                lds_barrier();
                each_slot<B2, NM>(slot);
                bA = nA;
                bW = nW;
            }
            wait_vm_lgkm0<0>();   // the loads past the end land before the buffers are reused
            __syncthreads();
        }
        const bool more = tile_of_round(round, nxt);
        if (more) begin(nxt);   // under the epilogue

        const int et = fresh_lane();
        // lane (er, eq) holds of block (mi, ni): row er, columns 4 eq + 0..3
        const int er = et & 15, eq = et >> 4;
        const int m1 = cur.m0 + wm0, n1 = cur.n0 + wn0;   // of this wave
        auto hold = [&](int mi) {
            if constexpr (kAcc) {
#pragma unroll
                for (int ni = 0; ni < FN; ++ni) asm volatile("" : "+a"(acc[ni][mi]));
            }
        };
        if constexpr (PART) {
#pragma unroll
            for (int mi = 0; mi < FM; ++mi) {
                hold(mi);
                const int m = m1 + mi * 16 + er;
                if (m < p.M) {
                    float *row = p.part + ((size_t)cur.slice * (size_t)p.part_rows + (size_t)(m - p.m_base)) * (size_t)p.part_ld;
#pragma unroll
                    for (int ni = 0; ni < FN; ++ni) {
                        const int n = n1 + ni * 16 + 4 * eq;
                        // (a row's last vector may end in columns that are not there, and not read)
                        if (n < p.N) *reinterpret_cast<f32x4 *>(row + n - p.n_base) = acc[ni][mi];
                    }
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        } else {
            // Each wave turns 16 rows at a time to row order through LDS of its own
            // (whose operations run in order: nothing waits between a write and its
            // read) and stores whole rows of its columns: chunk c of row r at c ^ (r & SWZ).
            constexpr int CPR = 2 * FN, SWZ = CPR % 8 == 0 ? 7 : 3;
            char *const region = smem + EPI + wave * REGION;
#pragma unroll
            for (int mi = 0; mi < FM; ++mi) {
                char *w = region + er * RB + 8 * (eq & 1);
                hold(mi);
#pragma unroll
                for (int ni = 0; ni < FN; ++ni) {
                    const f32x4 x = acc[ni][mi];
                    *reinterpret_cast<u32x2 *>(w + (((2 * ni + (eq >> 1)) ^ (er & SWZ)) << 4)) =
                        u32x2{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3])};
                }
                asm volatile("" ::: "memory");
#pragma unroll
                for (int it = 0; it < FN / 2; ++it) {
                    const int row = (it * 64 + et) / CPR, j = (it * 64 + et) % CPR;
                    const u32x4 o = *reinterpret_cast<const u32x4 *>(region + row * RB + ((j ^ (row & SWZ)) << 4));
                    const int m = m1 + mi * 16 + row, n = n1 + j * 8;
                    if (m >= p.M) continue;
                    uint16_t *to = p.C + (size_t)m * (size_t)p.N + n;
                    typedef u32x4 Loose __attribute__((aligned(2)));
                    if (n + 8 <= p.N) *reinterpret_cast<Loose *>(to) = o;
                    else
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            if (n + e < p.N) to[e] = (uint16_t)(o[e / 2] >> (16 * (e & 1)));
                }
                asm volatile("" ::: "memory");
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        if (!more) return;
    }
}

// Few rows (at most 16 MT): a workgroup takes 16 columns, each of its waves every
// kFewWaves-th block of 512 of the depth (a word of scales per row). A wave streams
// its own stages of A and W through a ring of kFewRing buffers of its own in LDS, so
// no barrier joins the waves before their sums are added in wave order.
//
// Bound by memory: 8 x 6144 x 12288 14.1 us (75 MB of W at 5.3 TB/s), with 1 to 16 rows.
// (Straight to registers in the matrix core's layout, where neighbouring lanes hold
// different rows, a load takes a clock per lane: 21.9 us, and 26.3 with 16 rows.)
constexpr int kFewWaves = 8, kFewRing = 2, kFewDepth = kFewMaxDepth;
template <int MT>
__global__ __launch_bounds__(kFewWaves * 64) void few_rows_kernel(const ProductParams p) {
    constexpr int SB = (MT + 1) * 2048;   // A's rows, then W's, 128 bytes each
    constexpr int L = 2 * MT + 2;         // loads per stage
    constexpr int ROWS = 16 * MT + 16;
    constexpr int RING = kFewWaves * kFewRing * SB;
    __shared__ __attribute__((aligned(1024))) char smem[RING + ROWS * (kFewDepth / kGroup)];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n0 = (int)blockIdx.x * 16;
    RowLoader<16 * MT, 1> la;
    RowLoader<16, 1> lw;
    la.init(p.A, 0, p.M, p.K, lane, 0);
    lw.init(p.W, n0, p.N, p.K, lane, 0);
    const uint32_t ring = (uint32_t)(uintptr_t)LDS_AS(smem) + (uint32_t)(wave * kFewRing * SB);
    // stage i of this wave starts at 512 (wave + kFewWaves (i / 4)) + 128 (i % 4)
    auto place = [&](int i) { return 512 * (wave + kFewWaves * (i >> 2)) + kGroup * (i & 3); };
    auto load_stage = [&](int i) {
        const int k0 = place(i);
        const uint32_t buf = ring + (uint32_t)(i % kFewRing) * SB;
        if (k0 + kGroup > p.K) {   // (as all that follow are)
            la.cut(k0, p.K, lane, 0);
            lw.cut(k0, p.K, lane, 0);
        }
#pragma unroll
        for (int q = 0; q < 2; ++q) lw.load(q, k0, buf + MT * 2048, 0);
#pragma unroll
        for (int q = 0; q < 2 * MT; ++q) la.load(q, k0, buf, 0);
    };
#pragma unroll
    for (int i = 0; i < kFewRing; ++i) load_stage(i);
    // the rows' scales, words of four stages
    const int words = p.S / 4;
    int *const scales = reinterpret_cast<int *>(smem + RING);
    for (int at = tid; at < ROWS * words; at += kFewWaves * 64) {
        const int row = at / words, word = at % words;
        const uint8_t *from = row < 16 * MT ? p.sA + (size_t)min(row, p.M - 1) * (size_t)p.S
                                       : p.sW + (size_t)min(n0 + row - 16 * MT, p.N - 1) * (size_t)p.S;
        scales[at] = *reinterpret_cast<const int *>(from + 4 * word);
    }
    __syncthreads();
    f32x4 acc[MT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) acc[mt] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    const int r = lane & 15, kq = lane >> 4, swz = (r >> 1) & 7;
    const char *const frag = smem + wave * kFewRing * SB + r * 128;
    int sa[MT] = {}, sw = 0;
    for (int i = 0; place(i) < p.K; ++i) {
        if ((i & 3) == 0) {
            const int word = wave + kFewWaves * (i >> 2);
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) sa[mt] = scales[(mt * 16 + r) * words + word];
            sw = scales[(MT * 16 + r) * words + word];
        }
        wait_vm_lgkm0<(kFewRing - 1) * L>();
        const char *f = frag + (i % kFewRing) * SB;
        i32x8 v[MT + 1];   // A's blocks, then W's
#pragma unroll
        for (int q = 0; q <= MT; ++q) {
            const i32x4 lo = *reinterpret_cast<const i32x4 *>(f + q * 2048 + ((kq ^ swz) << 4));
            const i32x4 hi = *reinterpret_cast<const i32x4 *>(f + q * 2048 + (((4 + kq) ^ swz) << 4));
            v[q] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the stage is in registers before its buffer is refilled
        load_stage(i + kFewRing);
        const int sh = 8 * (i & 3);
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
            acc[mt] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(v[MT], v[mt], acc[mt], 0, 0, 0, (int)((uint32_t)sw >> sh),
                                                                       0, (int)((uint32_t)sa[mt] >> sh));
    }
    wait_vm_lgkm0<0>();   // the loads issued past the end have landed
    __syncthreads();
    f32x4 *sum = reinterpret_cast<f32x4 *>(smem);   // partial sums [wave][row][16 columns]
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) sum[((wave * MT + mt) * 16 + r) * 4 + kq] = acc[mt];
    __syncthreads();
    if (tid >= MT * 64) return;
    const int row = tid >> 2, n = n0 + (tid & 3) * 4;
    f32x4 x = sum[tid];
#pragma unroll
    for (int q = 1; q < kFewWaves; ++q) x += sum[q * MT * 64 + tid];
    if (row >= p.M) return;
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (n + e < p.N) p.C[(size_t)row * (size_t)p.N + n + e] = (uint16_t)pack_bf16x2(x[e], 0.0f);
}

template <bool PART>
hipError_t launch_product(ProductParams p, const TilePlan &pl, hipStream_t stream) {
    const Tile8 &t = kTiles8[pl.cfg];
    const int64_t items = (int64_t)pl.tiles_m * pl.tiles_n * pl.slices;
    const dim3 grid((unsigned)std::min<int64_t>(items, kCUs * t.wg_per_cu));
    switch (pl.cfg) {   // (a template instance for each row of kTiles8)
    case 0: product_kernel<256, 256, 2, 2, 1, PART><<<grid, kThreads, 0, stream>>>(p); break;
    case 1: product_kernel<256, 128, 2, 3, 1, PART><<<grid, kThreads, 0, stream>>>(p); break;
    case 2: product_kernel<128, 128, 2, 2, 2, PART><<<grid, kThreads, 0, stream>>>(p); break;
    case 3: product_kernel<128, 128, 2, 4, 1, PART><<<grid, kThreads, 0, stream>>>(p); break;
    case 4: product_kernel<128, 64, 1, 2, 2, PART><<<grid, kThreads, 0, stream>>>(p); break;
    default: product_kernel<64, 64, 1, 4, 2, PART><<<grid, kThreads, 0, stream>>>(p); break;
    }
    return hipGetLastError();
}

hipError_t launch_products(ProductParams p, const Cut &cut, float *part, hipStream_t stream) {
    if (cut.part[0].cfg == kFewRows) {
        const dim3 grid((unsigned)((p.N + 15) / 16));
        if (p.M <= 16) few_rows_kernel<1><<<grid, kFewWaves * 64, 0, stream>>>(p);
        else if (p.M <= 32) few_rows_kernel<2><<<grid, kFewWaves * 64, 0, stream>>>(p);
        else few_rows_kernel<3><<<grid, kFewWaves * 64, 0, stream>>>(p);
        return hipGetLastError();
    }
    for (int i = 0; i < 2 && cut.part[i].tiles_m; ++i) {
        const TilePlan &pl = cut.part[i];
        p.tiles_m = pl.tiles_m;
        p.tiles_n = pl.tiles_n;
        p.slices = pl.slices;
        p.kslice = pl.kslice * kGroup;
        p.group_m = kTiles8[pl.cfg].rows == 256 ? 4 : 8;
        p.m_base = cut.row0(i);
        p.n_base = cut.col0(i);
        p.part = part;
        p.part_rows = cut.rows_of(i);
        p.part_ld = part_ld(cut.cols_of(i));
        hipError_t e = pl.slices > 1 ? launch_product<true>(p, pl, stream) : launch_product<false>(p, pl, stream);
        if (e == hipSuccess && pl.slices > 1)
            e = launch_join_parts(cut.rows_of(i), cut.cols_of(i), pl.slices, part,
                                  p.C + (size_t)p.m_base * (size_t)p.N + p.n_base, p.N, false, false, stream);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

constexpr int kMaxRows = 1 << 20, kMaxDepth = 1 << 17;

int check_sizes(int M, int N, int K) {
    if (M < 1 || N < 1 || K < 1 || K % 16)
        return set_error(COMPASS_ERR_INVALID, "need positive M, N and K with K a multiple of 16");
    if (M > kMaxRows || N > kMaxRows || K > kMaxDepth)
        return set_error(COMPASS_ERR_UNSUPPORTED, "M = %d, N = %d, K = %d beyond %d, %d, %d", M, N, K, kMaxRows, kMaxRows,
                         kMaxDepth);
    return COMPASS_OK;
}

bool misaligned(const void *p) { return ((uintptr_t)p & 15) != 0; }

}  // namespace

int op_fp8_gemm_workspace(int M, int N, int K, size_t *bytes) {
    const int rc = check_sizes(M, N, K);
    if (rc != COMPASS_OK) return rc;
    if (!bytes) return set_error(COMPASS_ERR_INVALID, "bytes is required");
    *bytes = plan_product(M, N, K).workspace();
    return COMPASS_OK;
}

int op_fp8_gemm(int M, int N, int K, const void *A, const void *A_scale, const void *W, const void *W_scale, void *C,
                void *ws, size_t ws_bytes, void *stream) {
    int rc = check_sizes(M, N, K);
    if (rc != COMPASS_OK) return rc;
    if (!A || !A_scale || !W || !W_scale || !C)
        return set_error(COMPASS_ERR_INVALID, "A, W, their scales and C are required");
    if (misaligned(A) || misaligned(W) || misaligned(C) || ((uintptr_t)A_scale & 3) || ((uintptr_t)W_scale & 3))
        return set_error(COMPASS_ERR_INVALID, "A, W and C must be 16-byte and the scales 4-byte aligned");
    const Cut cut = plan_product(M, N, K);
    if (const size_t need = cut.workspace(); need && (!ws || misaligned(ws) || ws_bytes < need))
        return set_error(COMPASS_ERR_INVALID, "workspace of %zu bytes (16-byte aligned), need %zu", ws_bytes, need);
    int cus;
    if ((rc = current_num_cu(&cus)) != COMPASS_OK) return rc;
    ProductParams p{};
    p.A = (const uint8_t *)A;
    p.W = (const uint8_t *)W;
    p.sA = (const uint8_t *)A_scale;
    p.sW = (const uint8_t *)W_scale;
    p.C = (uint16_t *)C;
    p.M = M;
    p.N = N;
    p.K = K;
    p.S = scale_cols(K);
    const hipError_t e = launch_products(p, cut, (float *)ws, (hipStream_t)stream);
    return e == hipSuccess ? COMPASS_OK : set_error(COMPASS_ERR_HIP, "8-bit product launch: %s", hipGetErrorString(e));
}

}  // namespace compass
