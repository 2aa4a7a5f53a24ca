// Softmax cross entropy of a vocabulary shard straight from hidden states and
// output weight, and its gradients (compass_xent_*).
//
//   z[m][v] = sum_k H[m][k] W[v][k]
//   lse[m]  = log sum_v exp z[m][v],  loss[m] = lse[m] - z[m][target[m]]
//   dz[m][v] = grad[m] (exp(z[m][v] - lse[m]) - [v == target[m]])
//   dH = dz W,  dW = dz^T H
//
// The logits never reach memory: forward, each tile of z is reduced to a
// maximum and a sum of exponentials per row in its epilogue; backward, z is
// computed again in pieces of the vocabulary and leaves its tile as dz in
// bf16, which two products then read.
//
// tile_kernel is one bf16 MFMA product C = A B over a reduction axis whose
// operands may each lie with the reduction along their rows (H, W in z = H W^T,
// dz in dz W) or across them (W in dz W, dz and H in dz^T H). Operands of the
// second kind go to LDS as they lie, 64 reduction rows of a tile's columns per
// stage, and reach the matrix cores through the transposing LDS read
// (ds_read_b64_tr_b16), so no transposed copy of W, H or dz is made.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "compass.h"
#include "gemm_core.h"
#include "gemm_cross.h"
#include "internal.h"
#include "kernel_params.h"
#include "xent_plan.h"

namespace compass {

namespace {

constexpr float kLog2e = 1.44269504088896340736f;

enum Epilogue : int {
    kStats = 0,   // row maxima and sums of exponentials, the targets' logits
    kDz = 1,      // dz in bf16
    kStore = 2,   // the product in bf16
    kPart = 3,    // fp32 partial sums of the product
    kStream = 4,  // kStore by stores that pass through the caches
};

struct TileParams {
    const uint16_t *A, *B;
    uint64_t a_bytes, b_bytes;   // extents; loads beyond them read zero
    int M, N, R;                 // rows and columns of C, reduction length
    int lda, ldb;                // elements between rows of A and B as they lie
    int tiles_m, tiles_n, group_m;
    int m_base, n_base;          // the first tile's row and column
    int slices, kslice;          // reduction slices (kslice a multiple of 64)
    // kStats
    float2 *parts;               // [2 tiles_n][M]: maximum, sum
    float *tlogit;
    // kStats, kDz
    const int64_t *target;
    int64_t v0;                  // vocabulary id of column 0
    // kDz
    const float *lse, *grad;
    uint16_t *dz;                // grad / *peak (exp(z - lse) - [target])
    int ldz;                     // columns [N, ldz) are zero
    float *peak;                 // kStore, kPart: the product is scaled by it
    // kStore, and kPart's last sum
    uint16_t *C;                 // bf16, rows of N
    // kPart
    float *part_out;             // fp32 [slices][M][N], or null: round to C
    const float *part_in;        // added first, same layout (or null)
};

// `read` of the fragments whose slot is I.
template <int F, int NF, int I, int R0, int R1, class Read>
__device__ __forceinline__ void read_slot(const Read &read) {
    if constexpr (F < NF) {
        if constexpr (slot_of(F, NF, R0, R1) == I) read(std::integral_constant<int, F>{});
        read_slot<F + 1, NF, I, R0, R1>(read);
    }
}

// MFMAs [I, I1) of a substep; `read(F)` of the next substep's FM + FN
// fragments spread over slots [R0, R1), `load(j)` of LC loads over [D0, D1).
template <int I, int I1, int R0, int R1, int LC, int D0, int D1, int FM, int FN, class Read, class Load>
__device__ __forceinline__ void mfma_run(f32x4 (&acc)[FN][FM], const bf16x8 (&a)[FM], const bf16x8 (&b)[FN],
                                         const Read &read, const Load &load) {
    if constexpr (I < I1) {
        constexpr int NI = I / FM, MI = slot_row<FM>(I);
        acc[NI][MI] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b[NI], a[MI], acc[NI][MI], 0, 0, 0);
        read_slot<0, FM + FN, I, R0, R1>(read);
#pragma unroll
        for (int j = 0; j < LC; ++j)
            if (slot_of(j, LC, D0, D1) == I) load(j);
        __builtin_amdgcn_sched_barrier(0);
        mfma_run<I + 1, I1, R0, R1, LC, D0, D1, FM, FN>(acc, a, b, read, load);
    }
}

// Over the four lanes that hold a row: the wave's 16-lane rows exchanged.
__device__ __forceinline__ void row_pairs(float x, bool far, float *a, float *b) {
    const uint32_t u = __builtin_bit_cast(uint32_t, x);
    const u32x2 r = far ? __builtin_amdgcn_permlane32_swap(u, u, false, false)
                        : __builtin_amdgcn_permlane16_swap(u, u, false, false);
    *a = __builtin_bit_cast(float, (uint32_t)r[0]);
    *b = __builtin_bit_cast(float, (uint32_t)r[1]);
}
__device__ __forceinline__ float row_max(float x) {
    float a, b;
    row_pairs(x, false, &a, &b);
    row_pairs(fmaxf(a, b), true, &a, &b);
    return fmaxf(a, b);
}
__device__ __forceinline__ float row_sum(float x) {
    float a, b;
    row_pairs(x, false, &a, &b);
    row_pairs(a + b, true, &a, &b);
    return a + b;
}

// The largest |grad| of a row with a target (1 without any). dz is stored as
// its multiple, and the products are scaled back in fp32: with one weight for
// all rows, as in a mean, the multiple is exactly 1, and -1 at the targets'
// columns is exact where grad itself would round by the same 2^-9 or so in
// every row (8192 x 50257 x 4096, mean loss: dH and dW off by 2.6e-3 of their norm,
// with it 1.9e-3; 1.7e-3 is their own rounding to bf16).
__device__ __forceinline__ float peak_of(float largest) {
    return largest > 0.0f && largest < INFINITY ? largest : 1.0f;
}
__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
    for (int d = 1; d < 64; d *= 2) x = fmaxf(x, __shfl_xor(x, d));
    return x;
}
// Up to so many rows dz's own workgroups find it (and leave it to the products),
// more take a launch (backward, found here: 1 x 2000 x 1024 21.6 -> 20.2 us,
// 250 x 20000 x 1024 63.3 -> 63.5).
constexpr int kOwnPeakRows = 256;

// BM x BN tiles, 4 waves, 2 x 2 over the tile. The main loop (stages of 64,
// DW + 1 buffers of A and DW of B, counted waits, one barrier per stage, LDS
// reads and loads one at a time between the MFMAs) is gemm_kernel's; see there
// for what each part of it is worth. A workgroup takes a tile of every round;
// with kPre the next tile's first stages are on their way while the epilogue
// runs (the epilogue's LDS is then the buffer that those stages leave free).
//
// What bounds it: the large tiles, the matrix cores at the clock the chip's
// power allows, 1.35 to 1.45 PFLOP/s (8192 x 50257 x 4096 forward 2.33 to 2.37 ms, its
// backward 7.3 to 7.6 ms from card to card; MFMA busy 0.66 to 0.74), and what a
// tile's edges cost beside its stages: 8192 x 50257 x 1024 forward went from 985 us
// with a workgroup per tile to 915 with the next tile's loads under the epilogue
// (799 now). Few rows: W from memory, 8 x 32000 x 4096 44 to 51 us (5.2 to 6.0 TB/s;
// 38 on the same W again).
template <int BM, int BN, int DW, bool AT, bool BT, int EPI>
__global__ __launch_bounds__(kThreads, (160 << 10) / (((DW + 1) * BM + DW * BN) * 128))
void tile_kernel(const TileParams p) {
    constexpr int WM = BM / 2, WN = BN / 2;
    constexpr int FM = WM / 16, FN = WN / 16;
    constexpr int LA = BM / 32, LW = BN / 32;
    constexpr int SA = BM * 128, SW = BN * 128;
    constexpr int NA = DW + 1;
    constexpr bool kAcc = NA * SA + DW * SW > (80 << 10);   // one workgroup per CU
    constexpr int kRegion = EPI == kStats ? 0 : FN * (EPI == kPart ? 2048 : 1024);   // bytes per wave, 32 rows
    constexpr bool kPre = 4 * kRegion <= SA;
    __shared__ __attribute__((aligned(1024))) char smem[NA * SA + DW * SW];
    static_assert(4 * kRegion <= NA * SA + DW * SW, "the epilogue regions fit");

    const int tid = threadIdx.x;
    const int lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm0 = (wave >> 1) * WM, wn0 = (wave & 1) * WN;
    const int tiles = p.tiles_m * p.tiles_n, total = tiles * p.slices, grid = (int)gridDim.x;
    const uint32_t lds0 = (uint32_t)(uintptr_t)LDS_AS(smem);
    const uint32_t ldsW = lds0 + NA * SA, ldsE = ldsW + DW * SW;

    // Tile of this workgroup in round j, false when there is none. Positions go
    // down group_m row tiles before the next column tile: what an XCD holds at a
    // time shares rows and columns in its L2, and the XCDs, at different rows, go
    // over the same columns together (8192 x 50257 x 4096 forward 2915 us where
    // all XCDs are at the same rows, 2472 so).
    struct Tile { int m0, n0, tn, slice, kb, ke; };
    auto tile_of_round = [&](int j, Tile &t) {
        const int pos = round_position(total, grid, (int)blockIdx.x, j);
        if (pos < 0) return false;
        t.slice = pos / tiles;
        const int tpos = pos - t.slice * tiles, gsz = p.group_m * p.tiles_n;
        const int grp = tpos / gsz, rin = tpos - grp * gsz;
        const int rows_here = min(p.group_m, p.tiles_m - grp * p.group_m);
        t.tn = rin / rows_here;
        t.m0 = p.m_base + (grp * p.group_m + rin - t.tn * rows_here) * BM;
        t.n0 = p.n_base + t.tn * BN;
        t.kb = t.slice * p.kslice;
        t.ke = min(p.R, t.kb + p.kslice);
        return true;
    };

    Loader<AT, BM> la;
    Loader<BT, BN> lb;
    // The lane's number, not known to the compiler to be the same at every call:
    // what is derived from it is computed where it is needed, not kept in
    // registers (and spilled) from one tile to the next.
    auto fresh_lane = [&]() {
        int l = lane;
        asm volatile("" : "+v"(l));
        return l;
    };
    auto begin = [&](const Tile &t) {   // the tile's first DW stages
        const int l = fresh_lane();
        la.init(p.A, p.a_bytes, t.m0, p.M, p.lda, t.kb, t.ke, l, wave);
        lb.init(p.B, p.b_bytes, t.n0, p.N, p.ldb, t.kb, t.ke, l, wave);
        i32x4 r;
#pragma unroll
        for (int i = 0; i < DW; ++i) {
            uint32_t o = la.next(r);
            load_blocks<LA>(r, lds0 + i * SA, la.off, o, wave);
            o = lb.next(r);
            load_blocks<LW>(r, ldsW + i * SW, lb.off, o, wave);
        }
    };

    Tile cur, nxt;
    if (!tile_of_round(0, nxt)) return;
    begin(nxt);
    // (one value for all lanes, here for good: left to the epilogues, its load
    // has the compiler wait for every load in flight inside the main loop)
    float peak = 1.0f;
    if constexpr (EPI == kDz) {
        if (p.M <= kOwnPeakRows) {   // every wave for itself
            float x = 0.0f;
#pragma unroll
            for (int m = lane; m < kOwnPeakRows; m += 64)
                if (m < p.M) x = fmaxf(x, p.target[m] >= 0 ? fabsf(p.grad[m]) : 0.0f);
            peak = peak_of(wave_max(x));
            if (blockIdx.x == 0 && tid == 0) *p.peak = peak;
        }
    }
    if (EPI != kStats && !(EPI == kDz && p.M <= kOwnPeakRows)) peak = *p.peak;
    if constexpr (EPI != kStats)
        peak = __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, peak)));
    for (int round = 1;; ++round) {
        cur = nxt;
        f32x4 acc[FN][FM];
#pragma unroll
        for (int ni = 0; ni < FN; ++ni)
#pragma unroll
            for (int mi = 0; mi < FM; ++mi) acc[ni][mi] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        {
            Reader<AT, BM, FM> ra;
            Reader<BT, BN, FN> rb;
            const int l = fresh_lane();
            ra.init(wm0, l);
            rb.init(wn0, l);
            const int KT = (cur.ke - cur.kb + kBK - 1) / kBK;
            const uint32_t wb = (uint32_t)wave * 1024u;
            // (stores of the tile before count too, and need not return in order
            // with these loads: all of both; by the builtin, for the compiler then
            // knows that nothing of the epilogue is in flight and puts no wait of
            // its own into the loop)
            if (kPre && round > 1) __builtin_amdgcn_s_waitcnt(0);
            else wait_vm_lgkm0<(DW - 1) * (LA + LW)>();
            lds_barrier();
            bf16x8 a0[FM], b0[FN], a1[FM], b1[FN];
#pragma unroll
            for (int mi = 0; mi < FM; ++mi) a0[mi] = ra.template read<0>(lds0, mi);
#pragma unroll
            for (int ni = 0; ni < FN; ++ni) b0[ni] = rb.template read<0>(ldsW, ni);
            constexpr int NM = FM * FN;
            constexpr int RE = NM - NM / 4;     // substep 0's reads end here, ahead of the barrier's wait
            constexpr int B1 = NM / 16;         // MFMAs of substep 1 before the barrier
            i32x4 sA, sB;
            // fragments in the order an MFMA substep needs them: b[0], a[..], b[1..]
            uint32_t aC = lds0, aF = lds0 + DW * SA, wC = ldsW;
            if constexpr (kAcc) {
                // Every accumulator in a register of its own from before the loop,
                // then around it: from the constant zero the compiler rotates them
                // (364 to 604 moves per stage and spills).
#pragma unroll
                for (int i = 0; i < NM; ++i) asm volatile("" : "+a"(acc[i / FM][slot_row<FM>(i)]));
            }
            for (int st = 0; st < KT; ++st) {
                const uint32_t aN = aC + SA == ldsW ? lds0 : aC + SA, wN = wC + SW == ldsE ? ldsW : wC + SW;
                if constexpr (kAcc) {
#pragma unroll
                    for (int i = 0; i < NM; ++i) asm volatile("" : "+a"(acc[i / FM][slot_row<FM>(i)]));
                }
                const uint32_t oA = la.next(sA), oB = lb.next(sB);
                auto read1 = [&](auto fc) __attribute__((always_inline)) {
                    constexpr int f = decltype(fc)::value;
                    if constexpr (f >= 1 && f <= FM) a1[f - 1] = ra.template read<1>(aC, f - 1);
                    else b1[f == 0 ? 0 : f - FM] = rb.template read<1>(wC, f == 0 ? 0 : f - FM);
                };
                auto read0 = [&](auto fc) __attribute__((always_inline)) {
                    constexpr int f = decltype(fc)::value;
                    if constexpr (f >= 1 && f <= FM) a0[f - 1] = ra.template read<0>(aN, f - 1);
                    else b0[f == 0 ? 0 : f - FM] = rb.template read<0>(wN, f == 0 ? 0 : f - FM);
                };
                auto loadA = [&](int j) { dma16(sA, la.off[j] + oA, aF + wb + (uint32_t)j * 4096u); };
                auto loadB = [&](int j) { dma16(sB, lb.off[j] + oB, wC + wb + (uint32_t)j * 4096u); };
                mfma_run<0, NM, 0, RE, LA, 0, NM, FM, FN>(acc, a0, b0, read1, loadA);
                mfma_run<0, B1, NM, NM + 1, 0, 0, 1, FM, FN>(acc, a1, b1, read0, loadA);
                wait_vm_lgkm0<(DW - 1) * LA + (DW - 2) * LW>();
                lds_barrier();
                mfma_run<B1, NM, B1, NM, LW, B1, B1 + (NM - B1) * 3 / 4, FM, FN>(acc, a1, b1, read0, loadB);
                aF = aC;
                aC = aN;
                wC = wN;
            }
            wait_vm_lgkm0<0>();   // the loads past the end land before the buffers are reused
            __syncthreads();
        }
        const bool more = tile_of_round(round, nxt);
        if (kPre && more) begin(nxt);

        const int et = fresh_lane();
        // lane (er, eq) holds of block (mi, ni): row er, columns 4 eq + 0..3
        const int er = et & 15, eq = et >> 4;
        const int m1 = cur.m0 + wm0, n1 = cur.n0 + wn0;   // of this wave
        const int c0 = n1 + 4 * eq;
        const bool edge = cur.n0 + BN > p.N;
        char *const region = smem + (kPre ? DW * SA : 0) + wave * kRegion;
        // A row of blocks stays in the accumulators until its turn: the compiler
        // would else copy all of them to vector registers here, and spill (the
        // statistics of 256 x 256 tiles: 43 registers, 34 MB written where now 3
        // are, 8192 x 6283 x 12288 924 -> 916 us).
        auto hold = [&](int mi) {
            if constexpr (kAcc) {
#pragma unroll
                for (int ni = 0; ni < FN; ++ni) asm volatile("" : "+a"(acc[ni][mi]));
            }
        };
        if constexpr (EPI == kStats) {
            // each half's maximum as it is and its sum relative to it: the largest
            // column's exponential is exactly 1, so that a sum is at least 1 and a
            // row's lse never below its largest logit. (In units of log 2 an
            // exponential is one operation less, but lse came back rounded twice at
            // the logit's size, and certain rows had losses below 0. What it costs:
            // 4096 x 32000 x 512 148 -> 150 us, 8192 x 50257 x 1024 792 -> 799.)
            float2 *out = p.parts + (size_t)(2 * cur.tn + (wave & 1)) * (size_t)p.M;
            const int inside = p.N - c0;   // columns from this lane's first on
#pragma unroll
            for (int mi = 0; mi < FM; ++mi) {
                const int m = m1 + mi * 16 + er;
                float z[FN][4], mx = -INFINITY;
                hold(mi);
#pragma unroll
                for (int ni = 0; ni < FN; ++ni)
#pragma unroll
                    for (int e = 0; e < 4; ++e) z[ni][e] = acc[ni][mi][e];
                if (edge) {
#pragma unroll
                    for (int ni = 0; ni < FN; ++ni)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (ni * 16 + e >= inside) z[ni][e] = -INFINITY;
                }
#pragma unroll
                for (int ni = 0; ni < FN; ++ni)
#pragma unroll
                    for (int e = 0; e < 4; ++e) mx = fmaxf(mx, z[ni][e]);
                mx = row_max(mx);
                const float sub = mx == -INFINITY ? 0.0f : mx;   // no column of this half is inside
                float sum = 0.0f;
#pragma unroll
                for (int ni = 0; ni < FN; ++ni)
#pragma unroll
                    for (int e = 0; e < 4; ++e) sum += __builtin_amdgcn_exp2f((z[ni][e] - sub) * kLog2e);
                sum = row_sum(sum);
                int t = -1;   // the target's place from this lane's first column
                if (m < p.M) {
                    if (eq == 0) out[m] = make_float2(mx, sum);
                    const int64_t id = p.target[m], at = id < p.v0 ? -1 : id - p.v0 - c0;   // (no difference wraps)
                    if (at >= 0 && at < WN && at < inside) t = (int)at;
                }
                if (__ballot(t >= 0)) {   // (a few per cent of the blocks hold a target)
                    float tz = 0.0f;
                    bool mine = false;
#pragma unroll
                    for (int ni = 0; ni < FN; ++ni)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (t == ni * 16 + e) tz = z[ni][e], mine = true;
                    if (mine) p.tlogit[m] = tz;
                }
                __builtin_amdgcn_sched_barrier(0);   // (rows of blocks started together spill)
            }
        } else if constexpr (EPI == kPart) {
            // Each wave turns 32 rows at a time to row order through its region and
            // stores whole rows of its columns, 32 bytes per lane; 16-byte chunk c
            // of row r at chunk c ^ (r & 7). The region is the wave's own and its
            // LDS operations run in order: nothing waits between a write and its
            // read.
            constexpr int CPR = 2 * FN, NIT = 32 * CPR / 64, RB = FN * 64;
#pragma unroll
            for (int mi = 0; mi < FM / 2; ++mi) {
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int ni = 0; ni < FN; ++ni)
                        *reinterpret_cast<f32x4 *>(region + (er + h * 16) * RB + (((4 * ni + eq) ^ (er & 7)) << 4)) =
                            acc[ni][2 * mi + h];
                asm volatile("" ::: "memory");
#pragma unroll
                for (int it = 0; it < NIT; ++it) {
                    const int row = (it * 64 + et) / CPR, j = (it * 64 + et) % CPR;
                    const char *w = region + row * RB;
                    // half of the lanes take their two chunks in the other order,
                    // so that 8 lanes read 8 different bank groups
                    const int sw = (j >> 2) & 1;
                    const f32x4 u0 = *reinterpret_cast<const f32x4 *>(w + (((2 * j + sw) ^ (row & 7)) << 4));
                    const f32x4 u1 = *reinterpret_cast<const f32x4 *>(w + (((2 * j + 1 - sw) ^ (row & 7)) << 4));
                    f32x4 x0, x1;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        x0[e] = peak * (sw ? u1[e] : u0[e]);
                        x1[e] = peak * (sw ? u0[e] : u1[e]);
                    }
                    const int m = m1 + mi * 32 + row, n = n1 + j * 8;
                    if (m < p.M && n < p.N) {   // N is a multiple of 8
                        const size_t at = ((size_t)cur.slice * (size_t)p.M + (size_t)m) * (size_t)p.N + n;
                        if (p.part_in) {
                            x0 += *reinterpret_cast<const f32x4 *>(p.part_in + at);
                            x1 += *reinterpret_cast<const f32x4 *>(p.part_in + at + 4);
                        }
                        if (p.part_out) {
                            *reinterpret_cast<f32x4 *>(p.part_out + at) = x0;
                            *reinterpret_cast<f32x4 *>(p.part_out + at + 4) = x1;
                        } else {
                            *reinterpret_cast<u32x4 *>(p.C + (size_t)m * (size_t)p.N + n) =
                                u32x4{pack_bf16x2(x0[0], x0[1]), pack_bf16x2(x0[2], x0[3]), pack_bf16x2(x1[0], x1[1]),
                                      pack_bf16x2(x1[2], x1[3])};
                        }
                    }
                }
                asm volatile("" ::: "memory");
            }
        } else {
            // The same, rounded to bf16 in the accumulators' layout, so that half
            // the bytes go through LDS: chunk c of row r at chunk c ^ (r & SWZ).
            constexpr int CPR = 2 * FN, RB = FN * 32, SWZ = CPR % 8 == 0 ? 7 : 3;
            // dz: the rows' weights and statistics, all loaded at once
            float lse[EPI == kDz ? FM : 1], g[EPI == kDz ? FM : 1];
            int t[EPI == kDz ? FM : 1];   // the target's place from this lane's first column, or -1
            if constexpr (EPI == kDz) {
#pragma unroll
                for (int mi = 0; mi < FM; ++mi) {
                    const int m = min(m1 + mi * 16 + er, p.M - 1);
                    const int64_t id = p.target[m], at = id < p.v0 ? -1 : id - p.v0 - c0;
                    lse[mi] = p.lse[m];
                    g[mi] = id < 0 ? 0.0f : p.grad[m] / peak;
                    t[mi] = at < 0 || at >= WN ? -1 : (int)at;
                }
            }
            uint16_t *out = EPI == kDz ? p.dz : p.C;
            const int ld = EPI == kDz ? p.ldz : p.N;
#pragma unroll
            for (int mi2 = 0; mi2 < FM / 2; ++mi2) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int mi = 2 * mi2 + h;
                    char *w = region + (er + h * 16) * RB + 8 * (eq & 1);
                    f32x4 x[FN];
                    hold(mi);
#pragma unroll
                    for (int ni = 0; ni < FN; ++ni) {
                        x[ni] = acc[ni][mi];
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            if constexpr (EPI == kDz) {
                                // (1 where the logit is all of lse: an lse in units of
                                // log 2 is off by its rounding, and so was 1 - pr)
                                const float pr = __builtin_amdgcn_exp2f((x[ni][e] - lse[mi]) * kLog2e);
                                x[ni][e] = g[mi] == 0.0f ? 0.0f : g[mi] * pr;   // (0 whatever the logits are)
                            } else {
                                x[ni][e] *= peak;
                            }
                        }
                    }
                    if constexpr (EPI == kDz) {
                        if (__ballot(t[mi] >= 0)) {   // (a few per cent of the blocks hold a target)
#pragma unroll
                            for (int ni = 0; ni < FN; ++ni)
#pragma unroll
                                for (int e = 0; e < 4; ++e)
                                    if (t[mi] == ni * 16 + e) x[ni][e] -= g[mi];
                        }
                        if (edge) {
#pragma unroll
                            for (int ni = 0; ni < FN; ++ni)
#pragma unroll
                                for (int e = 0; e < 4; ++e)
                                    if (c0 + ni * 16 + e >= p.N) x[ni][e] = 0.0f;
                        }
                    }
#pragma unroll
                    for (int ni = 0; ni < FN; ++ni)
                        *reinterpret_cast<u32x2 *>(w + (((2 * ni + (eq >> 1)) ^ (er & SWZ)) << 4)) =
                            u32x2{pack_bf16x2(x[ni][0], x[ni][1]), pack_bf16x2(x[ni][2], x[ni][3])};
                    __builtin_amdgcn_sched_barrier(0);   // (rows of blocks started together spill)
                }
                asm volatile("" ::: "memory");
#pragma unroll
                for (int it = 0; it < FN; ++it) {
                    const int row = (it * 64 + et) / CPR, j = (it * 64 + et) % CPR;
                    const u32x4 o = *reinterpret_cast<const u32x4 *>(region + row * RB + ((j ^ (row & SWZ)) << 4));
                    const int m = m1 + mi2 * 32 + row, n = n1 + j * 8;
                    u32x4 *to = reinterpret_cast<u32x4 *>(out + (size_t)m * (size_t)ld + n);
                    if (m < p.M && n < ld) {
                        if constexpr (EPI == kStream) __builtin_nontemporal_store(o, to);
                        else *to = o;
                    }
                }
                asm volatile("" ::: "memory");
            }
        }
        if (!more) return;
        if (!kPre) {
            __builtin_amdgcn_s_waitcnt(0);
            __syncthreads();
            begin(nxt);
        }
    }
}

// peak_of all rows, in one workgroup.
__global__ __launch_bounds__(1024) void peak_kernel(int M, const int64_t *target, const float *grad, float *peak) {
    __shared__ float s[16];
    float x = 0.0f;
#pragma unroll 8
    for (int m = threadIdx.x; m < M; m += 1024) {
        const float g = fabsf(grad[m]);
        x = fmaxf(x, target[m] >= 0 ? g : 0.0f);
    }
    x = wave_max(x);
    if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = x;
    __syncthreads();
    if (threadIdx.x != 0) return;
#pragma unroll
    for (int i = 1; i < 16; ++i) x = fmaxf(x, s[i]);
    *peak = peak_of(x);
}

// Joins a row's parts: lse = max + log sum_i s_i exp(m_i - max). ROWS rows per
// workgroup, 256 / ROWS threads each: 16 rows read whole 128-byte lines of the
// parts; few rows (at most 256) take a workgroup each (8 rows of 1000 parts:
// 20.6 us with 16).
template <int ROWS>
__global__ __launch_bounds__(256) void stats_kernel(int M, int V, int parts, const float2 *__restrict__ part,
                                                    const int64_t *target, int64_t v0, float *lse, float *tlogit,
                                                    float *loss) {
    constexpr int Q = 256 / ROWS;
    __shared__ float2 s_part[Q][ROWS];
    const int r = threadIdx.x % ROWS, q = threadIdx.x / ROWS;
    const int m = (int)blockIdx.x * ROWS + r;
    float mx = -INFINITY, sum = 0.0f;
    auto add = [&](float2 x) {
        const float top = fmaxf(mx, x.x), sub = top == -INFINITY ? 0.0f : top;
        sum = sum * __builtin_amdgcn_exp2f((mx - sub) * kLog2e) + x.y * __builtin_amdgcn_exp2f((x.x - sub) * kLog2e);
        mx = top;
    };
    if (m < M) {
#pragma unroll 4
        for (int i = q; i < parts; i += Q) add(part[(size_t)i * (size_t)M + m]);
    }
    s_part[q][r] = make_float2(mx, sum);
#pragma unroll
    for (int half = Q / 2; half > 0; half /= 2) {
        __syncthreads();
        if (q < half) {
            add(s_part[q + half][r]);
            s_part[q][r] = make_float2(mx, sum);
        }
    }
    if (q != 0 || m >= M) return;
    const float l = mx + logf(sum);
    const int64_t t = target[m];
    float tl = 0.0f;
    if (t >= v0 && t - v0 < V) tl = tlogit[m];
    else tlogit[m] = 0.0f;
    lse[m] = l;
    if (loss) loss[m] = t < 0 ? 0.0f : l - tl;
}

// The same over the n ranks' shards of the vocabulary.
__global__ __launch_bounds__(256) void join_ranks_kernel(int n, int M, const float *__restrict__ lse_parts,
                                                         const float *__restrict__ tlogit_parts, const int64_t *target,
                                                         float *lse, float *loss) {
    const int m = (int)blockIdx.x * 256 + (int)threadIdx.x;
    if (m >= M) return;
    float mx = -INFINITY;
    for (int q = 0; q < n; ++q) mx = fmaxf(mx, lse_parts[(size_t)q * (size_t)M + m]);
    const float sub = mx == -INFINITY ? 0.0f : mx;
    float sum = 0.0f, tl = 0.0f;
    for (int q = 0; q < n; ++q) {
        sum += __builtin_amdgcn_exp2f((lse_parts[(size_t)q * (size_t)M + m] - sub) * kLog2e);
        tl += tlogit_parts[(size_t)q * (size_t)M + m];
    }
    const float l = sub + logf(sum);
    lse[m] = l;
    loss[m] = target[m] < 0 ? 0.0f : l - tl;
}

// out = bf16(sum of the slices in order), 4 values per thread.
__global__ __launch_bounds__(256) void join_slices_kernel(size_t count4, int slices, const f32x4 *__restrict__ part,
                                                          uint16_t *out) {
    const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= count4) return;
    f32x4 x = part[i];
#pragma unroll 8
    for (int s = 1; s < slices; ++s) x += part[(size_t)s * count4 + i];
    *reinterpret_cast<u32x2 *>(out + 4 * i) = u32x2{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3])};
}

// ------------------------------------------------------------------- plans

template <bool AT, bool BT, int EPI>
hipError_t launch_tiles(TileParams p, const TilePlan &pl, hipStream_t stream) {
    p.tiles_m = pl.tiles_m;
    p.tiles_n = pl.tiles_n;
    p.slices = pl.slices;
    p.kslice = pl.kslice;
    p.group_m = kTiles[pl.cfg].rows == 256 ? 4 : 8;
    const int64_t items = (int64_t)pl.tiles_m * pl.tiles_n * pl.slices;
    const dim3 grid((unsigned)std::min<int64_t>(items, kCUs * kTiles[pl.cfg].wg_per_cu));
    // (a template instance for each row of kTiles)
    switch (pl.cfg) {
    case 0: tile_kernel<256, 256, 2, AT, BT, EPI><<<grid, kThreads, 0, stream>>>(p); break;
    case 1: tile_kernel<256, 192, 2, AT, BT, EPI><<<grid, kThreads, 0, stream>>>(p); break;
    case 2: tile_kernel<256, 128, 2, AT, BT, EPI><<<grid, kThreads, 0, stream>>>(p); break;
    case 3: tile_kernel<192, 192, 2, AT, BT, EPI><<<grid, kThreads, 0, stream>>>(p); break;
    case 4: tile_kernel<128, 192, 3, AT, BT, EPI><<<grid, kThreads, 0, stream>>>(p); break;
    case 5: tile_kernel<128, 128, 2, AT, BT, EPI><<<grid, kThreads, 0, stream>>>(p); break;
    case 6: tile_kernel<128, 128, 4, AT, BT, EPI><<<grid, kThreads, 0, stream>>>(p); break;
    case 7: tile_kernel<128, 64, 4, AT, BT, EPI><<<grid, kThreads, 0, stream>>>(p); break;
    case 8: tile_kernel<64, 64, 4, AT, BT, EPI><<<grid, kThreads, 0, stream>>>(p); break;
    default: tile_kernel<64, 256, 3, AT, BT, EPI><<<grid, kThreads, 0, stream>>>(p); break;
    }
    return hipGetLastError();
}

// A product in the one or two launches of its plan.
template <bool AT, bool BT, int EPI>
hipError_t launch_pair(TileParams p, const PairPlan &pl, bool along_m, hipStream_t stream) {
    hipError_t e = launch_tiles<AT, BT, EPI>(p, pl.part[0], stream);
    if (e == hipSuccess && pl.part[1].tiles_m > 0) {
        (along_m ? p.m_base : p.n_base) = pl.first;
        p.parts += (size_t)2 * pl.part[0].tiles_n * (size_t)p.M;
        e = launch_tiles<AT, BT, EPI>(p, pl.part[1], stream);
    }
    return e;
}

int hip_error(hipError_t e, const char *what) {
    return set_error(COMPASS_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

size_t forward_bytes(const PairPlan &pl, int M) { return (size_t)stat_parts(pl) * (size_t)M * sizeof(float2); }

constexpr int kMaxRows = 1 << 20, kMaxVocab = 1 << 24, kMaxDepth = 1 << 17;

int check_sizes(int M, int V, int K) {
    if (M < 1 || V < 1 || K < 1 || K % 8)
        return set_error(COMPASS_ERR_INVALID, "need positive M, V and K with K a multiple of 8");
    if (M > kMaxRows || V > kMaxVocab || K > kMaxDepth)
        return set_error(COMPASS_ERR_UNSUPPORTED, "M = %d, V = %d, K = %d beyond %d, %d, %d", M, V, K, kMaxRows,
                         kMaxVocab, kMaxDepth);
    return COMPASS_OK;
}

// The kernels address a tile's rows of dz with 32-bit offsets from its first:
// the rows of a tile (at most 256) span at most kTileSpanMax bytes. The
// library's own pieces are within that.
int check_piece(int M, const BackwardPlan &b) {
    if ((uint64_t)std::min(M, 256) * (uint64_t)b.ldz * 2 > kTileSpanMax)
        return set_error(COMPASS_ERR_UNSUPPORTED, "pieces of %d columns: a tile's rows of dz would span more than 1 GiB",
                         b.pieces.cols);
    return COMPASS_OK;
}

bool misaligned(const void *p) { return ((uintptr_t)p & 15) != 0; }

}  // namespace

int op_xent_workspace(int M, int V, int K, int backward, int piece, size_t *bytes) {
    const int rc = check_sizes(M, V, K);
    if (rc != COMPASS_OK) return rc;
    if (!bytes || piece < 0) return set_error(COMPASS_ERR_INVALID, "bytes is required, piece must not be negative");
    if (backward) {
        const BackwardPlan b = plan_backward(M, V, K, piece);
        if (const int bad = check_piece(M, b)) return bad;
        *bytes = b.dz_bytes + b.part_bytes;
    } else {
        *bytes = forward_bytes(plan_pair(kLogits, K % 64 != 0, M, V, K, false), M);
    }
    return COMPASS_OK;
}

int op_xent_forward(int M, int V, int K, const void *H, const void *W, const int64_t *target, int64_t v0, float *lse,
                    float *tlogit, float *loss, void *ws, size_t ws_bytes, void *stream) {
    int rc = check_sizes(M, V, K);
    if (rc != COMPASS_OK) return rc;
    if (!H || !W || !target || !lse || !tlogit || !ws)
        return set_error(COMPASS_ERR_INVALID, "H, W, target, lse, tlogit and the workspace are required");
    if (misaligned(H) || misaligned(W) || misaligned(ws))
        return set_error(COMPASS_ERR_INVALID, "H, W and the workspace must be 16-byte aligned");
    if (v0 < 0 || v0 > INT64_MAX - V)
        return set_error(COMPASS_ERR_INVALID, "v0 must not be negative, v0 + V must fit 64 bits");
    const PairPlan pl = plan_pair(kLogits, K % 64 != 0, M, V, K, false);
    if (ws_bytes < forward_bytes(pl, M))
        return set_error(COMPASS_ERR_INVALID, "workspace of %zu bytes, need %zu", ws_bytes, forward_bytes(pl, M));
    int cus;
    if ((rc = current_num_cu(&cus)) != COMPASS_OK) return rc;
    TileParams p{};
    p.A = (const uint16_t *)H;
    p.B = (const uint16_t *)W;
    p.a_bytes = (uint64_t)M * (uint64_t)K * 2;
    p.b_bytes = (uint64_t)V * (uint64_t)K * 2;
    p.M = M;
    p.N = V;
    p.R = p.lda = p.ldb = K;
    p.parts = (float2 *)ws;
    p.tlogit = tlogit;
    p.target = target;
    p.v0 = v0;
    hipError_t e = launch_pair<false, false, kStats>(p, pl, false, (hipStream_t)stream);
    if (e != hipSuccess) return hip_error(e, "logits launch");
    if (M <= 256)
        stats_kernel<1><<<dim3((unsigned)M), 256, 0, (hipStream_t)stream>>>(M, V, stat_parts(pl), p.parts, target, v0,
                                                                            lse, tlogit, loss);
    else
        stats_kernel<16><<<dim3((unsigned)((M + 15) / 16)), 256, 0, (hipStream_t)stream>>>(
            M, V, stat_parts(pl), p.parts, target, v0, lse, tlogit, loss);
    e = hipGetLastError();
    return e == hipSuccess ? COMPASS_OK : hip_error(e, "statistics launch");
}

int op_xent_join(int n, int M, const float *lse_parts, const float *tlogit_parts, const int64_t *target, float *lse,
                 float *loss, void *stream) {
    if (n < 1 || M < 1) return set_error(COMPASS_ERR_INVALID, "need positive n and M");
    if (!lse_parts || !tlogit_parts || !target || !lse || !loss)
        return set_error(COMPASS_ERR_INVALID, "every operand is required");
    int cus;
    const int rc = current_num_cu(&cus);
    if (rc != COMPASS_OK) return rc;
    join_ranks_kernel<<<dim3((unsigned)((M + 255) / 256)), 256, 0, (hipStream_t)stream>>>(n, M, lse_parts, tlogit_parts,
                                                                                       target, lse, loss);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? COMPASS_OK : hip_error(e, "join launch");
}

int op_xent_backward(int M, int V, int K, const void *H, const void *W, const int64_t *target, int64_t v0,
                     const float *lse, const float *grad, void *dH, void *dW, int piece, void *ws, size_t ws_bytes,
                     void *stream) {
    int rc = check_sizes(M, V, K);
    if (rc != COMPASS_OK) return rc;
    if (!H || !W || !target || !lse || !grad || !dH || !dW || !ws)
        return set_error(COMPASS_ERR_INVALID, "every operand and the workspace are required");
    if (misaligned(H) || misaligned(W) || misaligned(dH) || misaligned(dW) || misaligned(ws))
        return set_error(COMPASS_ERR_INVALID, "H, W, dH, dW and the workspace must be 16-byte aligned");
    if (v0 < 0 || v0 > INT64_MAX - V || piece < 0)
        return set_error(COMPASS_ERR_INVALID, "v0 and piece must not be negative, v0 + V must fit 64 bits");
    const BackwardPlan b = plan_backward(M, V, K, piece);
    if ((rc = check_piece(M, b)) != COMPASS_OK) return rc;
    if (ws_bytes < b.dz_bytes + b.part_bytes)
        return set_error(COMPASS_ERR_INVALID, "workspace of %zu bytes, need %zu", ws_bytes, b.dz_bytes + b.part_bytes);
    int cus;
    if ((rc = current_num_cu(&cus)) != COMPASS_OK) return rc;
    const hipStream_t s = (hipStream_t)stream;
    uint16_t *dz = (uint16_t *)ws;
    float *peak = (float *)((char *)ws + b.dz_bytes - 256);
    float *part = (float *)((char *)ws + b.dz_bytes);
    if (M > kOwnPeakRows) {
        peak_kernel<<<1, 1024, 0, s>>>(M, target, grad, peak);
        if (const hipError_t e = hipGetLastError(); e != hipSuccess) return hip_error(e, "peak launch");
    }
    const uint64_t h_bytes = (uint64_t)M * (uint64_t)K * 2;
    const bool ragged = K % 64 != 0;
    for (int i = 0; i < b.pieces.count; ++i) {
        const int c0 = i * b.pieces.cols, cols = std::min(b.pieces.cols, V - c0);
        const uint16_t *Wp = (const uint16_t *)W + (size_t)c0 * (size_t)K;
        const uint64_t w_bytes = (uint64_t)cols * (uint64_t)K * 2;
        TileParams p{};
        p.A = (const uint16_t *)H;
        p.B = Wp;
        p.a_bytes = h_bytes;
        p.b_bytes = w_bytes;
        p.M = M;
        p.N = cols;
        p.R = p.lda = p.ldb = K;
        p.target = target;
        p.v0 = v0 + c0;
        p.lse = lse;
        p.grad = grad;
        p.peak = peak;
        p.dz = dz;
        p.ldz = dz_columns(cols);
        hipError_t e = launch_pair<false, false, kDz>(p, plan_pair(kGradLogits, ragged, M, p.ldz, K, false), false, s);
        if (e != hipSuccess) return hip_error(e, "dz launch");

        TileParams q{};
        q.A = dz;
        q.a_bytes = (uint64_t)M * (uint64_t)p.ldz * 2;
        q.lda = p.ldz;
        // dW's rows of this piece = dz^T H
        q.B = (const uint16_t *)H;
        q.b_bytes = h_bytes;
        q.M = cols;
        q.N = q.ldb = K;
        q.R = M;
        q.peak = peak;
        q.C = (uint16_t *)dW + (size_t)c0 * (size_t)K;
        // dW is not read again here: its stores pass through the caches. But with
        // few rows the stores are most of the work, and where rows do not start on
        // 128-byte lines the caches put the halves of a line together (30 x 100003 x
        // 1032 backward 229 -> 197 us, 16 x 50257 x 1032 110 -> 102; the other way
        // round 97 x 58829 x 912 105 -> 114, 16 x 32000 x 4096 171 -> 202)
        const PairPlan dw = plan_pair(kGradWeight, ragged, cols, K, M, true);
        e = ragged && M <= kBK ? launch_pair<true, true, kStore>(q, dw, true, s)
                               : launch_pair<true, true, kStream>(q, dw, true, s);
        if (e != hipSuccess) return hip_error(e, "dW launch");
        // dH += dz W over this piece
        q.B = Wp;
        q.b_bytes = w_bytes;
        q.M = M;
        q.R = p.ldz;
        q.C = (uint16_t *)dH;
        q.part_in = i > 0 ? part : nullptr;
        // the last piece of an unsplit sum leaves rounded
        q.part_out = b.dh.slices > 1 || i + 1 < b.pieces.count ? part : nullptr;
        // (a narrower last piece keeps the slice count, so that it adds to the
        // same partial sums; slices that start past its end add nothing)
        TilePlan pl = b.dh;
        const int stages = p.ldz / kBK;
        pl.kslice = (stages + pl.slices - 1) / pl.slices * kBK;
        e = q.part_in || q.part_out ? launch_tiles<false, true, kPart>(q, pl, s)
                                    : launch_tiles<false, true, kStore>(q, pl, s);
        if (e != hipSuccess) return hip_error(e, "dH launch");
    }
    if (b.dh.slices > 1) {
        const size_t count4 = (size_t)M * (size_t)K / 4;
        join_slices_kernel<<<dim3((unsigned)((count4 + 255) / 256)), 256, 0, s>>>(count4, b.dh.slices, (const f32x4 *)part,
                                                                               (uint16_t *)dH);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return hip_error(e, "dH join launch");
    }
    return COMPASS_OK;
}

}  // namespace compass
