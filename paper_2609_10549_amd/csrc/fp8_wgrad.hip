// A weight's gradient from an activation kept in 8-bit rows (fp8.h; compass_fp8_wgrad):
//
//   dW[n][k] = sum_m dY[m][n] X[m][k] 2^sx[m][k / 128]
//
// One bf16 product over rows that lie across the reduction in both operands. X's
// values become bf16 on their way to LDS, where a row's group still shares a scale:
// four significant bits and a power of two, nothing is rounded.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "compass.h"
#include "fp8.h"
#include "fp8_plan.h"
#include "gemm_core.h"
#include "gemm_cross.h"
#include "internal.h"

namespace compass {

namespace {

struct GradParams {
    const uint16_t *dY;
    const uint8_t *X, *sX;
    void *dW;
    float *part;                 // split: fp32 [slices][part_rows][part_ld], from the first tile on
    int part_rows, part_ld;
    int M, N, K, S;              // S: bytes of a row of scales
    int f32, accumulate;         // dW in fp32 (else bf16); added to what it holds
    int tiles_n, tiles_k, group_n;
    int n_base, k_base;          // the first tile's row and column
    int slices, mslice;          // slices of the reduction (mslice a multiple of 64)
};

template <int I, int I1, class Step>
__device__ __forceinline__ void each_slot(const Step &step) {
    if constexpr (I < I1) {
        step(std::integral_constant<int, I>{});
        each_slot<I + 1, I1>(step);
    }
}

// 64 rows of BK columns of X per stage: 16 values of a row per thread and turn,
// loaded to registers a stage ahead, then put to bf16 and to LDS as Reader<true>
// expects them.
template <int BK>
struct XStage {
    static constexpr int J = BK / 64, RB = BK * 2, CPR = BK / 16;   // turns, bytes of an LDS row, chunks of a row
    static constexpr int STEP = 256 / CPR;                          // rows between a thread's turns
    static_assert(STEP % 16 == 0, "the same place in the chunks' permutation");
    struct Piece { u32x4 v[J]; uint32_t s[J]; };
    uint32_t off[J], soff[J], at[2];
    bool odd;                   // the lane's halves go out in the other order
    const uint8_t *x, *sx;      // the next stage's first row, at the tile's first column and group
    int left;                   // rows from there to the last
    __device__ __forceinline__ void init(const GradParams &p, int k0, int mb, int tid) {
        x = p.X + (uint64_t)mb * (uint64_t)p.K + (uint64_t)k0;
        sx = p.sX + (uint64_t)mb * (uint64_t)p.S + (uint64_t)(k0 / kGroup);
        left = p.M - mb;
        const int row = tid / CPR, c = tid % CPR;
#pragma unroll
        for (int j = 0; j < J; ++j) {
            off[j] = (uint32_t)(row + j * STEP) * (uint32_t)p.K + (uint32_t)c * 16u;
            soff[j] = (uint32_t)(row + j * STEP) * (uint32_t)p.S + (uint32_t)groups_from(k0, c * 16);
        }
        // 4 neighbouring lanes' first halves lie in every other chunk: the next 4 lanes
        // write their second ones with them, so that the 8 lanes that LDS takes at a
        // time meet all banks
        odd = (tid >> 2) & 1;
#pragma unroll
        for (int h = 0; h < 2; ++h) at[h] = (uint32_t)(row * RB + (((2 * c + (odd ? 1 - h : h)) ^ cross_swizzle<RB>(row)) << 4));
    }
    // Rows behind the last are zeros under the smallest scale, whatever dY's rows there are.
    __device__ __forceinline__ void load(const GradParams &p, int k0, Piece &t, int j) const {
        const int rows = min(left, 128);   // (a stage reads 64, of its last one past the row's end)
        const __amdgpu_buffer_rsrc_t rx =
            __builtin_amdgcn_make_buffer_rsrc((void *)x, (short)0, max(rows * p.K - k0, 0), 0x00020000);
        const __amdgpu_buffer_rsrc_t rs =
            __builtin_amdgcn_make_buffer_rsrc((void *)sx, (short)0, max(rows * p.S - k0 / kGroup, 0), 0x00020000);
        t.v[j] = __builtin_amdgcn_raw_buffer_load_b128(rx, (int)off[j], 0, 0);
        t.s[j] = __builtin_amdgcn_raw_buffer_load_b8(rs, (int)soff[j], 0, 0);
    }
    __device__ __forceinline__ void next(const GradParams &p) {
        x += (int64_t)64 * p.K;
        sx += (int64_t)64 * p.S;
        left -= 64;
    }
    // half h (8 values; of the lanes that are odd the other one) of turn j to the stage
    // at LDS offset buf
    __device__ __forceinline__ void put(const Piece &t, int j, int h, uint32_t buf) const {
        // (the conversion takes the scale's exponent field, which is the byte; 255 is NaN there too)
        const float scale = __builtin_bit_cast(float, t.s[j] << 23 | (t.s[j] == 255u ? 1u << 22 : 0u));
        u32x4 o;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const uint32_t mine = t.v[j][2 * h + e], other = t.v[j][2 - 2 * h + e];
            const uint32_t w = odd ? other : mine;
            o[2 * e] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, false));
            o[2 * e + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, true));
        }
        typedef __attribute__((address_space(3))) u32x4 lds16;
        ((lds16 *)(uintptr_t)(buf + at[h]))[j * STEP * RB / 16] = o;
    }
    // t holds a whole stage from here on: the compiler waits here
    __device__ __forceinline__ static void arrived(Piece &t) {
#pragma unroll
        for (int j = 0; j < J; ++j) asm volatile("" : "+v"(t.v[j]), "+v"(t.s[j]));
    }
};

// Block f of substep S of the stage at LDS offset buf, as Reader<true>::read.
template <int S, int RB, class R>
__device__ __forceinline__ bf16x8 fragment(const R &r, uint32_t buf, int f) {
    typedef __attribute__((address_space(3))) s16x4 lds4;
    lds4 *q = (lds4 *)(uintptr_t)(buf + r.at[f]) + S * 4 * RB;
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(q);
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(q + RB / 2);
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}

// BN x BK tiles of dW, 4 waves, 2 x 2 over the tile, two stage buffers (64 of the
// reduction) of each operand, one barrier per stage: behind it the stage is in
// registers, and its buffers take dY's stage after the next one by loads that go to
// LDS, X's from the registers where it has been on its way for a stage.
//
// What bounds it: the large tiles, the transposed reads and the matrix cores at the
// clock that the power allows, 1.25 to 1.35 PFLOP/s in whole rounds (8192 x 4096 x 4096
// 203 to 219 us from card to card), and what X costs beside them, 0.2 of the time
// (without its conversion and loads 0.8; a conversion is a slow operation). 8192 x 6144 x
// 12288 973 to 1035 us: 4.5 rounds of 256 x 256 tiles, three of them and three of 256 x
// 128; added to what dW holds, which the epilogue reads as it stores, 85 to 95 us more. Few
// rows: dW's stores, 64 x 6144 x 12288 45 us (3.4 TB/s). Between them latency: 777 x 5000 x
// 1552 30 us (added to dW 32), two rounds of 13 stages, each of which waits for loads that
// are less than a stage old. What did not help: conversions over
// three quarters of a stage in place of a half, the barrier later, three or four
// workgroups of the small tiles per CU in place of two and three (26.9 -> 28.8), 64 x 128
// tiles for 128 x 64 (31), 192 x 256 tiles (1011).
template <int BN, int BK, int WGS>
__global__ __launch_bounds__(kThreads, WGS) void grad_kernel(const GradParams p) {
    constexpr int FN = BN / 32, FK = BK / 32, NM = FN * FK;   // blocks of 16 x 16 of a wave
    constexpr int LD = BN / 32;                               // loads of dY per wave and stage
    constexpr int SD = BN * 128, SX = BK * 128;
    constexpr int REGION = 16 * FK * 64;                      // epilogue: 16 rows of fp32 per wave
    constexpr int EPI = 2 * (SD + SX), LDS = EPI + 4 * REGION;
    constexpr bool kAcc = WGS == 1;
    constexpr int B1 = NM / 16;                               // MFMAs of the second half before the barrier
    static_assert(LDS * WGS <= (160 << 10), "LDS");
    __shared__ __attribute__((aligned(1024))) char smem[LDS];

    const int tid = threadIdx.x;
    const int lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wn0 = (wave >> 1) * (BN / 2), wk0 = (wave & 1) * (BK / 2);
    const int tiles = p.tiles_n * p.tiles_k, total = tiles * p.slices, grid = (int)gridDim.x;
    const uint32_t lds0 = (uint32_t)(uintptr_t)LDS_AS(smem), ldsX = lds0 + 2 * SD;

    struct Tile { int n0, k0, slice, mb, me; };
    auto tile_of_round = [&](int j, Tile &t) {
        const int pos = round_position(total, grid, (int)blockIdx.x, j);
        if (pos < 0) return false;
        t.slice = pos / tiles;
        const int tpos = pos - t.slice * tiles, gsz = p.group_n * p.tiles_k;
        const int grp = tpos / gsz, rin = tpos - grp * gsz;
        const int rows_here = min(p.group_n, p.tiles_n - grp * p.group_n);
        const int tk = rin / rows_here;
        t.n0 = p.n_base + (grp * p.group_n + rin - tk * rows_here) * BN;
        t.k0 = p.k_base + tk * BK;
        t.mb = t.slice * p.mslice;
        t.me = min(p.M, t.mb + p.mslice);
        return true;
    };
    auto fresh = [](int x) {   // as in the other tiled kernels: not kept in registers from tile to tile
        asm volatile("" : "+v"(x));
        return x;
    };

    Loader<true, BN> ld;
    XStage<BK> xs;
    auto load_dy = [&](int j, i32x4 r, uint32_t buf) __attribute__((always_inline)) {
        dma16(r, ld.off[j], buf + (uint32_t)((j * 4 + wave) * 1024));
    };
    typename XStage<BK>::Piece x0, x1;
    auto begin = [&](const Tile &t) {   // the loads of the first two stages
        const int id = fresh(tid);
        ld.init(p.dY, (uint64_t)p.M * (uint64_t)p.N * 2u, t.n0, p.N, p.N, t.mb, t.me, id & 63, wave);
        xs.init(p, t.k0, t.mb, id);
        i32x4 r;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            ld.next(r);
            asm volatile("s_nop 4" : "+s"(r));
#pragma unroll
            for (int j = 0; j < LD; ++j) load_dy(j, r, lds0 + i * SD);
        }
#pragma unroll
        for (int j = 0; j < xs.J; ++j) xs.load(p, t.k0, x0, j);
        xs.next(p);
#pragma unroll
        for (int j = 0; j < xs.J; ++j) xs.load(p, t.k0, x1, j);
        xs.next(p);
    };

    Tile cur, nxt;
    if (!tile_of_round(0, nxt)) return;
    begin(nxt);
    for (int round = 1;; ++round) {
        cur = nxt;
        f32x4 acc[FK][FN];
#pragma unroll
        for (int ki = 0; ki < FK; ++ki)
#pragma unroll
            for (int ni = 0; ni < FN; ++ni) acc[ki][ni] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        auto pin = [&]() __attribute__((always_inline)) {   // as in the 8-bit product
#pragma unroll
            for (int i = 0; i < NM; ++i) {
                if constexpr (kAcc) asm volatile("" : "+a"(acc[i / FN][i % FN]));
                else asm volatile("" : "+v"(acc[i / FN][i % FN]));
            }
        };
        {
            Reader<true, BN, FN> ra;
            Reader<true, BK, FK> rb;
            const int l = fresh(lane);
            ra.init(wn0, l);
            rb.init(wk0, l);
            const int MT = (cur.me - cur.mb + kBK - 1) / kBK;
#pragma unroll
            for (int h = 0; h < 2 * xs.J; ++h) xs.put(x0, h / 2, h % 2, ldsX);
#pragma unroll
            for (int h = 0; h < 2 * xs.J; ++h) xs.put(x1, h / 2, h % 2, ldsX + SX);
#pragma unroll
            for (int j = 0; j < xs.J; ++j) xs.load(p, cur.k0, x0, j);   // the third stage's
            xs.next(p);
            __builtin_amdgcn_s_waitcnt(0);
            lds_barrier();
            bf16x8 a0[FN], b0[FK], a1[FN], b1[FK];
#pragma unroll
            for (int f = 0; f < FN; ++f) a0[f] = fragment<0, 2 * BN>(ra, lds0, f);
#pragma unroll
            for (int f = 0; f < FK; ++f) b0[f] = fragment<0, 2 * BK>(rb, ldsX, f);
            uint32_t dC = lds0, xC = ldsX;
            i32x4 r;
            pin();
            for (int st = 0; st < MT; ++st) {
                pin();
                const uint32_t dN = dC == lds0 ? lds0 + SD : lds0, xN = xC == ldsX ? ldsX + SX : ldsX;
                // fragments in the order the MFMAs need them: b[0], a[..], b[1..]
                constexpr int RE = NM - NM / 4;
                each_slot<0, NM>([&](auto ic) __attribute__((always_inline)) {
                    constexpr int I = decltype(ic)::value, ki = I / FN, ni = slot_row<FN>(I);
                    acc[ki][ni] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b0[ki], a0[ni], acc[ki][ni], 0, 0, 0);
#pragma unroll
                    for (int f = 0; f < FN + FK; ++f)
                        if (slot_of(f, FN + FK, 0, RE) == I) {
                            if (f >= 1 && f <= FN) a1[f - 1] = fragment<1, 2 * BN>(ra, dC, f - 1);
                            else b1[f == 0 ? 0 : f - FN] = fragment<1, 2 * BK>(rb, xC, f == 0 ? 0 : f - FN);
                        }
                    __builtin_amdgcn_sched_barrier(0);
                });
                auto second = [&](auto ic) __attribute__((always_inline)) {
                    constexpr int I = decltype(ic)::value, ki = I / FN, ni = slot_row<FN>(I);
                    acc[ki][ni] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b1[ki], a1[ni], acc[ki][ni], 0, 0, 0);
                    if constexpr (I >= B1) {
#pragma unroll
                        for (int f = 0; f < FN + FK; ++f)
                            if (slot_of(f, FN + FK, B1, NM) == I) {
                                if (f >= 1 && f <= FN) a0[f - 1] = fragment<0, 2 * BN>(ra, dN, f - 1);
                                else b0[f == 0 ? 0 : f - FN] = fragment<0, 2 * BK>(rb, xN, f == 0 ? 0 : f - FN);
                            }
                        constexpr int XE = B1 + (NM - B1) / 2, DE = B1 + (NM - B1) * 3 / 4;
#pragma unroll
                        for (int h = 0; h < 2 * xs.J; ++h)
                            if (slot_of(h, 2 * xs.J, B1, XE) == I) {
                                xs.put(x0, h / 2, h % 2, xC);
                                if (h % 2 == 1) xs.load(p, cur.k0, x0, h / 2);
                            }
#pragma unroll
                        for (int j = 0; j < LD; ++j)
                            if (slot_of(j, LD, B1, DE) == I) load_dy(j, r, dC);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                };
                each_slot<0, B1>(second);
                pin();
                ld.next(r);
                // the next stage has landed, and this one is in registers: its buffers
                // take the stage after it
                wait_vm_lgkm0<0>();
                lds_barrier();
                xs.arrived(x0);
                each_slot<B1, NM>(second);
                xs.next(p);
                dC = dN;
                xC = xN;
            }
            wait_vm_lgkm0<0>();   // the loads past the end land before the buffers are reused
            __syncthreads();
        }
        const bool more = tile_of_round(round, nxt);
        if (more) begin(nxt);   // under the epilogue

        // Each wave turns 16 rows at a time to row order through LDS of its own and
        // stores whole rows of its columns, 8 values per lane; 16-byte chunk c of row r
        // at chunk c ^ (r & 7). Lane (er, eq) holds row er, columns 4 eq + 0..3 of a block.
        const int et = fresh(lane);
        const int er = et & 15, eq = et >> 4;
        const int n1 = cur.n0 + wn0, k1 = cur.k0 + wk0;
        constexpr int CPR = 2 * FK, NIT = 16 * CPR / 64, RB = FK * 64;
        char *const region = smem + EPI + wave * REGION;
#pragma unroll
        for (int ni = 0; ni < FN; ++ni) {
            if constexpr (kAcc) {
#pragma unroll
                for (int ki = 0; ki < FK; ++ki) asm volatile("" : "+a"(acc[ki][ni]));
            }
#pragma unroll
            for (int ki = 0; ki < FK; ++ki)
                *reinterpret_cast<f32x4 *>(region + er * RB + (((4 * ki + eq) ^ (er & 7)) << 4)) = acc[ki][ni];
            asm volatile("" ::: "memory");
#pragma unroll
            for (int it = 0; it < NIT; ++it) {
                const int row = (it * 64 + et) / CPR, j = (it * 64 + et) % CPR;
                const char *w = region + row * RB;
                f32x4 y0 = *reinterpret_cast<const f32x4 *>(w + (((2 * j) ^ (row & 7)) << 4));
                f32x4 y1 = *reinterpret_cast<const f32x4 *>(w + (((2 * j + 1) ^ (row & 7)) << 4));
                const int n = n1 + ni * 16 + row, k = k1 + j * 8;
                if (n >= p.N || k >= p.K) continue;   // K is a multiple of 16
                const size_t at = (size_t)n * (size_t)p.K + k;
                if (p.part || p.f32) {
                    float *to = (float *)p.dW + at;
                    if (p.part)
                        to = p.part + ((size_t)cur.slice * (size_t)p.part_rows + (size_t)(n - p.n_base)) * (size_t)p.part_ld +
                             (k - p.k_base);
                    if (!p.part && p.accumulate) {
                        y0 += *reinterpret_cast<const f32x4 *>(to);
                        y1 += *reinterpret_cast<const f32x4 *>(to + 4);
                    }
                    if (p.part) {
                        *reinterpret_cast<f32x4 *>(to) = y0;
                        *reinterpret_cast<f32x4 *>(to + 4) = y1;
                    } else {
                        __builtin_nontemporal_store(y0, reinterpret_cast<f32x4 *>(to));
                        __builtin_nontemporal_store(y1, reinterpret_cast<f32x4 *>(to + 4));
                    }
                } else {
                    u32x4 *to = reinterpret_cast<u32x4 *>((uint16_t *)p.dW + at);
                    if (p.accumulate) {
                        const u32x4 was = *to;
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            f32x4 &x = e < 2 ? y0 : y1;
                            x[2 * (e & 1)] += __builtin_bit_cast(float, was[e] << 16);
                            x[2 * (e & 1) + 1] += __builtin_bit_cast(float, was[e] & 0xFFFF0000u);
                        }
                    }
                    const u32x4 o = {pack_bf16x2(y0[0], y0[1]), pack_bf16x2(y0[2], y0[3]), pack_bf16x2(y1[0], y1[1]),
                                     pack_bf16x2(y1[2], y1[3])};
                    __builtin_nontemporal_store(o, to);
                }
            }
            asm volatile("" ::: "memory");
            __builtin_amdgcn_sched_barrier(0);
        }
        if (!more) return;
    }
}

// The sum of the slices in order, 4 values per thread, rounded once; with
// accumulate, added to what is there.
template <bool F32>
__global__ __launch_bounds__(256) void join_kernel(int rows, int cols, int slices, const float *__restrict__ part, void *out,
                                                   int64_t ld, int accumulate) {
    const uint32_t per = (uint32_t)part_ld(cols) / 4, count = (uint32_t)rows * per;
    const uint32_t i = blockIdx.x * 256 + threadIdx.x;
    if (i >= count) return;
    const f32x4 *from = reinterpret_cast<const f32x4 *>(part) + i;
    f32x4 x = *from;
#pragma unroll 4
    for (int s = 1; s < slices; ++s) x += from[(size_t)s * count];
    const uint32_t row = i / per, c = (i - row * per) * 4;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if ((int)c + e >= cols) break;
        const int64_t at = (int64_t)row * ld + c + e;
        if constexpr (F32) {
            float *to = (float *)out + at;
            *to = accumulate ? *to + x[e] : x[e];
        } else {
            uint16_t *to = (uint16_t *)out + at;
            *to = (uint16_t)pack_bf16x2(accumulate ? x[e] + __builtin_bit_cast(float, (uint32_t)*to << 16) : x[e], 0.0f);
        }
    }
}

hipError_t launch_grad(GradParams p, const Cut &cut, float *part, hipStream_t stream) {
    for (int i = 0; i < 2 && cut.part[i].tiles_m; ++i) {
        const TilePlan &pl = cut.part[i];
        p.tiles_n = pl.tiles_m;
        p.tiles_k = pl.tiles_n;
        p.slices = pl.slices;
        p.mslice = pl.kslice * kBK;
        p.group_n = kGradTiles[pl.cfg].rows == 256 ? 4 : 8;
        p.n_base = cut.row0(i);
        p.k_base = cut.col0(i);
        p.part = pl.slices > 1 ? part : nullptr;
        p.part_rows = cut.rows_of(i);
        p.part_ld = part_ld(cut.cols_of(i));
        const int64_t items = (int64_t)pl.tiles_m * pl.tiles_n * pl.slices;
        const dim3 grid((unsigned)std::min<int64_t>(items, kCUs * kGradTiles[pl.cfg].wg_per_cu));
        switch (pl.cfg) {   // (a template instance for each row of kGradTiles)
        case 0: grad_kernel<256, 256, 1><<<grid, kThreads, 0, stream>>>(p); break;
        case 1: grad_kernel<256, 128, 1><<<grid, kThreads, 0, stream>>>(p); break;
        case 2: grad_kernel<128, 128, 2><<<grid, kThreads, 0, stream>>>(p); break;
        case 3: grad_kernel<128, 64, 2><<<grid, kThreads, 0, stream>>>(p); break;
        default: grad_kernel<64, 64, 3><<<grid, kThreads, 0, stream>>>(p); break;
        }
        hipError_t e = hipGetLastError();
        if (e == hipSuccess && pl.slices > 1) {
            const size_t at = (size_t)p.n_base * (size_t)p.K + (size_t)p.k_base;
            void *to = p.f32 ? (void *)((float *)p.dW + at) : (void *)((uint16_t *)p.dW + at);
            e = launch_join_parts(cut.rows_of(i), cut.cols_of(i), pl.slices, part, to, p.K, p.f32 != 0, p.accumulate != 0,
                                  stream);
        }
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

constexpr int kMaxRows = 1 << 20, kMaxDepth = 1 << 17;

int check_sizes(int M, int N, int K) {
    if (M < 1 || N < 1 || K < 1 || K % 16 || N % 8)
        return set_error(COMPASS_ERR_INVALID, "need positive M, N and K with K a multiple of 16, N of 8");
    if (M > kMaxRows || N > kMaxRows || K > kMaxDepth)
        return set_error(COMPASS_ERR_UNSUPPORTED, "M = %d, N = %d, K = %d beyond %d, %d, %d", M, N, K, kMaxRows, kMaxRows,
                         kMaxDepth);
    return COMPASS_OK;
}

bool misaligned(const void *p) { return ((uintptr_t)p & 15) != 0; }

}  // namespace

hipError_t launch_join_parts(int rows, int cols, int slices, const float *part, void *out, int64_t ld, bool f32,
                             bool accumulate, hipStream_t stream) {
    // (a split output has at most 1024 tiles: below 2^32 threads)
    const dim3 grid((unsigned)(((size_t)rows * (size_t)(part_ld(cols) / 4) + 255) / 256));
    if (f32) join_kernel<true><<<grid, 256, 0, stream>>>(rows, cols, slices, part, out, ld, accumulate);
    else join_kernel<false><<<grid, 256, 0, stream>>>(rows, cols, slices, part, out, ld, accumulate);
    return hipGetLastError();
}

int op_fp8_wgrad_workspace(int M, int N, int K, size_t *bytes) {
    const int rc = check_sizes(M, N, K);
    if (rc != COMPASS_OK) return rc;
    if (!bytes) return set_error(COMPASS_ERR_INVALID, "bytes is required");
    *bytes = plan_grad(M, N, K).workspace();
    return COMPASS_OK;
}

int op_fp8_wgrad(int M, int N, int K, int gtype, const void *dY, const void *X, const void *X_scale, void *dW,
                 int accumulate, void *ws, size_t ws_bytes, void *stream) {
    int rc = check_sizes(M, N, K);
    if (rc != COMPASS_OK) return rc;
    if (gtype != COMPASS_BF16 && gtype != COMPASS_F32)
        return set_error(COMPASS_ERR_INVALID, "unknown element type %d", gtype);
    if (accumulate != 0 && accumulate != 1)
        return set_error(COMPASS_ERR_INVALID, "accumulate = %d, must be 0 or 1", accumulate);
    if (!dY || !X || !X_scale || !dW) return set_error(COMPASS_ERR_INVALID, "dY, X8, its scale and dW are required");
    if (misaligned(dY) || misaligned(X) || misaligned(dW) || ((uintptr_t)X_scale & 3))
        return set_error(COMPASS_ERR_INVALID, "dY, X8 and dW must be 16-byte and the scale 4-byte aligned");
    const Cut cut = plan_grad(M, N, K);
    if (const size_t need = cut.workspace(); need && (!ws || misaligned(ws) || ws_bytes < need))
        return set_error(COMPASS_ERR_INVALID, "workspace of %zu bytes (16-byte aligned), need %zu", ws_bytes, need);
    int cus;
    if ((rc = current_num_cu(&cus)) != COMPASS_OK) return rc;
    GradParams p{};
    p.dY = (const uint16_t *)dY;
    p.X = (const uint8_t *)X;
    p.sX = (const uint8_t *)X_scale;
    p.dW = dW;
    p.M = M;
    p.N = N;
    p.K = K;
    p.S = scale_cols(K);
    p.f32 = gtype == COMPASS_F32;
    p.accumulate = accumulate;
    const hipError_t e = launch_grad(p, cut, (float *)ws, (hipStream_t)stream);
    return e == hipSuccess ? COMPASS_OK : set_error(COMPASS_ERR_HIP, "weight gradient launch: %s", hipGetErrorString(e));
}

}  // namespace compass
