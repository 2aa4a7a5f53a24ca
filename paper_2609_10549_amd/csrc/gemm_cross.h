// Operands of tiled bf16 products that lie along or across the reduction: their
// stages' loads to LDS and their fragments from it. One that lies across goes to LDS
// as it lies and is transposed by the LDS read (ds_read_b64_tr_b16).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "gemm_core.h"

namespace compass {

typedef short s16x4 __attribute__((ext_vector_type(4)));

// f(row) of the 16-byte chunk permutation of an operand that lies across the
// reduction: chunk c of LDS row `row` is at chunk c ^ f. Two neighbouring
// chunks (16 columns) stay together, and the eight rows that half a wave reads
// at once fall into eight different 32-byte bank groups (rows of 128 or 384
// bytes: odd rows start half a line of banks on, four groups each).
template <int RB>
__device__ __forceinline__ int cross_swizzle(int row) {
    return RB % 256 == 0 ? 2 * ((row & 3) | ((row >> 1) & 4)) : 2 * (((row >> 1) & 1) | ((row >> 2) & 2));
}

// Loads of one operand's stages: `D` rows (or columns) of the tile, 64 of the
// reduction per stage. T: the operand lies across the reduction.
template <bool T, int D>
struct Loader {
    static constexpr int L = D / 32;     // loads per wave and stage
    static constexpr int RB = D * 2;     // bytes of an LDS row (T)
    uint32_t off[L];
    i32x4 rsrc;
    uint64_t base;
    int64_t left, step;
    int kc, ke;

    __device__ __forceinline__ void init(const uint16_t *p, uint64_t bytes, int d0, int dim, int ld, int kb, int kend,
                                         int lane, int wave) {
        if constexpr (T) {
            const uint64_t o = ((uint64_t)kb * (uint64_t)ld + (uint64_t)d0) * 2u;
            base = (uint64_t)p + o;
            left = (int64_t)bytes - (int64_t)o;
            step = (int64_t)ld * 128;
            constexpr int CPR = RB / 16;   // chunks per row
#pragma unroll
            for (int j = 0; j < L; ++j) {
                const int at = (j * 4 + wave) * 64 + lane;
                const int row = at / CPR, chunk = (at % CPR) ^ cross_swizzle<RB>(row);
                off[j] = (uint32_t)row * (uint32_t)ld * 2u + (uint32_t)chunk * 16u;
            }
        } else {
            rsrc = tile_rsrc4(p, bytes, (uint64_t)d0 * (uint64_t)ld * 2u);
            // resource words that came out of vector registers need five wait
            // states before a load reads them
            asm volatile("s_nop 4" : "+s"(rsrc));
            const int lrow0 = 8 * wave + (lane >> 3);
#pragma unroll
            for (int q = 0; q < L; ++q) {
                const int i = 32 * q + lrow0;
                off[q] = d0 + i < dim ? (uint32_t)i * (uint32_t)ld * 2u : kOOBRow;
            }
            kc = kb + ((lane & 7) ^ ((4 * wave + (lane >> 4)) & 7)) * 8;
            ke = kend;
        }
    }

    // The resource of the next stage and the lane's offset in it.
    __device__ __forceinline__ uint32_t next(i32x4 &r) {
        if constexpr (T) {
            const int64_t b = left < 0 ? 0 : left < (int64_t)kTileSpanMax ? left : (int64_t)kTileSpanMax;
            r[0] = (int)(uint32_t)base;
            r[1] = (int)((uint32_t)(base >> 32) & 0xFFFFu);
            r[2] = (int)b;
            r[3] = 0x00020000;
            base += (uint64_t)step;
            left -= step;
            return 0u;
        } else {
            r = rsrc;
            const uint32_t o = kc < ke ? (uint32_t)kc * 2u : kOOBCol;
            kc += kBK;
            return o;
        }
    }
};

// Fragments of one operand out of its LDS stage: F blocks of 16 rows (columns).
template <bool T, int D, int F>
struct Reader {
    static constexpr int RB = D * 2;
    uint32_t at[T ? F : 2];   // T: lane address of each block; else of each half of the stage
    __device__ __forceinline__ void init(uint32_t d0, int lane) {
        const int r = lane & 15, kq = lane >> 4;
        if constexpr (T) {
            const int row = kq * 8 + (r >> 2);
            const uint32_t line = (uint32_t)(row * RB + (r & 1) * 8);
#pragma unroll
            for (int f = 0; f < F; ++f) {
                const int chunk = (((int)d0 / 8 + 2 * f + ((r & 3) >> 1)) ^ cross_swizzle<RB>(row));
                at[f] = line + (uint32_t)chunk * 16u;
            }
        } else {
            const int swz = (r >> 1) & 7;
#pragma unroll
            for (int s = 0; s < 2; ++s) at[s] = (d0 + (uint32_t)r) * 128u + (uint32_t)(((4 * s + kq) ^ swz) << 4);
        }
    }
    // block f of substep S (32 of the reduction) of the stage at LDS offset buf
    template <int S>
    __device__ __forceinline__ bf16x8 read(uint32_t buf, int f) const {
        if constexpr (T) {
            typedef __attribute__((address_space(3))) s16x4 lds4;
            const uint32_t a = buf + at[f] + S * 32 * RB;
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4 *)(uintptr_t)a);
            const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4 *)(uintptr_t)(a + 4 * RB));
            return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        } else {
            typedef const __attribute__((address_space(3))) bf16x8 lds8;
            return *(lds8 *)(uintptr_t)(buf + at[S] + (uint32_t)f * 2048u);
        }
    }
};

}  // namespace compass
