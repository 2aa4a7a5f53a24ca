// Device pieces that the tiled bf16 GEMM kernels share: bounded buffer
// resources, global -> LDS loads, counted waits, the order of MFMAs.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kernel_params.h"

namespace compass {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));

#define LDS_AS(p) ((__attribute__((address_space(3))) void *)(p))

// Buffer loads of a tile go through a resource based at the tile's first
// row (A, the partial) or first column (W), bounded by the bytes left in the
// operand, at most kTileSpanMax; offsets are relative to that base. An
// out-of-range row or column takes an offset at or beyond the bound:
// kOOBRow = 2^31 for a row, kOOBCol = 2^30 for a K column. A valid row offset
// plus a valid column offset stays below the 2^30 bound (the host checks the
// tile's span), a valid one plus an out-of-range one reaches it, and two
// out-of-range ones sum to 3 * 2^30, below 2^32, so no sum wraps.
constexpr uint32_t kOOBRow = 0x80000000u;
constexpr uint32_t kOOBCol = 0x40000000u;

__device__ __forceinline__ __amdgpu_buffer_rsrc_t tile_rsrc(const void *base, uint64_t total, uint64_t off) {
    const uint64_t left = total > off ? total - off : 0;
    const uint32_t bound = (uint32_t)(left < kTileSpanMax ? left : kTileSpanMax);
    return __builtin_amdgcn_make_buffer_rsrc((void *)((const char *)base + off), (short)0, (int)bound, 0x00020000);
}

__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi) {
    const __bf16 a = (__bf16)lo, b = (__bf16)hi;   // round to nearest even
    return (uint32_t)__builtin_bit_cast(uint16_t, a) | ((uint32_t)__builtin_bit_cast(uint16_t, b) << 16);
}

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

// At most VM vector-memory operations (and no LDS read) still in flight.
template <int VM>
__device__ __forceinline__ void wait_vm_lgkm0() {
    static_assert(VM >= 0 && VM < 64, "vmcnt range");
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(VM) : "memory");
}

// Workgroup barrier with no memory fence: the caller has already waited for
// the LDS traffic that must be complete (s_waitcnt), and the scheduling
// barriers keep the compiler from moving LDS accesses across it.
__device__ __forceinline__ void lds_barrier() {
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// Buffer resource words of tile_rsrc as plain scalars, for dma16.
__device__ __forceinline__ i32x4 tile_rsrc4(const void *base, uint64_t total, uint64_t off) {
    const uint64_t left = total > off ? total - off : 0;
    const uint32_t bound = (uint32_t)(left < kTileSpanMax ? left : kTileSpanMax);
    const uint64_t a = (uint64_t)base + off;
    i32x4 r;
    r[0] = __builtin_amdgcn_readfirstlane((int)(uint32_t)a);
    r[1] = __builtin_amdgcn_readfirstlane((int)((uint32_t)(a >> 32) & 0xFFFFu));
    r[2] = __builtin_amdgcn_readfirstlane((int)bound);
    r[3] = 0x00020000;
    return r;
}

// One global -> LDS load: 16 bytes per lane from rsrc + voff to LDS byte
// address lds + 16 * lane. It has no register result, so nothing of it is
// live in a register while it is in flight; it is written as an instruction
// because the compiler, which cannot see that two halves of one LDS array
// are different buffers, would otherwise wait for every load in flight before
// each LDS read. The waits are wait_vm_lgkm0's, counted where they are made.
// (s_nop: a scalar write of M0 needs a wait state before the load reads it.)
__device__ __forceinline__ void dma16(i32x4 rsrc, uint32_t voff, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                 :
                 : "s"(lds), "v"(voff), "s"(rsrc)
                 : "memory");
}

// `CNT` loads of one operand into the 1 KiB blocks j * 4 + wave of the LDS
// buffer at `lds`.
template <int CNT>
__device__ __forceinline__ void load_blocks(i32x4 rsrc, uint32_t lds, const uint32_t *off, uint32_t kc2, int wave) {
#pragma unroll
    for (int j = 0; j < CNT; ++j) dma16(rsrc, off[j] + kc2, lds + (uint32_t)((j * 4 + wave) * 1024));
}

// Where operation `k` of n falls among MFMA slots [lo, hi).
constexpr int slot_of(int k, int n, int lo, int hi) { return lo + k * (hi - lo) / n; }

// Block row of MFMA slot i (block column i / FM): down one column of blocks, up
// the next, so that consecutive MFMAs always share an operand. The operand that
// stays costs no switching in the matrix core, and power is what bounds these
// GEMMs: 8192 x 6144 x 12288 845 -> 832 us, 8192 x 12288 x 6144 with partial
// 906 -> 897 (going down every column before).
template <int FM>
constexpr int slot_row(int i) { return i / FM % 2 ? FM - 1 - i % FM : i % FM; }

constexpr int kBK = 64;   // K depth of one LDS stage

}  // namespace compass
