// 8-bit rows: e4m3 values with one scale for each 128 consecutive values of a
// row, as the kernels write and read them.
//
//   value = v 2^(b - 127), v the e4m3 value, b the byte of its group's scale
//   b: the smallest in [0, 254] with amax <= 448 2^(b - 127), amax the largest
//   magnitude of the group's finite values (448: the largest e4m3 value)
//
// A scale is a power of two, so scaling rounds nothing (a value is off by its one
// rounding to e4m3), the matrix core applies it by itself, and v 2^(b - 127) has
// four significant bits: exact in bf16. A value that is not finite becomes NaN
// and leaves its group's scale alone.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace compass {

constexpr int kGroup = 128;            // values per scale
constexpr uint32_t kUnitScale = 127;   // the byte of 2^0

// rows x cols of out (bf16 or fp32, rows ld apart) = the sum of the slices' partial
// sums (rows of part_ld(cols)) in order, rounded once; with accumulate, added to what is
// there.
hipError_t launch_join_parts(int rows, int cols, int slices, const float *part, void *out, int64_t ld, bool f32,
                             bool accumulate, hipStream_t stream);

// Bytes of the scales of a row of n values: whole words, which the product loads.
__host__ __device__ constexpr int scale_cols(int n) { return (n + 4 * kGroup - 1) / (4 * kGroup) * 4; }

// |x| as an ordered number, 0 where x is not finite.
__device__ __forceinline__ uint32_t finite_magnitude(float x) {
    const uint32_t b = __builtin_bit_cast(uint32_t, x) & 0x7FFFFFFFu;
    return b < 0x7F800000u ? b : 0u;
}

// The scale's byte from the bits of amax: its exponent less 8 (448 = 1.75 2^8),
// one more where its fraction is over 1.75.
__device__ __forceinline__ uint32_t scale_byte(uint32_t amax) {
    const int b = (int)((amax + 0x1FFFFFu) >> 23) - 8;
    return (uint32_t)(b < 0 ? 0 : b);
}
// 2^(127 - byte) for bytes up to 247, the largest that scale_byte gives.
__device__ __forceinline__ float scale_inverse(uint32_t byte) {
    return __builtin_bit_cast(float, (254u - byte) << 23);
}

__device__ __forceinline__ float nan_unless_finite(float x) { return x - (x - x); }   // (keeps -0)

// Four values, scaled (at most 448) and rounded to nearest even.
__device__ __forceinline__ uint32_t pack_e4m3(float a, float b, float c, float d) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(nan_unless_finite(a), nan_unless_finite(b), 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(nan_unless_finite(c), nan_unless_finite(d), w, true);
}

// Largest over the 16 lanes of a row of lanes (LANES = 16) or two (32).
template <int CTRL>
__device__ __forceinline__ uint32_t dpp_max(uint32_t x) {
    const uint32_t y = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xF, 0xF, true);
    return x > y ? x : y;
}
template <int LANES>
__device__ __forceinline__ uint32_t lanes_max(uint32_t x) {
    static_assert(LANES == 16 || LANES == 32, "one or two rows of 16 lanes");
    x = dpp_max<0xB1>(x);    // quad permute 1 0 3 2
    x = dpp_max<0x4E>(x);    // quad permute 2 3 0 1
    x = dpp_max<0x141>(x);   // mirror within 8
    x = dpp_max<0x140>(x);   // mirror within 16
    if constexpr (LANES == 32) {
        typedef unsigned int u32x2_ __attribute__((ext_vector_type(2)));
        const u32x2_ r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
        x = r[0] > r[1] ? r[0] : r[1];
    }
    return x;
}

// V values of a group that 128 / V neighbouring lanes hold (values past the
// row's end are 0): their e4m3 bytes at row + c, as far as N, and, by the lane
// that holds the group's first, the scale's byte. Every lane of the wave calls.
template <int V>
__device__ __forceinline__ void store_e4m3(uint8_t *row, uint8_t *scales, int c, int N, const float (&f)[V]) {
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < V; ++e) {
        const uint32_t b = finite_magnitude(f[e]);
        top = top > b ? top : b;
    }
    const uint32_t byte = scale_byte(lanes_max<kGroup / V>(top));
    const float inv = scale_inverse(byte);
    uint32_t w[V / 4];
#pragma unroll
    for (int i = 0; i < V / 4; ++i)
        w[i] = pack_e4m3(f[4 * i] * inv, f[4 * i + 1] * inv, f[4 * i + 2] * inv, f[4 * i + 3] * inv);
    if (c + V <= N) {
        typedef uint32_t Word __attribute__((aligned(1)));
        typedef unsigned int Two __attribute__((ext_vector_type(2), aligned(1)));
        if constexpr (V == 8) *reinterpret_cast<Two *>(row + c) = Two{w[0], w[1]};
        else *reinterpret_cast<Word *>(row + c) = w[0];
    } else {
#pragma unroll
        for (int e = 0; e < V; ++e)
            if (c + e < N) row[c + e] = (uint8_t)(w[e / 4] >> (8 * (e & 3)));
    }
    if (c % kGroup == 0 && c < N) scales[c / kGroup] = (uint8_t)byte;
}

}  // namespace compass
