// Device pieces of the row-wise kernels (layer norm, embedding): bf16 and fp32
// elements by vector, sums over a wave.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace compass {

struct Bf16 { uint16_t bits; };

// V consecutive elements as they lie in memory. 16-byte vectors (8 bf16,
// 4 fp32) for aligned rows, single elements otherwise.
template <class T, int V>
struct alignas(sizeof(T) * V < 16 ? sizeof(T) * V : 16) Pack {
    T e[V];
};

__device__ __forceinline__ float to_f32(Bf16 x) { return __builtin_bit_cast(float, (uint32_t)x.bits << 16); }
__device__ __forceinline__ float to_f32(float x) { return x; }
template <class T>
__device__ __forceinline__ T from_f32(float x);
template <>
__device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <>
__device__ __forceinline__ Bf16 from_f32<Bf16>(float x) {   // round to nearest even
    return Bf16{__builtin_bit_cast(uint16_t, (__bf16)x)};
}

// Loads and stores that pass through the caches without staying (whole vectors;
// single elements go the ordinary way, lanes share their lines). An output of
// more than the caches hold would otherwise be allocated line by line and
// written back later: what a kernel measured with and without stands there.
typedef unsigned int u32x4_ __attribute__((ext_vector_type(4)));
template <class T, int V>
__device__ __forceinline__ void store_stream(T *p, const Pack<T, V> &o) {
    constexpr int N = sizeof(T) * V / 16;
    if constexpr (sizeof(T) * V % 16 == 0 && N > 0) {
        struct Quads { u32x4_ q[N]; };
        const Quads q = __builtin_bit_cast(Quads, o);
#pragma unroll
        for (int i = 0; i < N; ++i) __builtin_nontemporal_store(q.q[i], reinterpret_cast<u32x4_ *>(p) + i);
    } else {
        *reinterpret_cast<Pack<T, V> *>(p) = o;
    }
}
template <class T, int V>
__device__ __forceinline__ Pack<T, V> load_stream(const T *p) {
    constexpr int N = sizeof(T) * V / 16;
    if constexpr (sizeof(T) * V % 16 == 0 && N > 0) {
        struct Quads { u32x4_ q[N]; } q;
#pragma unroll
        for (int i = 0; i < N; ++i) q.q[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_ *>(p) + i);
        return __builtin_bit_cast(Pack<T, V>, q);
    } else {
        return *reinterpret_cast<const Pack<T, V> *>(p);
    }
}

template <int CTRL>
__device__ __forceinline__ float dpp(float x) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xF, 0xF, true));
}

// Sum over the 64 lanes, the same bits in every lane: pairs, quads, eights and
// sixteens through the data-parallel moves, then between the rows of 16.
__device__ __forceinline__ float wave_sum(float x) {
    x += dpp<0xB1>(x);    // quad permute 1 0 3 2
    x += dpp<0x4E>(x);    // quad permute 2 3 0 1
    x += dpp<0x141>(x);   // mirror within 8
    x += dpp<0x140>(x);   // mirror within 16
    typedef unsigned int u32x2_ __attribute__((ext_vector_type(2)));
    uint32_t b = __builtin_bit_cast(uint32_t, x);
    u32x2_ r = __builtin_amdgcn_permlane16_swap(b, b, false, false);
    x = __builtin_bit_cast(float, (uint32_t)r[0]) + __builtin_bit_cast(float, (uint32_t)r[1]);
    b = __builtin_bit_cast(uint32_t, x);
    r = __builtin_amdgcn_permlane32_swap(b, b, false, false);
    return __builtin_bit_cast(float, (uint32_t)r[0]) + __builtin_bit_cast(float, (uint32_t)r[1]);
}

}  // namespace compass
