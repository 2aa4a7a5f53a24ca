// Device pieces of the row-wise kernels (norms, embedding, 8-bit rows): bf16 and
// fp32 elements by vector, sums over a wave.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace compass {

struct Bf16 { uint16_t bits; };

typedef unsigned int u32x4_ __attribute__((ext_vector_type(4)));

// V consecutive elements as they lie in memory: whole 16-byte pieces. (Held in
// the pieces' own type: from a struct of elements the compiler makes a load per
// element.)
template <class T, int V>
struct Pack {
    static constexpr int Q = (int)sizeof(T) * V / 16;
    static_assert(Q > 0 && sizeof(T) * V % 16 == 0, "whole pieces");
    u32x4_ q[Q];
};

__device__ __forceinline__ void unpack(const u32x4_ &q, float (&f)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = __builtin_bit_cast(float, (uint32_t)q[i] << 16);
        f[2 * i + 1] = __builtin_bit_cast(float, (uint32_t)q[i] & 0xFFFF0000u);
    }
}
template <class T, int V>
__device__ __forceinline__ void unpack(const Pack<T, V> &p, float (&f)[V]) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int e = 0; e < V; ++e) f[e] = __builtin_bit_cast(float, (uint32_t)p.q[e / 4][e % 4]);
    } else {
        static_assert(V == 8, "one piece of bf16");
        unpack(p.q[0], f);
    }
}
__device__ __forceinline__ uint32_t bf16_bits(float x) {   // rounded to nearest even
    return (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)x);
}
template <class T, int V>
__device__ __forceinline__ Pack<T, V> pack(const float (&f)[V]) {
    Pack<T, V> p;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int e = 0; e < V; ++e) p.q[e / 4][e % 4] = __builtin_bit_cast(uint32_t, f[e]);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) p.q[0][i] = bf16_bits(f[2 * i]) | bf16_bits(f[2 * i + 1]) << 16;
    }
    return p;
}
__device__ __forceinline__ void put_element(Bf16 *p, float x) { p->bits = (uint16_t)bf16_bits(x); }
__device__ __forceinline__ void put_element(float *p, float x) { *p = x; }

// Elements [i, i + V) of a row of N. LOOSE: a row starts on any element and a
// vector may be cut by either end (the card loads and stores 16 bytes from any
// address, at the cost of the extra line they touch); otherwise rows start on
// 16 bytes and hold whole vectors. STREAM: passes through the caches without
// staying. An output of more than the caches hold would otherwise be allocated
// line by line and written back later: what a kernel measured with and without
// stands there.
template <bool LOOSE>
struct Piece { typedef u32x4_ type; };
template <>
struct Piece<true> { typedef u32x4_ type __attribute__((aligned(2))); };

template <class T, int V, bool LOOSE, bool STREAM = false>
__device__ __forceinline__ Pack<T, V> load_pack(const T *row, int i, int N) {
    typedef typename Piece<LOOSE>::type At;
    Pack<T, V> p;
    if ((!LOOSE || i >= 0) && i + V <= N) {
        const At *from = reinterpret_cast<const At *>(row + i);
#pragma unroll
        for (int j = 0; j < Pack<T, V>::Q; ++j) p.q[j] = STREAM ? __builtin_nontemporal_load(from + j) : from[j];
        return p;
    }
#pragma unroll
    for (int j = 0; j < Pack<T, V>::Q; ++j) p.q[j] = u32x4_{0, 0, 0, 0};
    if constexpr (LOOSE) {
        if (i < N && i > -V) {
#pragma unroll
            for (int e = 0; e < V; ++e)
                if (i + e >= 0 && i + e < N) {
                    if constexpr (sizeof(T) == 4) p.q[e / 4][e % 4] = __builtin_bit_cast(uint32_t, row[i + e]);
                    else p.q[0][e / 2] |= (uint32_t)row[i + e].bits << (16 * (e & 1));
                }
        }
    }
    return p;
}
template <class T, int V, bool LOOSE, bool STREAM = true>
__device__ __forceinline__ void store_pack(T *row, int i, int N, const float (&f)[V]) {
    typedef typename Piece<LOOSE>::type At;
    if ((!LOOSE || i >= 0) && i + V <= N) {
        const Pack<T, V> p = pack<T, V>(f);
        At *to = reinterpret_cast<At *>(row + i);
#pragma unroll
        for (int j = 0; j < Pack<T, V>::Q; ++j) {
            if (STREAM) __builtin_nontemporal_store(p.q[j], to + j);
            else to[j] = p.q[j];
        }
    } else if constexpr (LOOSE) {
        if (i < N && i > -V) {
#pragma unroll
            for (int e = 0; e < V; ++e)
                if (i + e >= 0 && i + e < N) put_element(row + i + e, f[e]);
        }
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

// V parameters of a norm from element i, `none` where there is no such vector.
template <int V, bool LOOSE>
__device__ __forceinline__ void load_param(const void *p, int f32, float none, int i, int N, float (&f)[V]) {
    if (!p) {
#pragma unroll
        for (int e = 0; e < V; ++e) f[e] = none;
    } else if (f32) {
        unpack(load_pack<float, V, LOOSE>((const float *)p, i, N), f);
    } else if constexpr (V == 8) {
        unpack(load_pack<Bf16, V, LOOSE>((const Bf16 *)p, i, N), f);
    } else {   // half a piece; few enough (once per column) to go by element
#pragma unroll
        for (int e = 0; e < V; ++e)
            f[e] = i + e < N ? __builtin_bit_cast(float, (uint32_t)((const Bf16 *)p)[i + e].bits << 16) : 0.0f;
    }
}

// Sum over the TPR threads that share a row, in wave order; `s` holds one
// value per wave. TPR <= 64: the wave alone, no barrier.
template <int TPR>
__device__ __forceinline__ float row_sum(float x, float *s) {
    x = wave_sum(x);
    if constexpr (TPR > 64) {
        if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = x;
        __syncthreads();
        x = s[0];
#pragma unroll
        for (int w = 1; w < TPR / 64; ++w) x += s[w];
    }
    return x;
}

}  // namespace compass
