// 8-bit rows from bf16 or fp32 ones and back (compass_fp8_quant, _dequant); the
// format is fp8.h's.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "compass.h"
#include "fp8.h"
#include "internal.h"
#include "rowops.h"

namespace compass {

namespace {

constexpr int kSpan = 4 * kGroup;   // values of a row that share a word of scales

struct QuantParams {
    int M, K;
    int64_t ld;             // elements between the rows of x
    const void *x;
    const uint8_t *q_in, *scale_in;
    uint8_t *q, *scale;
    void *out;
};

// A wave takes a span of a row: 8 values per lane and pass (fp32: two passes of
// 4), so that a group is 16 lanes' (32), and its four scales, those behind the row's
// last group among them. Bound by memory: 8192 x 12288 bf16 (303 MB) 57 us (5.3 TB/s).
template <class T, int V, bool LOOSE>
__global__ __launch_bounds__(256) void quant_kernel(const QuantParams p) {
    const int lane = threadIdx.x & 63;
    const uint32_t spans = (uint32_t)(p.K + kSpan - 1) / kSpan, items = (uint32_t)p.M * spans;
    for (uint32_t item = blockIdx.x * 4 + (threadIdx.x >> 6); item < items; item += gridDim.x * 4) {
        const uint32_t m = item / spans, span = item % spans;
        const T *x = (const T *)p.x + (int64_t)m * p.ld;
        uint8_t *q = p.q + (uint64_t)m * (uint64_t)p.K, *scale = p.scale + (uint64_t)m * (uint64_t)scale_cols(p.K);
        constexpr int PASSES = kSpan / (64 * V);
        Pack<T, V> in[PASSES];
#pragma unroll
        for (int i = 0; i < PASSES; ++i) in[i] = load_pack<T, V, LOOSE>(x, (int)span * kSpan + (i * 64 + lane) * V, p.K);
#pragma unroll
        for (int i = 0; i < PASSES; ++i) {
            const int c = (int)span * kSpan + (i * 64 + lane) * V;
            float f[V];
            unpack(in[i], f);
            store_e4m3<V>(q, scale, c, p.K, f);
            if (c % kGroup == 0 && c >= p.K) scale[c / kGroup] = (uint8_t)kUnitScale;
        }
    }
}

// x (M x K) transposed: rows of K of M values, groups along M. A workgroup takes
// 128 rows (a group) of 64 columns: each thread's vectors, the columns' largest
// through LDS, then the bytes, turned in LDS to rows of 128. Bound by latency where
// it is small: 500 x 1031 fp32 5.3 us; a weight is close to memory's pace: 6144 x 12288
// bf16 (226 MB) 46 to 54 us (4.6 TB/s; along the rows 41).
template <class T, int V, bool LOOSE>
__global__ __launch_bounds__(256) void quant_across_kernel(const QuantParams p) {
    constexpr int CV = 64 / V, RP = 256 / CV, PASSES = kGroup / RP;   // vectors per row, rows per pass
    constexpr int LINE = kGroup + 16;                                 // bytes of an LDS row (16-byte reads)
    __shared__ uint32_t top[RP][64 + 1];
    __shared__ __attribute__((aligned(16))) uint8_t turned[64 * LINE];
    __shared__ uint8_t bytes[64];
    const int tid = threadIdx.x, cv = tid % CV, r = tid / CV;
    const int k0 = (int)blockIdx.x * 64, m0 = (int)blockIdx.y * kGroup;
    float f[PASSES][V];
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
        const int m = m0 + i * RP + r;
        Pack<T, V> in;
#pragma unroll
        for (int j = 0; j < Pack<T, V>::Q; ++j) in.q[j] = u32x4_{0, 0, 0, 0};
        if (m < p.M) in = load_pack<T, V, LOOSE>((const T *)p.x + (int64_t)m * p.ld, k0 + cv * V, p.K);
        unpack(in, f[i]);
    }
#pragma unroll
    for (int e = 0; e < V; ++e) {
        uint32_t t = 0;
#pragma unroll
        for (int i = 0; i < PASSES; ++i) {
            const uint32_t b = finite_magnitude(f[i][e]);
            t = t > b ? t : b;
        }
        top[r][cv * V + e] = t;
    }
    __syncthreads();
    if (tid < 64) {
        uint32_t t = top[0][tid];
#pragma unroll
        for (int i = 1; i < RP; ++i) t = t > top[i][tid] ? t : top[i][tid];
        bytes[tid] = (uint8_t)scale_byte(t);
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < V; ++e) {
        const int k = cv * V + e;
        const float inv = scale_inverse(bytes[k]);
#pragma unroll
        for (int i = 0; i < PASSES; ++i) {
            const float v = f[i][e] * inv;
            turned[k * LINE + i * RP + r] = (uint8_t)pack_e4m3(v, v, v, v);
        }
    }
    __syncthreads();
    const int S = scale_cols(p.M);
    if (tid < 64 && k0 + tid < p.K) {
        uint8_t *scale = p.scale + (uint64_t)(k0 + tid) * (uint64_t)S;
        scale[m0 / kGroup] = bytes[tid];
        if (m0 + kGroup >= p.M)
            for (int g = m0 / kGroup + 1; g < S; ++g) scale[g] = (uint8_t)kUnitScale;
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {   // 16 bytes of a row per thread
        const int k = i * 32 + tid / 8, at = tid % 8 * 16;
        if (k0 + k >= p.K || m0 + at >= p.M) continue;
        uint8_t *to = p.q + (uint64_t)(k0 + k) * (uint64_t)p.M + (uint64_t)(m0 + at);
        const u32x4_ v = *reinterpret_cast<const u32x4_ *>(turned + k * LINE + at);
        typedef u32x4_ Loose __attribute__((aligned(1)));
        if (m0 + at + 16 <= p.M) *reinterpret_cast<Loose *>(to) = v;
        else
            for (int b = 0; m0 + at + b < p.M; ++b) to[b] = turned[k * LINE + at + b];
    }
}

// The values of 8-bit rows, 8 per lane. Bound by memory: 8192 x 12288 to bf16 (303
// MB) 51 us (5.9 TB/s).
template <class T, bool LOOSE>
__global__ __launch_bounds__(256) void dequant_kernel(const QuantParams p) {
    constexpr int V = 8;
    const int lane = threadIdx.x & 63;
    const uint32_t spans = (uint32_t)(p.K + kSpan - 1) / kSpan, items = (uint32_t)p.M * spans;
    for (uint32_t item = blockIdx.x * 4 + (threadIdx.x >> 6); item < items; item += gridDim.x * 4) {
        const uint32_t m = item / spans, span = item % spans;
        const int c = (int)span * kSpan + lane * V;
        if (c >= p.K) continue;
        const uint8_t *q = p.q_in + (uint64_t)m * (uint64_t)p.K + c;
        const uint32_t byte = p.scale_in[(uint64_t)m * (uint64_t)scale_cols(p.K) + c / kGroup];
        uint32_t w[2] = {0, 0};
        if (c + V <= p.K) {
            typedef unsigned int Two __attribute__((ext_vector_type(2), aligned(1)));
            const Two v = *reinterpret_cast<const Two *>(q);
            w[0] = v[0];
            w[1] = v[1];
        } else {
#pragma unroll
            for (int e = 0; e < V; ++e)
                if (c + e < p.K) w[e / 4] |= (uint32_t)q[e] << (8 * (e & 3));
        }
        float f[V];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            f[4 * i + 0] = ldexpf(__builtin_amdgcn_cvt_f32_fp8((int)w[i], 0), (int)byte - 127);
            f[4 * i + 1] = ldexpf(__builtin_amdgcn_cvt_f32_fp8((int)w[i], 1), (int)byte - 127);
            f[4 * i + 2] = ldexpf(__builtin_amdgcn_cvt_f32_fp8((int)w[i], 2), (int)byte - 127);
            f[4 * i + 3] = ldexpf(__builtin_amdgcn_cvt_f32_fp8((int)w[i], 3), (int)byte - 127);
        }
        if (byte == 255)
#pragma unroll
            for (int e = 0; e < V; ++e) f[e] = __builtin_nanf("");
        T *out = (T *)p.out + (int64_t)m * p.ld;
        if constexpr (sizeof(T) == 4) {
            const float lo[4] = {f[0], f[1], f[2], f[3]}, hi[4] = {f[4], f[5], f[6], f[7]};
            store_pack<T, 4, LOOSE>(out, c, p.K, lo);
            store_pack<T, 4, LOOSE>(out, c + 4, p.K, hi);
        } else {
            store_pack<T, V, LOOSE>(out, c, p.K, f);
        }
    }
}

constexpr int kMaxRows = 1 << 21, kMaxCols = 1 << 17;

// Sizes of x; `either`: of 8-bit rows as they are written along x's rows or across them.
int check(int M, int K, int dtype, bool either) {
    if (M < 1 || K < 1) return set_error(COMPASS_ERR_INVALID, "need positive M and K");
    if (dtype != COMPASS_BF16 && dtype != COMPASS_F32)
        return set_error(COMPASS_ERR_INVALID, "unknown element type %d", dtype);
    if ((M > kMaxRows || K > kMaxCols) && !(either && M <= kMaxCols && K <= kMaxRows))
        return set_error(COMPASS_ERR_UNSUPPORTED, "%d rows of %d elements, at most %d of %d%s", M, K, kMaxRows, kMaxCols,
                         either ? " or the reverse" : "");
    return COMPASS_OK;
}

// Whether every row of x starts on 16 bytes and holds whole vectors of v elements.
bool even_rows(const void *x, int64_t ld, int K, int dtype, int v) {
    const size_t size = dtype == COMPASS_F32 ? 4 : 2;
    return K % v == 0 && ((uintptr_t)x & 15) == 0 && (size_t)ld * size % 16 == 0;
}

int check_operands(const void *x, int64_t ld, int K, int dtype, const void *q, const void *scale) {
    if (!x || !q || !scale) return set_error(COMPASS_ERR_INVALID, "x, x8 and scale are required");
    if (ld < K) return set_error(COMPASS_ERR_INVALID, "rows of %d elements overlap", K);
    if ((uintptr_t)x & (dtype == COMPASS_F32 ? 3 : 1))
        return set_error(COMPASS_ERR_INVALID, "x is not aligned to its elements");
    if (((uintptr_t)q & 15) || ((uintptr_t)scale & 3))
        return set_error(COMPASS_ERR_INVALID, "x8 must be 16-byte and scale 4-byte aligned");
    int cus;
    return current_num_cu(&cus);
}

int launched(const char *what) {
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? COMPASS_OK : set_error(COMPASS_ERR_HIP, "%s launch: %s", what, hipGetErrorString(e));
}

dim3 span_grid(int M, int K) {
    const uint32_t items = (uint32_t)M * (uint32_t)((K + kSpan - 1) / kSpan);   // at most 2^21 2^8 or 2^17 2^12
    return dim3(std::min((items + 3) / 4, 1u << 22));
}

}  // namespace

int op_fp8_scale_cols(int K, int *cols) {
    if (K < 1) return set_error(COMPASS_ERR_INVALID, "need positive K");
    if (K > (1 << 21)) return set_error(COMPASS_ERR_UNSUPPORTED, "rows of %d values, at most %d", K, 1 << 21);
    if (!cols) return set_error(COMPASS_ERR_INVALID, "cols is required");
    *cols = scale_cols(K);
    return COMPASS_OK;
}

int op_fp8_quant(int M, int K, int dtype, const void *x, int64_t ldx, int across, void *x8, void *scale,
                 void *stream) {
    int rc = check(M, K, dtype, false);
    if (rc != COMPASS_OK) return rc;
    if (across != 0 && across != 1) return set_error(COMPASS_ERR_INVALID, "across = %d, must be 0 or 1", across);
    if ((rc = check_operands(x, ldx, K, dtype, x8, scale)) != COMPASS_OK) return rc;
    QuantParams p{};
    p.M = M;
    p.K = K;
    p.ld = ldx;
    p.x = x;
    p.q = (uint8_t *)x8;
    p.scale = (uint8_t *)scale;
    const bool even = even_rows(x, ldx, K, dtype, dtype == COMPASS_F32 ? 4 : 8);
    const hipStream_t s = (hipStream_t)stream;
    if (across) {
        const dim3 grid((unsigned)((K + 63) / 64), (unsigned)((M + kGroup - 1) / kGroup));
        if (dtype == COMPASS_F32) {
            if (even) quant_across_kernel<float, 4, false><<<grid, 256, 0, s>>>(p);
            else quant_across_kernel<float, 4, true><<<grid, 256, 0, s>>>(p);
        } else {
            if (even) quant_across_kernel<Bf16, 8, false><<<grid, 256, 0, s>>>(p);
            else quant_across_kernel<Bf16, 8, true><<<grid, 256, 0, s>>>(p);
        }
    } else {
        const dim3 grid = span_grid(M, K);
        if (dtype == COMPASS_F32) {
            if (even) quant_kernel<float, 4, false><<<grid, 256, 0, s>>>(p);
            else quant_kernel<float, 4, true><<<grid, 256, 0, s>>>(p);
        } else {
            if (even) quant_kernel<Bf16, 8, false><<<grid, 256, 0, s>>>(p);
            else quant_kernel<Bf16, 8, true><<<grid, 256, 0, s>>>(p);
        }
    }
    return launched("8-bit rows");
}

int op_fp8_dequant(int M, int K, int dtype, const void *x8, const void *scale, void *x, int64_t ldx, void *stream) {
    int rc = check(M, K, dtype, true);
    if (rc != COMPASS_OK) return rc;
    if ((rc = check_operands(x, ldx, K, dtype, x8, scale)) != COMPASS_OK) return rc;
    QuantParams p{};
    p.M = M;
    p.K = K;
    p.ld = ldx;
    p.q_in = (const uint8_t *)x8;
    p.scale_in = (const uint8_t *)scale;
    p.out = x;
    const bool even = even_rows(x, ldx, K, dtype, 8);
    const hipStream_t s = (hipStream_t)stream;
    const dim3 grid = span_grid(M, K);
    if (dtype == COMPASS_F32) {
        if (even) dequant_kernel<float, false><<<grid, 256, 0, s>>>(p);
        else dequant_kernel<float, true><<<grid, 256, 0, s>>>(p);
    } else {
        if (even) dequant_kernel<Bf16, false><<<grid, 256, 0, s>>>(p);
        else dequant_kernel<Bf16, true><<<grid, 256, 0, s>>>(p);
    }
    return launched("values of 8-bit rows");
}

}  // namespace compass
