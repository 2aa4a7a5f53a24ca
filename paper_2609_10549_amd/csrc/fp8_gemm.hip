// Products of 8-bit rows (fp8.h): an 8-bit product and a weight's gradient from an
// activation kept in 8 bits.
//
//   compass_fp8_gemm:  C[m][n] = sum_g 2^(sa[m][g] + sw[n][g]) sum_{k in g} A[m][k] W[n][k]
//   compass_fp8_wgrad: dW[n][k] = sum_m dY[m][n] X[m][k] 2^sx[m][k / 128]
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "compass.h"
#include "fp8.h"
#include "gemm_core.h"
#include "internal.h"

namespace compass {

namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));

struct ProductParams {
    const uint8_t *A, *W, *sA, *sW;
    uint16_t *C;
    int M, N, K;
};

// 64 x 64 tiles, 4 waves of 32 x 32, a group of 128 per stage.
__global__ __launch_bounds__(256) void product_kernel(const ProductParams p) {
    __shared__ __attribute__((aligned(16))) uint8_t s[2][64 * 128];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int m0 = (int)blockIdx.y * 64, n0 = (int)blockIdx.x * 64;
    const int r = lane & 15, kq = lane >> 4, wm = (wave >> 1) * 32, wn = (wave & 1) * 32;
    const int S = scale_cols(p.K), G = (p.K + kGroup - 1) / kGroup;
    f32x4 acc[2][2];
    for (int i = 0; i < 2; ++i)
        for (int j = 0; j < 2; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    for (int g = 0; g < G; ++g) {
        __syncthreads();
        for (int i = 0; i < 4; ++i) {
            const int at = i * 256 + tid, op = at / 512, row = at % 512 / 8, chunk = at % 8, k = g * kGroup + chunk * 16;
            const int d = (op ? n0 : m0) + row;
            u32x4 v = u32x4{0, 0, 0, 0};
            if (d < (op ? p.N : p.M) && k < p.K)
                v = *reinterpret_cast<const u32x4 *>((op ? p.W : p.A) + (size_t)d * (size_t)p.K + k);
            *reinterpret_cast<u32x4 *>(&s[op][row * 128 + ((chunk ^ (row & 7)) * 16)]) = v;
        }
        __syncthreads();
        i32x8 a[2], b[2];
        int sa[2], sw[2];
        for (int i = 0; i < 2; ++i) {
            for (int h = 0; h < 2; ++h) {
                const int ra = wm + i * 16 + r, rb = wn + i * 16 + r, c = kq * 2 + h;
                const i32x4 x = *reinterpret_cast<const i32x4 *>(&s[0][ra * 128 + ((c ^ (ra & 7)) * 16)]);
                const i32x4 y = *reinterpret_cast<const i32x4 *>(&s[1][rb * 128 + ((c ^ (rb & 7)) * 16)]);
                for (int e = 0; e < 4; ++e) {
                    a[i][4 * h + e] = x[e];
                    b[i][4 * h + e] = y[e];
                }
            }
            const int m = min(m0 + wm + i * 16 + r, p.M - 1), n = min(n0 + wn + i * 16 + r, p.N - 1);
            sa[i] = p.sA[(size_t)m * S + g];
            sw[i] = p.sW[(size_t)n * S + g];
        }
        for (int i = 0; i < 2; ++i)
            for (int j = 0; j < 2; ++j)
                acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b[j], a[i], acc[i][j], 0, 0, 0, sw[j], 0, sa[i]);
    }
    // a lane holds row r, columns 4 kq + 0..3 of a block
    for (int i = 0; i < 2; ++i)
        for (int j = 0; j < 2; ++j)
            for (int e = 0; e < 4; ++e) {
                const int m = m0 + wm + i * 16 + r, n = n0 + wn + j * 16 + 4 * kq + e;
                if (m < p.M && n < p.N) p.C[(size_t)m * (size_t)p.N + n] = (uint16_t)pack_bf16x2(acc[i][j][e], 0.0f);
            }
}

struct GradParams {
    const uint16_t *dY;
    const uint8_t *X, *sX;
    void *dW;
    int M, N, K, f32, accumulate;
};

// 64 x 64 tiles of dW, 32 rows of the reduction per stage: both operands turned
// on their way to LDS, X's values put to bf16 (exactly: four bits and a power of
// two).
__global__ __launch_bounds__(256) void grad_kernel(const GradParams p) {
    __shared__ __attribute__((aligned(16))) uint16_t s[2][64][40];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int n0 = (int)blockIdx.y * 64, k0 = (int)blockIdx.x * 64;
    const int r = lane & 15, kq = lane >> 4, wm = (wave >> 1) * 32, wn = (wave & 1) * 32;
    const int S = scale_cols(p.K);
    f32x4 acc[2][2];
    for (int i = 0; i < 2; ++i)
        for (int j = 0; j < 2; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    for (int mb = 0; mb < p.M; mb += 32) {
        __syncthreads();
        for (int i = 0; i < 8; ++i) {
            const int at = i * 256 + tid, row = at / 64, col = at % 64, m = mb + row;
            uint16_t y = 0, x = 0;
            if (m < p.M && n0 + col < p.N) y = p.dY[(size_t)m * (size_t)p.N + n0 + col];
            if (m < p.M && k0 + col < p.K) {
                const int k = k0 + col;
                const uint32_t byte = p.sX[(size_t)m * S + k / kGroup];
                float v = ldexpf(__builtin_amdgcn_cvt_f32_fp8((int)p.X[(size_t)m * (size_t)p.K + k], 0), (int)byte - 127);
                if (byte == 255) v = __builtin_nanf("");
                x = (uint16_t)pack_bf16x2(v, 0.0f);
            }
            s[0][col][row] = y;
            s[1][col][row] = x;
        }
        __syncthreads();
        bf16x8 a[2], b[2];
        for (int i = 0; i < 2; ++i) {
            a[i] = *reinterpret_cast<const bf16x8 *>(&s[0][wm + i * 16 + r][kq * 8]);
            b[i] = *reinterpret_cast<const bf16x8 *>(&s[1][wn + i * 16 + r][kq * 8]);
        }
        for (int i = 0; i < 2; ++i)
            for (int j = 0; j < 2; ++j)
                acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b[j], a[i], acc[i][j], 0, 0, 0);
    }
    for (int i = 0; i < 2; ++i)
        for (int j = 0; j < 2; ++j)
            for (int e = 0; e < 4; ++e) {
                const int n = n0 + wm + i * 16 + r, k = k0 + wn + j * 16 + 4 * kq + e;
                if (n >= p.N || k >= p.K) continue;
                const size_t at = (size_t)n * (size_t)p.K + k;
                float x = acc[i][j][e];
                if (p.f32) {
                    float *to = (float *)p.dW + at;
                    *to = p.accumulate ? *to + x : x;
                } else {
                    uint16_t *to = (uint16_t *)p.dW + at;
                    if (p.accumulate) x += __builtin_bit_cast(float, (uint32_t)*to << 16);
                    *to = (uint16_t)pack_bf16x2(x, 0.0f);
                }
            }
}

constexpr int kMaxRows = 1 << 20, kMaxDepth = 1 << 17;

int check_sizes(int M, int N, int K, bool grad) {
    if (M < 1 || N < 1 || K < 1 || K % 16 || (grad && N % 8))
        return set_error(COMPASS_ERR_INVALID, "need positive M, N and K with K a multiple of 16%s",
                         grad ? ", N of 8" : "");
    if (M > kMaxRows || N > kMaxRows || K > kMaxDepth)
        return set_error(COMPASS_ERR_UNSUPPORTED, "M = %d, N = %d, K = %d beyond %d, %d, %d", M, N, K, kMaxRows, kMaxRows,
                         kMaxDepth);
    return COMPASS_OK;
}

bool misaligned(const void *p) { return ((uintptr_t)p & 15) != 0; }

}  // namespace

int op_fp8_gemm_workspace(int M, int N, int K, size_t *bytes) {
    const int rc = check_sizes(M, N, K, false);
    if (rc != COMPASS_OK) return rc;
    if (!bytes) return set_error(COMPASS_ERR_INVALID, "bytes is required");
    *bytes = 0;
    return COMPASS_OK;
}

int op_fp8_gemm(int M, int N, int K, const void *A, const void *A_scale, const void *W, const void *W_scale, void *C,
                void *ws, size_t ws_bytes, void *stream) {
    int rc = check_sizes(M, N, K, false);
    if (rc != COMPASS_OK) return rc;
    if (!A || !A_scale || !W || !W_scale || !C)
        return set_error(COMPASS_ERR_INVALID, "A, W, their scales and C are required");
    if (misaligned(A) || misaligned(W) || misaligned(C) || ((uintptr_t)A_scale & 3) || ((uintptr_t)W_scale & 3))
        return set_error(COMPASS_ERR_INVALID, "A, W and C must be 16-byte and the scales 4-byte aligned");
    int cus;
    if ((rc = current_num_cu(&cus)) != COMPASS_OK) return rc;
    const ProductParams p{(const uint8_t *)A, (const uint8_t *)W, (const uint8_t *)A_scale, (const uint8_t *)W_scale,
                          (uint16_t *)C, M, N, K};
    product_kernel<<<dim3((unsigned)((N + 63) / 64), (unsigned)((M + 63) / 64)), 256, 0, (hipStream_t)stream>>>(p);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? COMPASS_OK : set_error(COMPASS_ERR_HIP, "8-bit product launch: %s", hipGetErrorString(e));
}

int op_fp8_wgrad_workspace(int M, int N, int K, size_t *bytes) {
    const int rc = check_sizes(M, N, K, true);
    if (rc != COMPASS_OK) return rc;
    if (!bytes) return set_error(COMPASS_ERR_INVALID, "bytes is required");
    *bytes = 0;
    return COMPASS_OK;
}

int op_fp8_wgrad(int M, int N, int K, int gtype, const void *dY, const void *X, const void *X_scale, void *dW,
                 int accumulate, void *ws, size_t ws_bytes, void *stream) {
    int rc = check_sizes(M, N, K, true);
    if (rc != COMPASS_OK) return rc;
    if (gtype != COMPASS_BF16 && gtype != COMPASS_F32)
        return set_error(COMPASS_ERR_INVALID, "unknown element type %d", gtype);
    if (accumulate != 0 && accumulate != 1)
        return set_error(COMPASS_ERR_INVALID, "accumulate = %d, must be 0 or 1", accumulate);
    if (!dY || !X || !X_scale || !dW) return set_error(COMPASS_ERR_INVALID, "dY, X8, its scale and dW are required");
    if (misaligned(dY) || misaligned(X) || misaligned(dW) || ((uintptr_t)X_scale & 3))
        return set_error(COMPASS_ERR_INVALID, "dY, X8 and dW must be 16-byte and the scale 4-byte aligned");
    int cus;
    if ((rc = current_num_cu(&cus)) != COMPASS_OK) return rc;
    const GradParams p{(const uint16_t *)dY, (const uint8_t *)X, (const uint8_t *)X_scale, dW, M, N, K,
                       gtype == COMPASS_F32, accumulate};
    grad_kernel<<<dim3((unsigned)((K + 63) / 64), (unsigned)((N + 63) / 64)), 256, 0, (hipStream_t)stream>>>(p);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? COMPASS_OK : set_error(COMPASS_ERR_HIP, "weight gradient launch: %s", hipGetErrorString(e));
}

}  // namespace compass
