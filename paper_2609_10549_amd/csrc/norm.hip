// Layer norm of a rank's row shard, forward and backward (compass_norm_*).
//
//   mean = sum x / N, rstd = 1 / sqrt(sum (x - mean)^2 / N + eps)
//   xh = (x - mean) rstd, y = xh gamma + beta
//   a = dy gamma, dx = rstd (a - mean(a) - xh mean(a xh))
//   dgamma = sum_m dy xh, dbeta = sum_m dy
//
// A row is read once and stays in the registers of the threads that share it
// (a wave, or a workgroup of up to 1024): the mean, then the sum of squared
// distances from it, both in fp32, then the result. Bound by memory.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "compass.h"
#include "internal.h"
#include "rowops.h"

namespace compass {

namespace {

struct NormParams {
    int M, N;
    int64_t ldx, ldy, lddy, lddx;   // elements between rows
    const void *x, *gamma, *beta, *dy;
    int param_f32;                  // gamma and beta in fp32 (else bf16)
    float eps;
    void *y, *dx;
    float *mean, *rstd;
    const float *mean_in, *rstd_in;
    float *part;                    // backward: [grid][2][N] sums of dy xh and dy
    int want_params;                // whether dgamma or dbeta is wanted
};

// V parameters from element i, `none` where there is no such vector.
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

// TPR threads per row, ITEMS vectors of V elements each.
//
// Bound by memory: 32768 x 8192 bf16 (1.07 GB) 200 us (5.4 TB/s, 211 without
// streaming stores); 8192 x 12288 fp32 140 us (5.7 TB/s); rows of odd length
// reach 3.4 (8192 x 5001 bf16 49 us; by single elements 98).
template <class T, int V, bool LOOSE, int TPR, int ITEMS>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void norm_forward_kernel(const NormParams p) {
    constexpr int THREADS = TPR < 256 ? 256 : TPR;
    __shared__ float s0[THREADS / 64], s1[THREADS / 64];
    const int t = threadIdx.x % TPR;
    const int m = (int)blockIdx.x * (THREADS / TPR) + (int)threadIdx.x / TPR;
    if (TPR == 64 && m >= p.M) return;
    const T *x = (const T *)p.x + (int64_t)m * p.ldx;
    float f[ITEMS][V];
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        unpack(load_pack<T, V, LOOSE>(x, (i * TPR + t) * V, p.N), f[i]);
#pragma unroll
        for (int e = 0; e < V; ++e) sum += f[i][e];
    }
    const float mean = row_sum<TPR>(sum, s0) / (float)p.N;
    float sq = 0.0f;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i)
#pragma unroll
        for (int e = 0; e < V; ++e) {
            f[i][e] -= mean;
            if ((i * TPR + t) * V + (LOOSE ? e : 0) < p.N) sq += f[i][e] * f[i][e];
        }
    const float rstd = 1.0f / sqrtf(row_sum<TPR>(sq, s1) / (float)p.N + p.eps);
    T *y = (T *)p.y + (int64_t)m * p.ldy;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const int c = (i * TPR + t) * V;
        float g[V], b[V];
        load_param<V, LOOSE>(p.gamma, p.param_f32, 1.0f, c, p.N, g);
        load_param<V, LOOSE>(p.beta, p.param_f32, 0.0f, c, p.N, b);
#pragma unroll
        for (int e = 0; e < V; ++e) f[i][e] = f[i][e] * rstd * g[e] + b[e];
        store_pack<T, V, LOOSE>(y, c, p.N, f[i]);
    }
    if (t == 0) {
        p.mean[m] = mean;
        p.rstd[m] = rstd;
    }
}

// Threads of a backward workgroup whose rows take TPR threads each.
constexpr int backward_threads(int tpr) { return tpr > 512 ? tpr : tpr % 192 == 0 ? 768 : 1024; }

// One workgroup per CU, 768 or 1024 threads: groups of TPR threads take a row
// each, every (gridDim x groups)-th, load the next while they work on one, and
// keep their columns' sums of dy xh and dy in registers to the end. What is
// held of a row between the two passes over it is what was loaded (x and dy as
// they lie), so that a row, the next one, gamma and the sums fit 128 registers.
//
// Bound by memory: a row's x and dy in, dx out. Each workgroup leaves 2 N sums,
// so few workgroups keep that traffic small. With the sums' join, bf16: 8192 x
// 12288 130 us (604 MB at 4.65 TB/s), without the next row's loads 149, with
// 512 workgroups 152; 32768 x 8192 310 us (5.2 TB/s); 8192 x 2048 27 us, as
// 1024 workgroups of 256 threads 50.
template <class T, int V, bool LOOSE, int TPR, int ITEMS>
__global__ __launch_bounds__(backward_threads(TPR)) void norm_backward_kernel(const NormParams p) {
    constexpr int THREADS = backward_threads(TPR), ROWS = THREADS / TPR, WAVES = TPR / 64;
    constexpr bool AHEAD = THREADS * V * ITEMS < 16384;   // else the next row has no registers
    __shared__ float2 s[2][THREADS / 64];
    __shared__ float comb[ROWS > 1 ? THREADS * V * 2 : 1];
    const int place = threadIdx.x % TPR, r = threadIdx.x / TPR;
    float g[ITEMS][V], dg[ITEMS][V], db[ITEMS][V];
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        load_param<V, LOOSE>(p.gamma, p.param_f32, 1.0f, (i * TPR + place) * V, p.N, g[i]);
#pragma unroll
        for (int e = 0; e < V; ++e) dg[i][e] = db[i][e] = 0.0f;
    }
    const int step = (int)gridDim.x * ROWS;
    const float inv = 1.0f / (float)p.N;
    Pack<T, V> nx[ITEMS], nd[ITEMS];
    float n_mean = 0.0f, n_rstd = 0.0f;
    auto fetch = [&](int m, int t) {
        const T *x = (const T *)p.x + (int64_t)m * p.ldx, *dy = (const T *)p.dy + (int64_t)m * p.lddy;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            nx[i] = load_pack<T, V, LOOSE>(x, (i * TPR + t) * V, p.N);
            nd[i] = load_pack<T, V, LOOSE>(dy, (i * TPR + t) * V, p.N);
        }
        n_mean = p.mean_in[m];
        n_rstd = p.rstd_in[m];
    };
    const int m0 = (int)blockIdx.x * ROWS;
    if (AHEAD && m0 + r < p.M) fetch(m0 + r, place);
    int par = 0;
    for (int mb = m0; mb < p.M; mb += step, par ^= 1) {   // the same count for all groups: they share barriers
        const int m = mb + r;
        const bool row = m < p.M;
        // (the longest loose bf16 rows: what follows from the place in the row is
        // worked out for each row, as kept over the loop it would be spilled; 8192 x
        // 8191 123 -> 124 us, x 6151 85 -> 90)
        int t = place;
        if constexpr (!AHEAD && LOOSE && sizeof(T) == 2) asm volatile("" : "+v"(t));
        if (!AHEAD && row) fetch(m, t);
        Pack<T, V> cx[ITEMS], cd[ITEMS];
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            cx[i] = nx[i];
            cd[i] = nd[i];
        }
        const float mean = n_mean, rstd = n_rstd;
        if (AHEAD && m + step < p.M) fetch(m + step, t);
        float c1 = 0.0f, c2 = 0.0f;
        if (row) {
#pragma unroll
            for (int i = 0; i < ITEMS; ++i) {
                float x[V], d[V];
                unpack(cx[i], x);
                unpack(cd[i], d);
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float xh = (x[e] - mean) * rstd, a = d[e] * g[i][e];   // past the row's end d is 0
                    dg[i][e] += d[e] * xh;
                    db[i][e] += d[e];
                    c1 += a;
                    c2 += a * xh;
                }
            }
        }
        c1 = wave_sum(c1);
        c2 = wave_sum(c2);
        if constexpr (WAVES > 1) {
            // the two halves of s by turns: a wave writes one again only
            // behind the next row's barrier, when all have read it
            if ((threadIdx.x & 63) == 0) s[par][threadIdx.x >> 6] = make_float2(c1, c2);
            __syncthreads();
            c1 = s[par][r * WAVES].x;
            c2 = s[par][r * WAVES].y;
#pragma unroll
            for (int w = 1; w < WAVES; ++w) {
                c1 += s[par][r * WAVES + w].x;
                c2 += s[par][r * WAVES + w].y;
            }
        }
        if (!row) continue;
        c1 *= inv;
        c2 *= inv;
        T *dx = (T *)p.dx + (int64_t)m * p.lddx;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            float x[V], d[V], o[V];
            unpack(cx[i], x);
            unpack(cd[i], d);
#pragma unroll
            for (int e = 0; e < V; ++e) o[e] = rstd * (d[e] * g[i][e] - c1 - (x[e] - mean) * rstd * c2);
            store_pack<T, V, LOOSE>(dx, (i * TPR + t) * V, p.N, o);
        }
    }
    if (!p.want_params) return;
    float *part = p.part + (size_t)blockIdx.x * 2 * (size_t)p.N;
    auto put = [&](int c, int kind, float x) {
        if (c < p.N) part[(size_t)kind * (size_t)p.N + c] = x;
    };
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        if constexpr (ROWS > 1) {   // one sum per workgroup, in row order, dealt to all its threads
            __syncthreads();
#pragma unroll
            for (int e = 0; e < V; ++e) {
                comb[(2 * e + 0) * THREADS + threadIdx.x] = dg[i][e];
                comb[(2 * e + 1) * THREADS + threadIdx.x] = db[i][e];
            }
            __syncthreads();
            for (int at = threadIdx.x; at < 2 * V * TPR; at += THREADS) {
                const int e2 = at / TPR, tt = at % TPR;
                const float *from = comb + e2 * THREADS + tt;
                float x = from[0];
#pragma unroll
                for (int q = 1; q < ROWS; ++q) x += from[q * TPR];
                put((i * TPR + tt) * V + e2 / 2, e2 & 1, x);
            }
        } else {
#pragma unroll
            for (int e = 0; e < V; ++e) {
                put((i * TPR + place) * V + e, 0, dg[i][e]);
                put((i * TPR + place) * V + e, 1, db[i][e]);
            }
        }
    }
}

// dgamma and dbeta from `parts` rows of 2 N sums: 64 columns per workgroup, 16
// waves that take every 16th row, joined in wave order.
__global__ __launch_bounds__(1024) void norm_params_kernel(int N, int parts, const float *__restrict__ part,
                                                           float *dgamma, float *dbeta) {
    __shared__ float s[16][64];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int c = (int)blockIdx.x * 64 + lane;
    float sum = 0.0f;
    if (c < 2 * N) {
#pragma unroll 8
        for (int i = w; i < parts; i += 16) sum += part[(size_t)i * 2 * (size_t)N + c];
    }
    s[w][lane] = sum;
    __syncthreads();
    if (w != 0 || c >= 2 * N) return;
#pragma unroll
    for (int i = 1; i < 16; ++i) sum += s[i][lane];
    if (c < N) {
        if (dgamma) dgamma[c] = sum;
    } else if (dbeta) {
        dbeta[c - N] = sum;
    }
}

constexpr int kMaxCols = 16384;   // a row's elements in 1024 threads' registers, 16 each
constexpr int kMaxRows = 1 << 21; // 1024 threads each, below the 2^32 of a launch

int hip_error(hipError_t e, const char *what) {
    return set_error(COMPASS_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

// Workgroups of the backward pass: at most one per CU.
constexpr int kMaxParts = 256;

struct Launch {
    const NormParams &p;
    hipStream_t stream;
    int parts;
    template <class T, int V, bool LOOSE, int TPR, int ITEMS>
    void forward() {
        constexpr int THREADS = TPR < 256 ? 256 : TPR, ROWS = THREADS / TPR;
        norm_forward_kernel<T, V, LOOSE, TPR, ITEMS>
            <<<dim3((unsigned)((p.M + ROWS - 1) / ROWS)), THREADS, 0, stream>>>(p);
    }
    template <class T, int V, bool LOOSE, int TPR, int ITEMS>
    void backward() {
        constexpr int THREADS = backward_threads(TPR), ROWS = THREADS / TPR;
        parts = std::min((p.M + ROWS - 1) / ROWS, kMaxParts);
        norm_backward_kernel<T, V, LOOSE, TPR, ITEMS><<<dim3((unsigned)parts), THREADS, 0, stream>>>(p);
    }
    // the fewest threads (and vectors each) that hold a row
    template <class T, int V, bool LOOSE>
    void pick(bool back) {
        const int n = (p.N + V - 1) / V;
        if (back) {
            if (n <= 64) backward<T, V, LOOSE, 64, 1>();
            else if (n <= 128) backward<T, V, LOOSE, 64, 2>();
            else if (n <= 256) backward<T, V, LOOSE, 128, 2>();
            else if (n <= 384) backward<T, V, LOOSE, 192, 2>();
            else if (n <= 512) backward<T, V, LOOSE, 256, 2>();
            else if (n <= 768) backward<T, V, LOOSE, 384, 2>();
            else if (n <= 1024) backward<T, V, LOOSE, 512, 2>();
            else if (n <= 1536) backward<T, V, LOOSE, 768, 2>();
            else if (n <= 2048) backward<T, V, LOOSE, 1024, 2>();
            else if constexpr (V == 4) {
                if (n <= 3072) backward<T, V, LOOSE, 1024, 3>();
                else backward<T, V, LOOSE, 1024, 4>();
            }
            return;
        }
        if (n <= 64) forward<T, V, LOOSE, 64, 1>();
        else if (n <= 128) forward<T, V, LOOSE, 64, 2>();
        else if (n <= 256) forward<T, V, LOOSE, 256, 1>();
        else if (n <= 512) forward<T, V, LOOSE, 256, 2>();
        else if (n <= 1024) forward<T, V, LOOSE, 512, 2>();
        else if (n <= 2048) forward<T, V, LOOSE, 1024, 2>();
        else if constexpr (V == 4) forward<T, V, LOOSE, 1024, 4>();
    }
};

bool aligned16(const void *p, int64_t ld, size_t size) {
    return ((uintptr_t)p & 15) == 0 && (size_t)ld * size % 16 == 0;
}

// 16-byte vectors: aligned ones where every row of every operand starts on 16
// bytes and holds whole vectors, loose ones otherwise.
int launch(const NormParams &p, int dtype, bool backward, hipStream_t stream) {
    const size_t size = dtype == COMPASS_F32 ? 4 : 2;
    const int64_t v = (int64_t)(16 / size);
    bool even = p.N % v == 0 && aligned16(p.x, p.ldx, size) && ((uintptr_t)p.gamma & 15) == 0;
    if (backward) even = even && aligned16(p.dy, p.lddy, size) && aligned16(p.dx, p.lddx, size);
    else even = even && aligned16(p.y, p.ldy, size) && ((uintptr_t)p.beta & 15) == 0;
    Launch l{p, stream, 0};
    if (dtype == COMPASS_F32) {
        if (even) l.pick<float, 4, false>(backward);
        else l.pick<float, 4, true>(backward);
    } else {
        if (even) l.pick<Bf16, 8, false>(backward);
        else l.pick<Bf16, 8, true>(backward);
    }
    return l.parts;
}

int check(int M, int N, int dtype, int ptype) {
    if (M < 1 || N < 1) return set_error(COMPASS_ERR_INVALID, "need positive M and N");
    if ((dtype != COMPASS_BF16 && dtype != COMPASS_F32) || (ptype != COMPASS_BF16 && ptype != COMPASS_F32))
        return set_error(COMPASS_ERR_INVALID, "unknown element type %d or %d", dtype, ptype);
    if (N > kMaxCols || M > kMaxRows)
        return set_error(COMPASS_ERR_UNSUPPORTED, "%d rows of %d elements, at most %d of %d", M, N, kMaxRows, kMaxCols);
    return COMPASS_OK;
}

bool off_element(const void *p, int dtype) { return ((uintptr_t)p & (dtype == COMPASS_F32 ? 3 : 1)) != 0; }

}  // namespace

int op_norm_forward(int M, int N, int dtype, int ptype, const void *x, int64_t ldx, const void *gamma,
                    const void *beta, float eps, void *y, int64_t ldy, float *mean, float *rstd, void *stream) {
    int rc = check(M, N, dtype, ptype);
    if (rc != COMPASS_OK) return rc;
    if (!x || !y || !mean || !rstd) return set_error(COMPASS_ERR_INVALID, "x, y, mean and rstd are required");
    if (ldx < N || ldy < N) return set_error(COMPASS_ERR_INVALID, "rows of %d elements overlap", N);
    if (!(eps >= 0.0f)) return set_error(COMPASS_ERR_INVALID, "eps must not be negative");
    if (off_element(x, dtype) || off_element(y, dtype) || off_element(gamma, ptype) || off_element(beta, ptype))
        return set_error(COMPASS_ERR_INVALID, "an operand is not aligned to its elements");
    int cus;
    if ((rc = current_num_cu(&cus)) != COMPASS_OK) return rc;
    NormParams p{};
    p.M = M;
    p.N = N;
    p.ldx = ldx;
    p.ldy = ldy;
    p.x = x;
    p.gamma = gamma;
    p.beta = beta;
    p.param_f32 = ptype == COMPASS_F32;
    p.eps = eps;
    p.y = y;
    p.mean = mean;
    p.rstd = rstd;
    launch(p, dtype, false, (hipStream_t)stream);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? COMPASS_OK : hip_error(e, "layer norm launch");
}

int op_norm_workspace(int M, int N, size_t *bytes) {
    const int rc = check(M, N, COMPASS_BF16, COMPASS_BF16);
    if (rc != COMPASS_OK) return rc;
    if (!bytes) return set_error(COMPASS_ERR_INVALID, "bytes is required");
    *bytes = (size_t)std::min(M, kMaxParts) * 2 * (size_t)N * 4;
    return COMPASS_OK;
}

int op_norm_backward(int M, int N, int dtype, int ptype, const void *dy, int64_t lddy, const void *x, int64_t ldx,
                     const void *gamma, const float *mean, const float *rstd, void *dx, int64_t lddx, float *dgamma,
                     float *dbeta, void *ws, size_t ws_bytes, void *stream) {
    int rc = check(M, N, dtype, ptype);
    if (rc != COMPASS_OK) return rc;
    if (!dy || !x || !mean || !rstd || !dx)
        return set_error(COMPASS_ERR_INVALID, "dy, x, mean, rstd and dx are required");
    if (lddy < N || ldx < N || lddx < N) return set_error(COMPASS_ERR_INVALID, "rows of %d elements overlap", N);
    if (off_element(dy, dtype) || off_element(x, dtype) || off_element(dx, dtype) || off_element(gamma, ptype))
        return set_error(COMPASS_ERR_INVALID, "an operand is not aligned to its elements");
    size_t need = 0;
    op_norm_workspace(M, N, &need);
    if (dgamma || dbeta) {
        if (!ws || ((uintptr_t)ws & 15) || ws_bytes < need)
            return set_error(COMPASS_ERR_INVALID, "workspace of %zu bytes (16-byte aligned), need %zu", ws_bytes, need);
    }
    int cus;
    if ((rc = current_num_cu(&cus)) != COMPASS_OK) return rc;
    NormParams p{};
    p.M = M;
    p.N = N;
    p.ldx = ldx;
    p.lddy = lddy;
    p.lddx = lddx;
    p.x = x;
    p.dy = dy;
    p.gamma = gamma;
    p.param_f32 = ptype == COMPASS_F32;
    p.dx = dx;
    p.mean_in = mean;
    p.rstd_in = rstd;
    p.part = (float *)ws;
    p.want_params = dgamma || dbeta;
    const int parts = launch(p, dtype, true, (hipStream_t)stream);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return hip_error(e, "layer norm launch");
    if (p.want_params) {
        norm_params_kernel<<<dim3((unsigned)((2 * N + 63) / 64)), 1024, 0, (hipStream_t)stream>>>(N, parts, p.part,
                                                                                               dgamma, dbeta);
        if ((e = hipGetLastError()) != hipSuccess) return hip_error(e, "weight gradient launch");
    }
    return COMPASS_OK;
}

}  // namespace compass
