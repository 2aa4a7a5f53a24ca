// Root-mean-square norm of a rank's row shard with the residual's addition,
// forward and backward (compass_rms_*).
//
//   h = x + residual, rounded to the stream's type
//   rstd = 1 / sqrt(sum h^2 / N + eps), y = h rstd gamma
//   hh = h rstd, a = dy gamma, dx = dh + rstd (a - hh mean(a hh))
//   dgamma = sum_m dy hh
//
// The norm is of h as it is stored, so that the backward pass, which reads it, is
// the gradient of what ran. y leaves in the stream's type, in 8 bits (fp8.h)
// straight from the fp32 values, or both. A row is read once and stays in the
// registers of the threads that share it; the sum of squares is fp32. Bound by
// memory.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "compass.h"
#include "fp8.h"
#include "internal.h"
#include "rowops.h"

namespace compass {

namespace {

struct RmsParams {
    int M, N;
    int64_t ldx, ldr, ldh, ldy, lddy, lddh, lddx;   // elements between rows
    const void *x, *residual, *gamma, *dy, *dh;
    int param_f32;                  // gamma in fp32 (else bf16)
    float eps;
    void *h, *y, *dx;
    uint8_t *y8, *scale;            // rows of N and of scale_cols(N) bytes
    float *rstd;
    const void *h_in;
    const float *rstd_in;
    float *part;                    // backward: [grid][N] sums of dy hh
    int want_gamma;
};

// TPR threads per row, ITEMS vectors of V elements each; EIGHT: y in 8 bits too, a
// group's largest value from the 16 lanes (fp32: 32) that hold it.
//
// Bound by memory: 32768 x 8192 bf16 with the residual (2.15 GB) 364 us (5.9 TB/s);
// 8192 x 12288 bf16 with the residual to 8 bits (0.70 GB) 130 us (5.4 TB/s). Single
// tokens are bound by latency, the loads, the sum over a workgroup's waves and the
// stores of a row one after another: 1 x 12288 4.1 us, 4 rows 4.6 to 4.8, 256 (one
// per CU) 6.0.
template <class T, int V, bool LOOSE, int TPR, int ITEMS, bool EIGHT>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void rms_forward_kernel(const RmsParams p) {
    constexpr int THREADS = TPR < 256 ? 256 : TPR;
    __shared__ float s0[THREADS / 64];
    const int t = threadIdx.x % TPR;
    const int m = (int)blockIdx.x * (THREADS / TPR) + (int)threadIdx.x / TPR;
    if (TPR == 64 && m >= p.M) return;
    const T *x = (const T *)p.x + (int64_t)m * p.ldx;
    float f[ITEMS][V];
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) unpack(load_pack<T, V, LOOSE>(x, (i * TPR + t) * V, p.N), f[i]);
    if (p.residual) {
        const T *r = (const T *)p.residual + (int64_t)m * p.ldr;
        Pack<T, V> q[ITEMS];
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) q[i] = load_pack<T, V, LOOSE>(r, (i * TPR + t) * V, p.N);
        T *h = (T *)p.h + (int64_t)m * p.ldh;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            float g[V];
            unpack(q[i], g);
#pragma unroll
            for (int e = 0; e < V; ++e) f[i][e] += g[e];
            store_pack<T, V, LOOSE>(h, (i * TPR + t) * V, p.N, f[i]);
            unpack(pack<T, V>(f[i]), f[i]);
        }
    }
    float sq = 0.0f;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i)
#pragma unroll
        for (int e = 0; e < V; ++e) sq += f[i][e] * f[i][e];
    const float rstd = 1.0f / sqrtf(row_sum<TPR>(sq, s0) / (float)p.N + p.eps);
    T *y = (T *)p.y + (int64_t)m * p.ldy;
    uint8_t *y8 = p.y8 + (int64_t)m * p.N, *scale = p.scale + (int64_t)m * scale_cols(p.N);
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const int c = (i * TPR + t) * V;
        float g[V];
        load_param<V, LOOSE>(p.gamma, p.param_f32, 1.0f, c, p.N, g);
#pragma unroll
        for (int e = 0; e < V; ++e) {
            f[i][e] = f[i][e] * rstd * g[e];
            // (past the row's end h is 0, but gamma may be what lies there)
            if (EIGHT && c + e >= p.N) f[i][e] = 0.0f;
        }
        if (!EIGHT || p.y) store_pack<T, V, LOOSE>(y, c, p.N, f[i]);
        if constexpr (EIGHT) store_e4m3<V>(y8, scale, c, p.N, f[i]);
    }
    if constexpr (EIGHT) {
        const int used = (p.N + kGroup - 1) / kGroup;
        if (t < scale_cols(p.N) - used) scale[used + t] = (uint8_t)kUnitScale;
    }
    if (t == 0) p.rstd[m] = rstd;
}

// Threads of a backward workgroup whose rows take TPR threads each.
constexpr int backward_threads(int tpr) { return tpr > 512 ? tpr : tpr % 192 == 0 ? 768 : 1024; }

// One workgroup per CU: groups of TPR threads take a row each, every (gridDim x
// groups)-th, load the next while they work on one, and keep their columns' sums
// of dy hh in registers to the end (each workgroup leaves N of them, so few
// workgroups keep that traffic small).
//
// Bound by memory: 8192 x 12288 bf16 with dh (805 MB) 151 us (5.3 TB/s), the join of
// the sums 5. Lengths whose registers hold no row ahead, with the join: 8192 x 4096 56 us
// (4.8 TB/s), 8192 x 8192 105 (5.1). Few rows, latency: 2048 x 4096 19 us with the join
// (3.5 TB/s); 1000 x 4097 fp32 16.4, four rows one after another per workgroup, whose
// 1536 places take 1025 vectors.
template <class T, int V, bool LOOSE, int TPR, int ITEMS>
__global__ __launch_bounds__(backward_threads(TPR)) void rms_backward_kernel(const RmsParams p) {
    constexpr int THREADS = backward_threads(TPR), ROWS = THREADS / TPR, WAVES = TPR / 64;
    // (beyond, the next row has no registers)
    constexpr bool AHEAD = THREADS * ITEMS <= (sizeof(T) == 2 ? 1536 : 2048);
    __shared__ float s[2][THREADS / 64];
    __shared__ float comb[ROWS > 1 ? THREADS * V : 1];
    const int place = threadIdx.x % TPR, r = threadIdx.x / TPR;
    float g[ITEMS][V], dg[ITEMS][V];
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        load_param<V, LOOSE>(p.gamma, p.param_f32, 1.0f, (i * TPR + place) * V, p.N, g[i]);
#pragma unroll
        for (int e = 0; e < V; ++e) dg[i][e] = 0.0f;
    }
    const int step = (int)gridDim.x * ROWS;
    const float inv = 1.0f / (float)p.N;
    Pack<T, V> nh[ITEMS], nd[ITEMS], nr[ITEMS];
    float n_rstd = 0.0f;
    auto fetch = [&](int m, int t) {
        const T *h = (const T *)p.h_in + (int64_t)m * p.ldh, *dy = (const T *)p.dy + (int64_t)m * p.lddy;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            nh[i] = load_pack<T, V, LOOSE>(h, (i * TPR + t) * V, p.N);
            nd[i] = load_pack<T, V, LOOSE>(dy, (i * TPR + t) * V, p.N);
        }
        if (p.dh) {
            const T *dh = (const T *)p.dh + (int64_t)m * p.lddh;
#pragma unroll
            for (int i = 0; i < ITEMS; ++i) nr[i] = load_pack<T, V, LOOSE>(dh, (i * TPR + t) * V, p.N);
        }
        n_rstd = p.rstd_in[m];
    };
#pragma unroll
    for (int i = 0; i < ITEMS; ++i)
#pragma unroll
        for (int j = 0; j < Pack<T, V>::Q; ++j) nr[i].q[j] = u32x4_{0, 0, 0, 0};
    const int m0 = (int)blockIdx.x * ROWS;
    if (AHEAD && m0 + r < p.M) fetch(m0 + r, place);
    int par = 0;
    for (int mb = m0; mb < p.M; mb += step, par ^= 1) {   // the same count for all groups: they share barriers
        const int m = mb + r;
        const bool row = m < p.M;
        int t = place;
        if (!AHEAD && row) fetch(m, t);
        Pack<T, V> ch[ITEMS], cd[ITEMS], cr[ITEMS];
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            ch[i] = nh[i];
            cd[i] = nd[i];
            cr[i] = nr[i];
        }
        const float rstd = n_rstd;
        if (AHEAD && m + step < p.M) fetch(m + step, t);
        float c1 = 0.0f;
        if (row) {
#pragma unroll
            for (int i = 0; i < ITEMS; ++i) {
                float h[V], d[V];
                unpack(ch[i], h);
                unpack(cd[i], d);
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float hh = h[e] * rstd;   // past the row's end h and d are 0
                    dg[i][e] += d[e] * hh;
                    c1 += d[e] * g[i][e] * hh;
                }
            }
        }
        c1 = wave_sum(c1);
        if constexpr (WAVES > 1) {
            // the two halves of s by turns: a wave writes one again only
            // behind the next row's barrier, when all have read it
            if ((threadIdx.x & 63) == 0) s[par][threadIdx.x >> 6] = c1;
            __syncthreads();
            c1 = s[par][r * WAVES];
#pragma unroll
            for (int w = 1; w < WAVES; ++w) c1 += s[par][r * WAVES + w];
        }
        if (!row) continue;
        c1 *= inv;
        T *dx = (T *)p.dx + (int64_t)m * p.lddx;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            float h[V], d[V], o[V];
            unpack(ch[i], h);
            unpack(cd[i], d);
            unpack(cr[i], o);
#pragma unroll
            for (int e = 0; e < V; ++e) o[e] += rstd * (d[e] * g[i][e] - h[e] * rstd * c1);
            store_pack<T, V, LOOSE>(dx, (i * TPR + t) * V, p.N, o);
        }
    }
    if (!p.want_gamma) return;
    float *part = p.part + (size_t)blockIdx.x * (size_t)p.N;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        if constexpr (ROWS > 1) {   // one sum per workgroup, in row order, dealt to all its threads
            __syncthreads();
#pragma unroll
            for (int e = 0; e < V; ++e) comb[e * THREADS + threadIdx.x] = dg[i][e];
            __syncthreads();
            for (int at = threadIdx.x; at < V * TPR; at += THREADS) {
                const int e = at / TPR, tt = at % TPR, c = (i * TPR + tt) * V + e;
                const float *from = comb + e * THREADS + tt;
                float x = from[0];
#pragma unroll
                for (int q = 1; q < ROWS; ++q) x += from[q * TPR];
                if (c < p.N) part[c] = x;
            }
        } else {
#pragma unroll
            for (int e = 0; e < V; ++e)
                if (const int c = (i * TPR + place) * V + e; c < p.N) part[c] = dg[i][e];
        }
    }
}

// dgamma from `parts` rows of N sums: 64 columns per workgroup, 16 waves that
// take every 16th row, joined in wave order.
__global__ __launch_bounds__(1024) void rms_weight_kernel(int N, int parts, const float *__restrict__ part,
                                                          float *dgamma) {
    __shared__ float s[16][64];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int c = (int)blockIdx.x * 64 + lane;
    float sum = 0.0f;
    if (c < N) {
#pragma unroll 8
        for (int i = w; i < parts; i += 16) sum += part[(size_t)i * (size_t)N + c];
    }
    s[w][lane] = sum;
    __syncthreads();
    if (w != 0 || c >= N) return;
#pragma unroll
    for (int i = 1; i < 16; ++i) sum += s[i][lane];
    dgamma[c] = sum;
}

constexpr int kMaxCols = 16384;   // a row's elements in 1024 threads' registers, 16 each
constexpr int kMaxRows = 1 << 21; // 1024 threads each, below the 2^32 of a launch
constexpr int kMaxParts = 256;    // workgroups of the backward pass: at most one per CU

int hip_error(hipError_t e, const char *what) {
    return set_error(COMPASS_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

struct Launch {
    const RmsParams &p;
    hipStream_t stream;
    int parts;
    template <class T, int V, bool LOOSE, int TPR, int ITEMS>
    void forward() {
        constexpr int THREADS = TPR < 256 ? 256 : TPR, ROWS = THREADS / TPR;
        const dim3 grid((unsigned)((p.M + ROWS - 1) / ROWS));
        if (p.y8) rms_forward_kernel<T, V, LOOSE, TPR, ITEMS, true><<<grid, THREADS, 0, stream>>>(p);
        else rms_forward_kernel<T, V, LOOSE, TPR, ITEMS, false><<<grid, THREADS, 0, stream>>>(p);
    }
    template <class T, int V, bool LOOSE, int TPR, int ITEMS>
    void backward() {
        constexpr int THREADS = backward_threads(TPR), ROWS = THREADS / TPR;
        parts = std::min((p.M + ROWS - 1) / ROWS, kMaxParts);
        rms_backward_kernel<T, V, LOOSE, TPR, ITEMS><<<dim3((unsigned)parts), THREADS, 0, stream>>>(p);
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
                if (n <= 1024 * 3) backward<T, V, LOOSE, 1024, 3>();
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
int launch(const RmsParams &p, int dtype, bool backward, hipStream_t stream) {
    const size_t size = dtype == COMPASS_F32 ? 4 : 2;
    const int64_t v = (int64_t)(16 / size);
    bool even = p.N % v == 0 && ((uintptr_t)p.gamma & 15) == 0;
    if (backward)
        even = even && aligned16(p.h_in, p.ldh, size) && aligned16(p.dy, p.lddy, size) &&
               aligned16(p.dx, p.lddx, size) && aligned16(p.dh, p.lddh, size);
    else
        even = even && aligned16(p.x, p.ldx, size) && aligned16(p.residual, p.ldr, size) &&
               aligned16(p.h, p.ldh, size) && aligned16(p.y, p.ldy, size);
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

int op_rms_forward(int M, int N, int dtype, int ptype, const void *x, int64_t ldx, const void *residual, int64_t ldr,
                   const void *gamma, float eps, void *h, int64_t ldh, void *y, int64_t ldy, void *y8, void *scale,
                   float *rstd, void *stream) {
    int rc = check(M, N, dtype, ptype);
    if (rc != COMPASS_OK) return rc;
    if (!x || !rstd) return set_error(COMPASS_ERR_INVALID, "x and rstd are required");
    if (!residual != !h) return set_error(COMPASS_ERR_INVALID, "residual and h come together");
    if (!y8 != !scale) return set_error(COMPASS_ERR_INVALID, "y8 and scale come together");
    if (!y && !y8) return set_error(COMPASS_ERR_INVALID, "y, or y8 and scale, are required");
    if (ldx < N || (residual && (ldr < N || ldh < N)) || (y && ldy < N))
        return set_error(COMPASS_ERR_INVALID, "rows of %d elements overlap", N);
    if (!(eps >= 0.0f)) return set_error(COMPASS_ERR_INVALID, "eps must not be negative");
    if (off_element(x, dtype) || off_element(residual, dtype) || off_element(h, dtype) || off_element(y, dtype) ||
        off_element(gamma, ptype) || off_element(rstd, COMPASS_F32))
        return set_error(COMPASS_ERR_INVALID, "an operand is not aligned to its elements");
    if (((uintptr_t)y8 & 15) || ((uintptr_t)scale & 3))
        return set_error(COMPASS_ERR_INVALID, "y8 must be 16-byte and scale 4-byte aligned");
    int cus;
    if ((rc = current_num_cu(&cus)) != COMPASS_OK) return rc;
    RmsParams p{};
    p.M = M;
    p.N = N;
    p.ldx = ldx;
    p.ldr = residual ? ldr : 0;
    p.ldh = residual ? ldh : 0;
    p.ldy = y ? ldy : 0;
    p.x = x;
    p.residual = residual;
    p.gamma = gamma;
    p.param_f32 = ptype == COMPASS_F32;
    p.eps = eps;
    p.h = h;
    p.y = y;
    p.y8 = (uint8_t *)y8;
    p.scale = (uint8_t *)scale;
    p.rstd = rstd;
    launch(p, dtype, false, (hipStream_t)stream);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? COMPASS_OK : hip_error(e, "norm launch");
}

int op_rms_workspace(int M, int N, size_t *bytes) {
    const int rc = check(M, N, COMPASS_BF16, COMPASS_BF16);
    if (rc != COMPASS_OK) return rc;
    if (!bytes) return set_error(COMPASS_ERR_INVALID, "bytes is required");
    *bytes = (size_t)std::min(M, kMaxParts) * (size_t)N * 4;
    return COMPASS_OK;
}

int op_rms_backward(int M, int N, int dtype, int ptype, const void *dy, int64_t lddy, const void *h, int64_t ldh,
                    const void *dh, int64_t lddh, const void *gamma, const float *rstd, void *dx, int64_t lddx,
                    float *dgamma, void *ws, size_t ws_bytes, void *stream) {
    int rc = check(M, N, dtype, ptype);
    if (rc != COMPASS_OK) return rc;
    if (!dy || !h || !rstd || !dx) return set_error(COMPASS_ERR_INVALID, "dy, h, rstd and dx are required");
    if (lddy < N || ldh < N || lddx < N || (dh && lddh < N))
        return set_error(COMPASS_ERR_INVALID, "rows of %d elements overlap", N);
    if (off_element(dy, dtype) || off_element(h, dtype) || off_element(dh, dtype) || off_element(dx, dtype) ||
        off_element(gamma, ptype) || off_element(rstd, COMPASS_F32) || off_element(dgamma, COMPASS_F32))
        return set_error(COMPASS_ERR_INVALID, "an operand is not aligned to its elements");
    size_t need = 0;
    op_rms_workspace(M, N, &need);
    if (dgamma && (!ws || ((uintptr_t)ws & 15) || ws_bytes < need))
        return set_error(COMPASS_ERR_INVALID, "workspace of %zu bytes (16-byte aligned), need %zu", ws_bytes, need);
    int cus;
    if ((rc = current_num_cu(&cus)) != COMPASS_OK) return rc;
    RmsParams p{};
    p.M = M;
    p.N = N;
    p.ldh = ldh;
    p.lddy = lddy;
    p.lddh = dh ? lddh : 0;
    p.lddx = lddx;
    p.h_in = h;
    p.dy = dy;
    p.dh = dh;
    p.gamma = gamma;
    p.param_f32 = ptype == COMPASS_F32;
    p.dx = dx;
    p.rstd_in = rstd;
    p.part = (float *)ws;
    p.want_gamma = dgamma != nullptr;
    const int parts = launch(p, dtype, true, (hipStream_t)stream);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return hip_error(e, "norm launch");
    if (dgamma) {
        rms_weight_kernel<<<dim3((unsigned)((N + 63) / 64)), 1024, 0, (hipStream_t)stream>>>(N, parts, p.part, dgamma);
        if ((e = hipGetLastError()) != hipSuccess) return hip_error(e, "weight gradient launch");
    }
    return COMPASS_OK;
}

}  // namespace compass
