// Embedding lookup and the table's gradient (compass_embed_*).
//
//   y[t] = scale table[ids[t] - v0], zeros where the id is not in the table
//   dtable[v] = scale sum_{t: ids[t] = v0 + v} dy[t]
//
// Gradient: the tokens are sorted by table row (stable, so that each row's sum
// runs in token order whatever the machine does), every table row finds its
// run in the sorted order, and one pass writes the whole table, each element
// once: the sum of the run's rows, or zero. A run of many tokens (frequent
// ones) would be one workgroup's long walk, so runs are cut: blocks of kRun
// sorted positions that lie inside one run are summed first, all at once, and
// the row adds those sums. No floating-point atomics anywhere.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "compass.h"
#include "internal.h"
#include "rowops.h"

namespace compass {

namespace {

constexpr int kRun = 32;

template <class T, int V>
__device__ __forceinline__ void store_vec(T *p, const float (&f)[V]) {
    Pack<T, V> o;
#pragma unroll
    for (int e = 0; e < V; ++e) o.e[e] = from_f32<T>(f[e]);
    *reinterpret_cast<Pack<T, V> *>(p) = o;
}

// One token per blockIdx.x, 256 V columns per blockIdx.y.
template <class T, int V>
__global__ __launch_bounds__(256) void lookup_kernel(int K, int64_t V0, int vocab, const int64_t *__restrict__ ids,
                                                     const T *__restrict__ table, int64_t ldt, float scale, T *y,
                                                     int64_t ldy) {
    const int c = ((int)blockIdx.y * 256 + (int)threadIdx.x) * V;
    if (c >= K) return;
    const int64_t row = ids[blockIdx.x] - V0;
    float f[V];
#pragma unroll
    for (int e = 0; e < V; ++e) f[e] = 0.0f;
    if (row >= 0 && row < vocab) {
        const Pack<T, V> p = *reinterpret_cast<const Pack<T, V> *>(table + row * ldt + c);
#pragma unroll
        for (int e = 0; e < V; ++e) f[e] = to_f32(p.e[e]) * scale;
    }
    store_vec<T, V>(y + (int64_t)blockIdx.x * ldy + c, f);
}

// Table row of a token, `vocab` for ids outside it.
__device__ __forceinline__ int table_row(int64_t id, int64_t v0, int vocab) {
    const int64_t r = id - v0;
    return r >= 0 && r < vocab ? (int)r : vocab;
}

// Stable sort by counting pairs: the place of token t is the number of tokens
// with a smaller row, or the same row and a smaller index. 64 tokens per
// workgroup; each of the 16 waves counts over its share of all tokens, one
// scalar row against 64 lanes at a time.
__global__ __launch_bounds__(1024) void rank_kernel(int T, int64_t v0, int vocab, const int64_t *__restrict__ ids,
                                                    int *order, int *sorted) {
    __shared__ int s[16][64];
    const int lane = threadIdx.x & 63;
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int t0 = (int)blockIdx.x * 64, t = t0 + lane;
    const int key = t < T ? table_row(ids[t], v0, vocab) : vocab;
    const int chunks = (T + 63) / 64;
    int n = 0;
    for (int c = w; c < chunks; c += 16) {
        const int at = c * 64 + lane;
        const int other = at < T ? table_row(ids[at], v0, vocab) : 0x7fffffff;
        if (c == (int)blockIdx.x) {
#pragma unroll 16
            for (int i = 0; i < 64; ++i) {
                const int k = __builtin_amdgcn_readlane(other, i);
                n += k < key || (k == key && i < lane) ? 1 : 0;
            }
        } else {
            const int below = c < (int)blockIdx.x ? key + 1 : key;   // before: k <= key, after: k < key
#pragma unroll 16
            for (int i = 0; i < 64; ++i) n += __builtin_amdgcn_readlane(other, i) < below ? 1 : 0;
        }
    }
    s[w][lane] = n;
    __syncthreads();
    if (w != 0 || t >= T) return;
#pragma unroll
    for (int i = 1; i < 16; ++i) n += s[i][lane];
    order[n] = t;
    sorted[n] = key;
}

// first[v]: the first sorted position whose row is at least v, v in [0, vocab].
__global__ __launch_bounds__(256) void runs_kernel(int T, int vocab, const int *__restrict__ sorted, int *first) {
    const int v = (int)blockIdx.x * 256 + (int)threadIdx.x;
    if (v > vocab) return;
    int lo = 0, hi = T;
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (sorted[mid] < v) lo = mid + 1;
        else hi = mid;
    }
    first[v] = lo;
}

// f += dy of the sorted positions [lo, hi), in order, several rows in flight.
template <class T, int V>
__device__ __forceinline__ void add_rows(float (&f)[V], const int *__restrict__ order, const T *__restrict__ dy,
                                         int64_t ld, int c, int lo, int hi) {
    int i = lo;
    for (; i + 4 <= hi; i += 4) {
        Pack<T, V> p[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) p[j] = *reinterpret_cast<const Pack<T, V> *>(dy + (int64_t)order[i + j] * ld + c);
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int e = 0; e < V; ++e) f[e] += to_f32(p[j].e[e]);
    }
    for (; i < hi; ++i) {
        const Pack<T, V> p = *reinterpret_cast<const Pack<T, V> *>(dy + (int64_t)order[i] * ld + c);
#pragma unroll
        for (int e = 0; e < V; ++e) f[e] += to_f32(p.e[e]);
    }
}

// Sums of the blocks of kRun sorted positions that lie inside one run.
template <class T, int V>
__global__ __launch_bounds__(256) void blocks_kernel(int K, int vocab, const int *__restrict__ order,
                                                     const int *__restrict__ sorted, const T *__restrict__ dy,
                                                     int64_t ld, float *part) {
    const int b = (int)blockIdx.x;
    const int row = sorted[b * kRun];
    if (row == vocab || sorted[b * kRun + kRun - 1] != row) return;
    const int c = ((int)blockIdx.y * 256 + (int)threadIdx.x) * V;
    if (c >= K) return;
    float f[V];
#pragma unroll
    for (int e = 0; e < V; ++e) f[e] = 0.0f;
    add_rows<T, V>(f, order, dy, ld, c, b * kRun, b * kRun + kRun);
    store_vec<float, V>(part + (size_t)b * (size_t)K + c, f);
}

// One table row per blockIdx.x, 256 V columns per blockIdx.y.
template <class T, class G, int V>
__global__ __launch_bounds__(256) void table_kernel(int K, const int *__restrict__ order, const int *__restrict__ first,
                                                    const T *__restrict__ dy, int64_t ld,
                                                    const float *__restrict__ part, float scale, int accumulate,
                                                    G *dtable, int64_t ldt) {
    const int c = ((int)blockIdx.y * 256 + (int)threadIdx.x) * V;
    if (c >= K) return;
    const int lo = first[blockIdx.x], hi = first[blockIdx.x + 1];
    G *out = dtable + (int64_t)blockIdx.x * ldt + c;
    if (accumulate && lo == hi) return;
    float f[V];
#pragma unroll
    for (int e = 0; e < V; ++e) f[e] = 0.0f;
    const int b0 = (lo + kRun - 1) / kRun, b1 = hi / kRun;   // whole blocks [b0, b1)
    if (b0 < b1) {
        add_rows<T, V>(f, order, dy, ld, c, lo, b0 * kRun);
        for (int b = b0; b < b1; ++b) {
            const Pack<float, V> q = *reinterpret_cast<const Pack<float, V> *>(part + (size_t)b * (size_t)K + c);
#pragma unroll
            for (int e = 0; e < V; ++e) f[e] += q.e[e];
        }
        add_rows<T, V>(f, order, dy, ld, c, b1 * kRun, hi);
    } else {
        add_rows<T, V>(f, order, dy, ld, c, lo, hi);
    }
#pragma unroll
    for (int e = 0; e < V; ++e) f[e] *= scale;
    if (accumulate) {
        const Pack<G, V> q = *reinterpret_cast<const Pack<G, V> *>(out);
#pragma unroll
        for (int e = 0; e < V; ++e) f[e] += to_f32(q.e[e]);
    }
    store_vec<G, V>(out, f);
}

constexpr int kMaxTokens = 1 << 20, kMaxVocab = 1 << 24, kMaxCols = 1 << 20;

int hip_error(hipError_t e, const char *what) {
    return set_error(COMPASS_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

int check(int T, int V, int K, int type) {
    if (T < 1 || V < 1 || K < 1) return set_error(COMPASS_ERR_INVALID, "need positive T, V and K");
    if (type != COMPASS_BF16 && type != COMPASS_F32) return set_error(COMPASS_ERR_INVALID, "unknown element type %d", type);
    if (T > kMaxTokens || V > kMaxVocab || K > kMaxCols)
        return set_error(COMPASS_ERR_UNSUPPORTED, "T = %d, V = %d, K = %d beyond %d, %d, %d", T, V, K, kMaxTokens,
                         kMaxVocab, kMaxCols);
    return COMPASS_OK;
}

size_t size_of(int type) { return type == COMPASS_F32 ? 4 : 2; }
bool off_element(const void *p, int type) { return ((uintptr_t)p & (size_of(type) - 1)) != 0; }
// whether every row starts on 16 bytes and holds whole vectors of V elements
bool rows_aligned(const void *p, int64_t ld, int type) {
    return ((uintptr_t)p & 15) == 0 && (size_t)ld * size_of(type) % 16 == 0;
}
unsigned col_blocks(int K, int V) { return (unsigned)((K + 256 * V - 1) / (256 * V)); }

// order, sorted [T], first [V + 1], then the sums of whole blocks
struct Scratch {
    size_t sorted, first, part, bytes;
};
Scratch scratch_of(int T, int V, int K) {
    Scratch s;
    s.sorted = align256((size_t)T * 4);
    s.first = s.sorted + align256((size_t)T * 4);
    s.part = s.first + align256(((size_t)V + 1) * 4);
    s.bytes = s.part + (size_t)(T / kRun) * (size_t)K * 4;
    return s;
}

template <class T, int V>
void lookup(int tokens, int K, int vocab, const int64_t *ids, int64_t v0, const void *table, int64_t ldt, float scale,
            void *y, int64_t ldy, hipStream_t s) {
    lookup_kernel<T, V><<<dim3((unsigned)tokens, col_blocks(K, V)), 256, 0, s>>>(K, v0, vocab, ids, (const T *)table, ldt,
                                                                              scale, (T *)y, ldy);
}

struct Gradient {
    int T, K, V;
    const int *order, *sorted, *first;
    float *part;
    const void *dy;
    int64_t ld;
    float scale;
    int accumulate;
    void *dtable;
    int64_t ldt;
};

template <class D, class G, int V>
void gradient(const Gradient &g, hipStream_t s) {
    if (g.T >= kRun)
        blocks_kernel<D, V><<<dim3((unsigned)(g.T / kRun), col_blocks(g.K, V)), 256, 0, s>>>(
            g.K, g.V, g.order, g.sorted, (const D *)g.dy, g.ld, g.part);
    table_kernel<D, G, V><<<dim3((unsigned)g.V, col_blocks(g.K, V)), 256, 0, s>>>(
        g.K, g.order, g.first, (const D *)g.dy, g.ld, g.part, g.scale, g.accumulate, (G *)g.dtable, g.ldt);
}

}  // namespace

int op_embed_forward(int T, int V, int K, int type, const int64_t *ids, int64_t v0, const void *table, int64_t ldt,
                     float scale, void *y, int64_t ldy, void *stream) {
    int rc = check(T, V, K, type);
    if (rc != COMPASS_OK) return rc;
    if (!ids || !table || !y) return set_error(COMPASS_ERR_INVALID, "ids, table and y are required");
    if (v0 < 0) return set_error(COMPASS_ERR_INVALID, "v0 must not be negative");
    if (ldt < K || ldy < K) return set_error(COMPASS_ERR_INVALID, "rows of %d elements overlap", K);
    if (off_element(table, type) || off_element(y, type))
        return set_error(COMPASS_ERR_INVALID, "an operand is not aligned to its elements");
    int cus;
    if ((rc = current_num_cu(&cus)) != COMPASS_OK) return rc;
    const hipStream_t s = (hipStream_t)stream;
    const bool wide = K % (int)(16 / size_of(type)) == 0 && rows_aligned(table, ldt, type) && rows_aligned(y, ldy, type);
    if (type == COMPASS_F32) {
        if (wide) lookup<float, 4>(T, K, V, ids, v0, table, ldt, scale, y, ldy, s);
        else lookup<float, 1>(T, K, V, ids, v0, table, ldt, scale, y, ldy, s);
    } else {
        if (wide) lookup<Bf16, 8>(T, K, V, ids, v0, table, ldt, scale, y, ldy, s);
        else lookup<Bf16, 1>(T, K, V, ids, v0, table, ldt, scale, y, ldy, s);
    }
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? COMPASS_OK : hip_error(e, "lookup launch");
}

int op_embed_workspace(int T, int V, int K, size_t *bytes) {
    const int rc = check(T, V, K, COMPASS_BF16);
    if (rc != COMPASS_OK) return rc;
    if (!bytes) return set_error(COMPASS_ERR_INVALID, "bytes is required");
    *bytes = scratch_of(T, V, K).bytes;
    return COMPASS_OK;
}

int op_embed_backward(int T, int V, int K, int dtype, int gtype, const int64_t *ids, int64_t v0, const void *dy,
                      int64_t ldy, float scale, void *dtable, int64_t ldt, int accumulate, void *ws, size_t ws_bytes,
                      void *stream) {
    int rc = check(T, V, K, dtype);
    if (rc != COMPASS_OK || (rc = check(T, V, K, gtype)) != COMPASS_OK) return rc;
    if (!ids || !dy || !dtable || !ws)
        return set_error(COMPASS_ERR_INVALID, "ids, dy, dtable and the workspace are required");
    if (v0 < 0) return set_error(COMPASS_ERR_INVALID, "v0 must not be negative");
    if (ldy < K || ldt < K) return set_error(COMPASS_ERR_INVALID, "rows of %d elements overlap", K);
    if (off_element(dy, dtype) || off_element(dtable, gtype))
        return set_error(COMPASS_ERR_INVALID, "an operand is not aligned to its elements");
    const Scratch sc = scratch_of(T, V, K);
    if (((uintptr_t)ws & 15) || ws_bytes < sc.bytes)
        return set_error(COMPASS_ERR_INVALID, "workspace of %zu bytes (16-byte aligned), need %zu", ws_bytes, sc.bytes);
    int cus;
    if ((rc = current_num_cu(&cus)) != COMPASS_OK) return rc;
    const hipStream_t s = (hipStream_t)stream;
    char *w = (char *)ws;
    int *order = (int *)w, *sorted = (int *)(w + sc.sorted), *first = (int *)(w + sc.first);
    rank_kernel<<<dim3((unsigned)((T + 63) / 64)), 1024, 0, s>>>(T, v0, V, ids, order, sorted);
    runs_kernel<<<dim3((unsigned)(V / 256 + 1)), 256, 0, s>>>(T, V, sorted, first);
    const Gradient g{T, K, V, order, sorted, first, (float *)(w + sc.part), dy, ldy, scale, accumulate, dtable, ldt};
    const bool d32 = dtype == COMPASS_F32, g32 = gtype == COMPASS_F32;
    // one vector width for both sides: that of the wider-vectored (bf16) one
    const int v = d32 && g32 ? 4 : 8;
    const bool wide = K % v == 0 && rows_aligned(dy, ldy, dtype) && rows_aligned(dtable, ldt, gtype);
    if (d32 && g32) wide ? gradient<float, float, 4>(g, s) : gradient<float, float, 1>(g, s);
    else if (d32) wide ? gradient<float, Bf16, 8>(g, s) : gradient<float, Bf16, 1>(g, s);
    else if (g32) wide ? gradient<Bf16, float, 8>(g, s) : gradient<Bf16, float, 1>(g, s);
    else wide ? gradient<Bf16, Bf16, 8>(g, s) : gradient<Bf16, Bf16, 1>(g, s);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? COMPASS_OK : hip_error(e, "table gradient launch");
}

}  // namespace compass
