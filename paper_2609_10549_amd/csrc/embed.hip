// Embedding lookup and the table's gradient (compass_embed_*).
//
//   y[t] = scale table[ids[t] - v0], zeros where the id is not in the table
//   dtable[v] = scale sum_{t: ids[t] = v0 + v} dy[t]
//
// Gradient: the tokens are sorted by table row (stable, so that each row's sum
// runs in token order whatever the machine does), every table row finds its
// run in the sorted order, and one pass writes the table, each element once:
// the sum of the run's rows, or zero. A long run (a frequent token) would be
// one workgroup's long walk, so blocks of sorted positions that lie inside
// one run are summed beside that pass, all at once, and a second, short one
// adds those sums for the rows that have any. No atomics anywhere.
//
// Times beside the kernels are of calls repeated on one set of inputs, so what of
// it fits the caches is read from them. (32768 tokens, 50257 x 4096 bf16, gradient:
// 146 us so, 160 with two sets in turn.)
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "compass.h"
#include "internal.h"
#include "rowops.h"

namespace compass {

namespace {

// Sorted positions of a block: 2^run_shift(T). Short batches take small blocks,
// so that the runs without one (below twice a block) are short walks too; in
// long ones the blocks' own workgroups count (500 tokens, 6283 x 1031 fp32: 16
// positions 22 us, 32 27; 8000 tokens, 20000 x 5001 bf16: 86 and 94; 32768 tokens,
// 50257 x 4096: 158 and 146).
constexpr int run_shift(int T) { return T < 16384 ? 4 : 5; }

// Elements by which a loose fp32 row's vectors are moved back so that they lie
// on whole 128-byte lines of what is written: a wave's streaming stores then
// leave no line half written (a masked write costs the memory a read) but at the
// row's ends. 14785 tokens, 65225 x 3890 fp32: gradient 257 -> 211 us, lookup 61
// -> 56; bf16 rows, whose end vectors are 8 stores, lose by it (8000 tokens,
// 20000 x 5001: 92 -> 103). kLineElements: at most so many more elements to cover.
template <bool LOOSE, class T>
__device__ __forceinline__ int line_shift(const T *row) {
    return LOOSE && sizeof(T) == 4 ? (int)(((uintptr_t)row & 127) / sizeof(T)) : 0;
}
template <bool LOOSE, class T>
constexpr int kLineElements = LOOSE && sizeof(T) == 4 ? 31 : 0;

// How a kernel's workgroups of 256 threads cover rows of K elements: groups of
// 2^shift threads, a vector of V elements each; blockIdx.y counts the column
// blocks of rows that one group does not cover.
struct Cover {
    int shift;
    __device__ __forceinline__ int group(int wg) const { return (wg << (8 - shift)) + ((int)threadIdx.x >> shift); }
    template <int V>
    __device__ __forceinline__ int column() const {
        return (((int)blockIdx.y << shift) + ((int)threadIdx.x & ((1 << shift) - 1))) * V;
    }
};

// An id's distance from v0 >= 0, -1 below it (no difference of two 64-bit numbers
// that wraps round: an id far below zero would come out in the table).
__device__ __forceinline__ int64_t row_of(int64_t id, int64_t v0) { return id < v0 ? -1 : id - v0; }

// TOKENS tokens per group, their rows in flight together.
//
// Bound by memory. 32768 tokens, 50257 x 4096 bf16, token frequencies as
// 1 / rank: 86 us with ordinary stores, 60 with streaming ones.
template <class T, int V, bool LOOSE, int TOKENS>
__global__ __launch_bounds__(256) void lookup_kernel(Cover cov, int tokens, int K, int64_t v0, int vocab,
                                                     const int64_t *__restrict__ ids, const T *__restrict__ table,
                                                     int64_t ldt, float scale, T *y, int64_t ldy) {
    const int t0 = cov.group((int)blockIdx.x) * TOKENS;
    if (t0 >= tokens) return;
    Pack<T, V> p[TOKENS];
    bool inside[TOKENS];
    int c[TOKENS];
#pragma unroll
    for (int j = 0; j < TOKENS; ++j) {
        const int64_t row = t0 + j < tokens ? row_of(ids[t0 + j], v0) : -1;
        inside[j] = row >= 0 && row < vocab;
        c[j] = cov.column<V>() - line_shift<LOOSE>(y + (int64_t)(t0 + j) * ldy);
        if (inside[j]) p[j] = load_pack<T, V, LOOSE>(table + row * ldt, c[j], K);
    }
#pragma unroll
    for (int j = 0; j < TOKENS; ++j) {
        if (t0 + j >= tokens) return;
        float f[V];
        unpack(p[j], f);
#pragma unroll
        for (int e = 0; e < V; ++e) f[e] = inside[j] ? f[e] * scale : 0.0f;
        if (c[j] < K) store_pack<T, V, LOOSE>(y + (int64_t)(t0 + j) * ldy, c[j], K, f);
    }
}

// Table row of a token, `vocab` for ids outside it.
__device__ __forceinline__ int table_row(int64_t id, int64_t v0, int vocab) {
    const int64_t r = row_of(id, v0);
    return r >= 0 && r < vocab ? (int)r : vocab;
}

// Sorts each chunk of kChunk tokens, stable, by counting pairs: the place of a
// token is the number of tokens of its chunk with a smaller row, or the same
// row and a smaller index. 64 tokens per workgroup; each of the 16 waves counts
// over 64 tokens of the chunk, one scalar row against 64 lanes at a time.
constexpr int kChunk = 1024;
__global__ __launch_bounds__(1024) void chunk_kernel(int T, int64_t v0, int vocab, const int64_t *__restrict__ ids,
                                                     int *order, int *sorted) {
    __shared__ int s[16][64];
    const int lane = threadIdx.x & 63;
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int b = (int)blockIdx.x, t = b * 64 + lane, c0 = b / 16 * 16;   // in 64s
    const int key = t < T ? table_row(ids[t], v0, vocab) : vocab;
    const int at = (c0 + w) * 64 + lane;
    const int other = at < T ? table_row(ids[at], v0, vocab) : 0x7fffffff;   // past the end: before nobody
    int n = 0;
    if (c0 + w == b) {
#pragma unroll
        for (int i = 0; i < 64; ++i) {
            const int k = __builtin_amdgcn_readlane(other, i);
            n += k < key || (k == key && i < lane) ? 1 : 0;
        }
    } else {
        const int below = c0 + w < b ? key + 1 : key;   // before: k <= key, after: k < key
#pragma unroll
        for (int i = 0; i < 64; ++i) n += __builtin_amdgcn_readlane(other, i) < below ? 1 : 0;
    }
    s[w][lane] = n;
    __syncthreads();
    if (w != 0 || t >= T) return;
#pragma unroll
    for (int i = 1; i < 16; ++i) n += s[i][lane];
    order[c0 * 64 + n] = t;
    sorted[c0 * 64 + n] = key;
}

// Merges the sorted chunks: an element's place is its place in its own chunk
// and, in every other, the number of elements before it, by binary search. 64
// neighbours per workgroup (their searches take nearly the same path), the
// chunks dealt to its 16 waves. The searches grow with the square of the batch:
// 32768 tokens 7.6 us, 65536 21, 131072 66, 262144 234, 2^20 (the longest) 3.2 ms.
__global__ __launch_bounds__(1024) void merge_kernel(int T, const int *__restrict__ chunk_order,
                                                     const int *__restrict__ chunk_sorted, int *order, int *sorted) {
    __shared__ int s[16][64];
    const int lane = threadIdx.x & 63;
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int at = (int)blockIdx.x * 64 + lane, own = (int)blockIdx.x / (kChunk / 64);
    const int chunks = (T + kChunk - 1) / kChunk;
    const int key = at < T ? chunk_sorted[at] : 0;
    int n = 0;
    for (int c = w; c < chunks; c += 16) {
        if (c == own) {
            n += at - own * kChunk;
            continue;
        }
        const int *run = chunk_sorted + (size_t)c * kChunk;
        const int below = c < own ? key + 1 : key;
        int lo = 0, hi = min(kChunk, T - c * kChunk);
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (run[mid] < below) lo = mid + 1;
            else hi = mid;
        }
        n += lo;
    }
    s[w][lane] = n;
    __syncthreads();
    if (w != 0 || at >= T) return;
#pragma unroll
    for (int i = 1; i < 16; ++i) n += s[i][lane];
    order[n] = chunk_order[at];
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

// f += the vector at column c of dy of the sorted positions [lo, hi), in order,
// kAhead rows in flight; the lanes of a group (or of its wave) fetch the token
// indices together.
constexpr int kAhead = 4;
template <class T, int V, bool LOOSE>
__device__ __forceinline__ void add_rows(float (&f)[V], int shift, int c, int K, const int *__restrict__ order,
                                         const T *__restrict__ dy, int64_t ld, int lo, int hi) {
    const int width = 1 << min(shift, 6), lane = (int)threadIdx.x & (width - 1);
    for (int base = lo; base < hi; base += width) {
        const int mine = base + lane < hi ? order[base + lane] : 0;
        const int n = min(width, hi - base);
        for (int i = 0; i < n; i += kAhead) {
            Pack<T, V> p[kAhead];
#pragma unroll
            for (int j = 0; j < kAhead; ++j) {
                const int tok = __shfl(mine, i + j, width);   // (width is a multiple of kAhead)
                if (i + j < n) p[j] = load_pack<T, V, LOOSE>(dy + (int64_t)tok * ld, c, K);
            }
#pragma unroll
            for (int j = 0; j < kAhead; ++j)
                if (i + j < n) {
                    float d[V];
                    unpack(p[j], d);
#pragma unroll
                    for (int e = 0; e < V; ++e) f[e] += d[e];
                }
        }
    }
}

struct Gradient {
    Cover cov;
    int T, K, V;
    int blocks, shift;              // 2^shift sorted positions each
    const int *order, *sorted, *first;
    float *part;                    // [blocks][ldp]
    int ldp;
    const void *dy;
    int64_t ld;
    float scale;
    void *dtable;
    int64_t ldt;
};

// Column of this thread's vector, `col` on lines, in a table row.
template <class G, bool LOOSE>
__device__ __forceinline__ int row_column(const Gradient &g, int row, int col) {
    return col - line_shift<LOOSE>((const G *)g.dtable + (int64_t)row * g.ldt);
}

// A table row's sums from column c on, scaled, to the table or onto it.
template <class G, int V, bool LOOSE, bool ACC>
__device__ __forceinline__ void put_row(const Gradient &g, int row, int c, float (&f)[V]) {
    G *out = (G *)g.dtable + (int64_t)row * g.ldt;
#pragma unroll
    for (int e = 0; e < V; ++e) f[e] *= g.scale;
    if constexpr (ACC) {
        float o[V];
        unpack(load_pack<G, V, LOOSE, true>(out, c, g.K), o);
#pragma unroll
        for (int e = 0; e < V; ++e) f[e] += o[e];
    }
    store_pack<G, V, LOOSE>(out, c, g.K, f);
}

// One launch of three kinds of groups, each kind rounded up to a workgroup:
//   blocks: the sum of a block of sorted positions that lies inside one run;
//   tokens: kAhead sorted positions; writes the table rows of the runs that
//     begin there, but for one that holds such a block;
//   zeros (not with ACC): kZeroRows table rows, those without tokens.
// In that order: reads and writes dealt evenly over the launch took longer.
//
// Bound by memory. 32768 distinct tokens, 50257 x 4096 bf16 (680 MB), the whole
// gradient: 220 us with the kinds dealt evenly, 200 in this order, 168 with 4
// rows in flight per thread in place of 8 (more waves; two vectors per thread
// in place of one: 229), 129 with streaming stores of the table. Adding to a
// table that is there (ACC), the loads of dy and the table stream too: 187 ->
// 168 us (without ACC that costs: 129 -> 150).
constexpr int kZeroRows = 8;
template <class T, class G, int V, bool LOOSE, bool ACC>
__global__ __launch_bounds__(256) void rows_kernel(const Gradient g) {
    const int per = 256 >> g.cov.shift;
    const int block_wgs = (g.blocks + per - 1) / per, token_wgs = ((g.T + kAhead - 1) / kAhead + per - 1) / per;
    const int readers = block_wgs + token_wgs, at = (int)blockIdx.x, col = g.cov.column<V>();
    const T *dy = (const T *)g.dy;
    float f[V] = {};
    if (at < block_wgs) {
        const int b = g.cov.group(at);
        if (b >= g.blocks) return;
        const int from = b << g.shift, to = from + (1 << g.shift);
        const int row = g.sorted[from];
        if (row == g.V || g.sorted[to - 1] != row) return;
        add_rows<T, V, LOOSE>(f, g.cov.shift, col, g.K, g.order, dy, g.ld, from, to);
        // (read back soon: no streaming)
        store_pack<float, V, false, false>(g.part + (size_t)b * (size_t)g.ldp, col, g.ldp, f);
    } else if (at < readers) {
        const int i0 = g.cov.group(at - block_wgs) * kAhead;
        if (i0 >= g.T) return;
        const int n = min(kAhead, g.T - i0), mine = i0 + min((int)threadIdx.x & (kAhead - 1), n - 1);
        const int my_row = g.sorted[mine], my_tok = g.order[mine];
        const int before = i0 > 0 ? g.sorted[i0 - 1] : -1;
        int row[kAhead];
        Pack<T, V> p[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            row[j] = __shfl(my_row, j, kAhead);
            const int tok = __shfl(my_tok, j, kAhead);
            // not a run of the groups before, nor an id outside the table
            if (j < n && row[j] != before && row[j] != g.V)
                p[j] = load_pack<T, V, LOOSE, ACC>(dy + (int64_t)tok * g.ld, row_column<G, LOOSE>(g, row[j], col), g.K);
        }
        int lo = i0;   // of the run at j
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            if (j >= n || row[j] == before || row[j] == g.V) continue;
            float d[V];
            unpack(p[j], d);
            const bool begins = j == 0 || row[j] != row[j - 1];
            if (begins) lo = i0 + j;
#pragma unroll
            for (int e = 0; e < V; ++e) f[e] = begins ? d[e] : f[e] + d[e];
            const int c = row_column<G, LOOSE>(g, row[j], col);
            if (j + 1 < n) {
                if (row[j + 1] == row[j]) continue;
            } else {   // the run may go on
                const int hi = g.first[row[j] + 1];
                if (((lo + (1 << g.shift) - 1) >> g.shift) < (hi >> g.shift)) continue;
                add_rows<T, V, LOOSE>(f, g.cov.shift, c, g.K, g.order, dy, g.ld, i0 + n, hi);
            }
            put_row<G, V, LOOSE, ACC>(g, row[j], c, f);
        }
    } else {
        const int row0 = g.cov.group(at - readers) * kZeroRows;
        int start[kZeroRows + 1];
#pragma unroll
        for (int i = 0; i <= kZeroRows; ++i) start[i] = g.first[min(row0 + i, g.V)];
#pragma unroll
        for (int i = 0; i < kZeroRows; ++i)
            if (row0 + i < g.V && start[i] == start[i + 1])
                store_pack<G, V, LOOSE>((G *)g.dtable + (int64_t)(row0 + i) * g.ldt,
                                        row_column<G, LOOSE>(g, row0 + i, col), g.K, f);
    }
}

// The rows whose runs hold whole blocks, found by the first such block: one
// workgroup of 16 waves per block and 64 V columns. The row's terms (the tokens
// before its first whole block, the blocks' sums, the tokens behind the last)
// are dealt to the waves, whose sums are joined in wave order, so that the most
// frequent token of a long batch is no long walk either (a token in 9 % of
// 32768 positions: 39 us by one group, 18 here; in all of them 450 and 185 for
// the whole gradient).
template <class T, class G, int V, bool LOOSE, bool ACC>
__global__ __launch_bounds__(1024) void long_rows_kernel(const Gradient g) {
    __shared__ float s[16][64 * V];
    const int b = (int)blockIdx.x;
    const int row = g.sorted[b << g.shift];
    if (row == g.V || g.sorted[((b + 1) << g.shift) - 1] != row || (b > 0 && g.sorted[(b - 1) << g.shift] == row)) return;
    const int lane = (int)threadIdx.x & 63, w = (int)threadIdx.x >> 6;
    const int c = row_column<G, LOOSE>(g, row, ((int)blockIdx.y * 64 + lane) * V);
    const int lo = g.first[row], hi = g.first[row + 1], b1 = hi >> g.shift;
    float f[V] = {};
    auto add = [&](const float (&d)[V]) {
#pragma unroll
        for (int e = 0; e < V; ++e) f[e] += d[e];
    };
    auto token = [&](int i) {
        float d[V];
        unpack(load_pack<T, V, LOOSE>((const T *)g.dy + (int64_t)g.order[i] * g.ld, c, g.K), d);
        add(d);
    };
#pragma unroll 2
    for (int i = lo + w; i < b << g.shift; i += 16) token(i);
#pragma unroll 4
    for (int i = b + w; i < b1; i += 16) {
        float d[V];
        unpack(load_pack<float, V, LOOSE>(g.part + (size_t)i * (size_t)g.ldp, c, LOOSE ? g.K : g.ldp), d);
        add(d);
    }
#pragma unroll 2
    for (int i = (b1 << g.shift) + w; i < hi; i += 16) token(i);
#pragma unroll
    for (int e = 0; e < V; ++e) s[w][e * 64 + lane] = f[e];
    __syncthreads();
    if (w != 0) return;
#pragma unroll 5   // (of V registers each: all 15 at once spill)
    for (int i = 1; i < 16; ++i)
#pragma unroll
        for (int e = 0; e < V; ++e) f[e] += s[i][e * 64 + lane];
    put_row<G, V, LOOSE, ACC>(g, row, c, f);
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

// The smallest group (8 to 256 threads) that holds a row, else 256. (Smaller
// groups that leave fewer threads past a row's end measured slower: 50257 x 1031
// bf16, 4000 tokens: 61 us, in 9 blocks of 16 threads 92.)
Cover cover(int K, int V) {
    const int vectors = (K + V - 1) / V;
    Cover c{3};
    while (c.shift < 8 && (1 << c.shift) < vectors) ++c.shift;
    return c;
}
dim3 grid(const Cover &c, int64_t wgs, int K, int V) {
    const int cols = V << c.shift;
    return dim3((unsigned)wgs, (unsigned)((K + cols - 1) / cols));
}
int64_t wgs_of(const Cover &c, int64_t groups) {
    const int per = 256 >> c.shift;
    return (groups + per - 1) / per;
}

// order, sorted [T], first [V + 1], the chunks' order and sorted [T] where
// there are several, then the sums of whole blocks
struct Scratch {
    size_t sorted, first, chunk_order, chunk_sorted, part, bytes;
    int ldp;
};
Scratch scratch_of(int T, int V, int K) {
    Scratch s;
    const size_t list = align256((size_t)T * 4);
    s.sorted = list;
    s.first = 2 * list;
    s.chunk_order = s.first + align256(((size_t)V + 1) * 4);
    s.chunk_sorted = s.chunk_order + (T > kChunk ? list : 0);
    s.part = s.chunk_sorted + (T > kChunk ? list : 0);
    s.ldp = (K + 7) / 8 * 8;
    s.bytes = s.part + (size_t)(T >> run_shift(T)) * (size_t)s.ldp * 4;
    return s;
}

template <class T, int V, bool LOOSE>
void lookup(int tokens, int K, int vocab, const int64_t *ids, int64_t v0, const void *table, int64_t ldt, float scale,
            void *y, int64_t ldy, hipStream_t s) {
    const int cols = K + kLineElements<LOOSE, T>;
    const Cover c = cover(cols, V);
    const auto go = [&](auto kernel, int per) {
        kernel<<<grid(c, wgs_of(c, (tokens + per - 1) / per), cols, V), 256, 0, s>>>(
            c, tokens, K, v0, vocab, ids, (const T *)table, ldt, scale, (T *)y, ldy);
    };
    if (tokens < 4096) go(lookup_kernel<T, V, LOOSE, 1>, 1);
    else go(lookup_kernel<T, V, LOOSE, 4>, 4);
}

template <class D, class G, int V, bool LOOSE, bool ACC>
void launch_gradient(Gradient g, hipStream_t s) {
    const int cols = g.K + kLineElements<LOOSE, G>;
    g.cov = cover(cols, V);
    const int64_t zeros = ACC ? 0 : ((int64_t)g.V + kZeroRows - 1) / kZeroRows;
    const int64_t wgs = wgs_of(g.cov, g.blocks) + wgs_of(g.cov, (g.T + kAhead - 1) / kAhead) + wgs_of(g.cov, zeros);
    rows_kernel<D, G, V, LOOSE, ACC><<<grid(g.cov, wgs, cols, V), 256, 0, s>>>(g);
    const dim3 by_block((unsigned)g.blocks, (unsigned)((cols + 64 * V - 1) / (64 * V)));
    if (g.blocks > 0) long_rows_kernel<D, G, V, LOOSE, ACC><<<by_block, 1024, 0, s>>>(g);
}
template <class D, class G, int V>
void gradient(const Gradient &g, bool loose, bool accumulate, hipStream_t s) {
    if (loose) accumulate ? launch_gradient<D, G, V, true, true>(g, s) : launch_gradient<D, G, V, true, false>(g, s);
    else accumulate ? launch_gradient<D, G, V, false, true>(g, s) : launch_gradient<D, G, V, false, false>(g, s);
}

}  // namespace

int op_embed_forward(int T, int V, int K, int type, const int64_t *ids, int64_t v0, const void *table, int64_t ldt,
                     float scale, void *y, int64_t ldy, void *stream) {
    int rc = check(T, V, K, type);
    if (rc != COMPASS_OK) return rc;
    if (!ids || !table || !y) return set_error(COMPASS_ERR_INVALID, "ids, table and y are required");
    if (v0 < 0 || v0 > INT64_MAX - V)
        return set_error(COMPASS_ERR_INVALID, "v0 must not be negative, v0 + V must fit 64 bits");
    if (ldt < K || ldy < K) return set_error(COMPASS_ERR_INVALID, "rows of %d elements overlap", K);
    if (off_element(table, type) || off_element(y, type))
        return set_error(COMPASS_ERR_INVALID, "an operand is not aligned to its elements");
    int cus;
    if ((rc = current_num_cu(&cus)) != COMPASS_OK) return rc;
    const hipStream_t s = (hipStream_t)stream;
    const bool even = K % (int)(16 / size_of(type)) == 0 && rows_aligned(table, ldt, type) && rows_aligned(y, ldy, type);
    if (type == COMPASS_F32) {
        if (even) lookup<float, 4, false>(T, K, V, ids, v0, table, ldt, scale, y, ldy, s);
        else lookup<float, 4, true>(T, K, V, ids, v0, table, ldt, scale, y, ldy, s);
    } else {
        if (even) lookup<Bf16, 8, false>(T, K, V, ids, v0, table, ldt, scale, y, ldy, s);
        else lookup<Bf16, 8, true>(T, K, V, ids, v0, table, ldt, scale, y, ldy, s);
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
    if (v0 < 0 || v0 > INT64_MAX - V)
        return set_error(COMPASS_ERR_INVALID, "v0 must not be negative, v0 + V must fit 64 bits");
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
    const dim3 by64((unsigned)((T + 63) / 64));
    if (T <= kChunk) {
        chunk_kernel<<<by64, 1024, 0, s>>>(T, v0, V, ids, order, sorted);
    } else {
        int *chunk_order = (int *)(w + sc.chunk_order), *chunk_sorted = (int *)(w + sc.chunk_sorted);
        chunk_kernel<<<by64, 1024, 0, s>>>(T, v0, V, ids, chunk_order, chunk_sorted);
        merge_kernel<<<by64, 1024, 0, s>>>(T, chunk_order, chunk_sorted, order, sorted);
    }
    runs_kernel<<<dim3((unsigned)(V / 256 + 1)), 256, 0, s>>>(T, V, sorted, first);
    const Gradient g{{}, T, K, V, T >> run_shift(T), run_shift(T), order, sorted, first, (float *)(w + sc.part),
                     sc.ldp, dy, ldy, scale, dtable, ldt};
    const bool d32 = dtype == COMPASS_F32, g32 = gtype == COMPASS_F32;
    // one vector width for both sides: 16 bytes of the smaller type
    const bool loose = K % (d32 && g32 ? 4 : 8) != 0 || !rows_aligned(dy, ldy, dtype) || !rows_aligned(dtable, ldt, gtype);
    const bool acc = accumulate != 0;
    if (d32 && g32) gradient<float, float, 4>(g, loose, acc, s);
    else if (d32) gradient<float, Bf16, 8>(g, loose, acc, s);
    else if (g32) gradient<Bf16, float, 8>(g, loose, acc, s);
    else gradient<Bf16, Bf16, 8>(g, loose, acc, s);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? COMPASS_OK : hip_error(e, "table gradient launch");
}

}  // namespace compass
