// extern "C" entry points declared in compass.h.
#include "compass.h"
#include "internal.h"

using namespace compass;

extern "C" {

int compass_schedule(int pattern, int ring, int n, int rank, int32_t *out, int cap) {
    return schedule_fill(pattern, ring, n, rank, out, cap);
}

int compass_ag_gemm(const compass_problem *p, const compass_links *links, void *stream) {
    return op_ag_gemm(p, links, stream);
}

int compass_gemm_rs(const compass_problem *p, const compass_links *links, void *stream) {
    return op_gemm_rs(p, links, stream);
}

int compass_decomp_gemm(const compass_problem *p, int d, const compass_links *links, void *stream) {
    return op_decomp(p, d, links, stream);
}

int compass_gemm(int M, int N, int K, const void *A, const void *W, void *C, const float *P, void *stream) {
    return op_gemm(M, N, K, A, W, C, P, stream);
}

int compass_gemm_noalloc(int M, int N, int K, const void *A, const void *W, void *C, const float *P, void *stream) {
    return op_gemm_noalloc(M, N, K, A, W, C, P, stream);
}

int compass_transfer(const compass_problem *p, const compass_links *links, void *stream) {
    return op_transfer(p, links, stream);
}

int compass_sequential(const compass_problem *p, const compass_links *links, void *stream) {
    return op_sequential(p, links, stream);
}

int compass_xent_workspace(int M, int V, int K, int backward, int piece, size_t *bytes) {
    return op_xent_workspace(M, V, K, backward, piece, bytes);
}

int compass_xent_forward(int M, int V, int K, const void *H, const void *W, const int64_t *target, int64_t v0, float
                         *lse, float *tlogit, float *loss, void *workspace, size_t workspace_bytes, void *stream) {
    return op_xent_forward(M, V, K, H, W, target, v0, lse, tlogit, loss, workspace, workspace_bytes, stream);
}

int compass_xent_join(int n, int M, const float *lse_parts, const float *tlogit_parts, const int64_t *target, float
                      *lse, float *loss, void *stream) {
    return op_xent_join(n, M, lse_parts, tlogit_parts, target, lse, loss, stream);
}

int compass_xent_backward(int M, int V, int K, const void *H, const void *W, const int64_t *target, int64_t v0, const
                          float *lse, const float *grad, void *dH, void *dW, int piece, void *workspace, size_t
                          workspace_bytes, void *stream) {
    return op_xent_backward(M, V, K, H, W, target, v0, lse, grad, dH, dW, piece, workspace, workspace_bytes,
                            stream);
}

int compass_norm_forward(int M, int N, int dtype, int ptype, const void *x, int64_t ldx, const void *gamma, const void
                         *beta, float eps, void *y, int64_t ldy, float *mean, float *rstd, void *stream) {
    return op_norm_forward(M, N, dtype, ptype, x, ldx, gamma, beta, eps, y, ldy, mean, rstd, stream);
}

int compass_norm_workspace(int M, int N, size_t *bytes) {
    return op_norm_workspace(M, N, bytes);
}

int compass_norm_backward(int M, int N, int dtype, int ptype, const void *dy, int64_t lddy, const void *x, int64_t
                          ldx, const void *gamma, const float *mean, const float *rstd, void *dx, int64_t lddx, float
                          *dgamma, float *dbeta, void *workspace, size_t workspace_bytes, void *stream) {
    return op_norm_backward(M, N, dtype, ptype, dy, lddy, x, ldx, gamma, mean, rstd, dx, lddx, dgamma, dbeta,
                            workspace, workspace_bytes, stream);
}

int compass_embed_forward(int T, int V, int K, int dtype, const int64_t *ids, int64_t v0, const void *table, int64_t
                          ldt, float scale, void *y, int64_t ldy, void *stream) {
    return op_embed_forward(T, V, K, dtype, ids, v0, table, ldt, scale, y, ldy, stream);
}

int compass_embed_workspace(int T, int V, int K, size_t *bytes) {
    return op_embed_workspace(T, V, K, bytes);
}

int compass_embed_backward(int T, int V, int K, int dtype, int gtype, const int64_t *ids, int64_t v0, const void *dy,
                           int64_t ldy, float scale, void *dtable, int64_t ldt, int accumulate, void *workspace,
                           size_t workspace_bytes, void *stream) {
    return op_embed_backward(T, V, K, dtype, gtype, ids, v0, dy, ldy, scale, dtable, ldt, accumulate, workspace,
                             workspace_bytes, stream);
}

int compass_rms_forward(int M, int N, int dtype, int ptype, const void *x, int64_t ldx, const void *residual, int64_t
                        ldr, const void *gamma, float eps, void *h, int64_t ldh, void *y, int64_t ldy, void *y8, void
                        *scale, float *rstd, void *stream) {
    return op_rms_forward(M, N, dtype, ptype, x, ldx, residual, ldr, gamma, eps, h, ldh, y, ldy, y8, scale, rstd,
                          stream);
}

int compass_rms_workspace(int M, int N, size_t *bytes) {
    return op_rms_workspace(M, N, bytes);
}

int compass_rms_backward(int M, int N, int dtype, int ptype, const void *dy, int64_t lddy, const void *h, int64_t ldh,
                         const void *dh, int64_t lddh, const void *gamma, const float *rstd, void *dx, int64_t lddx,
                         float *dgamma, void *workspace, size_t workspace_bytes, void *stream) {
    return op_rms_backward(M, N, dtype, ptype, dy, lddy, h, ldh, dh, lddh, gamma, rstd, dx, lddx, dgamma, workspace,
                           workspace_bytes, stream);
}

int compass_fp8_scale_cols(int K, int *cols) {
    return op_fp8_scale_cols(K, cols);
}

int compass_fp8_quant(int M, int K, int dtype, const void *x, int64_t ldx, int across, void *x8, void *scale, void
                      *stream) {
    return op_fp8_quant(M, K, dtype, x, ldx, across, x8, scale, stream);
}

int compass_fp8_dequant(int M, int K, int dtype, const void *x8, const void *scale, void *x, int64_t ldx, void
                        *stream) {
    return op_fp8_dequant(M, K, dtype, x8, scale, x, ldx, stream);
}

int compass_fp8_gemm_workspace(int M, int N, int K, size_t *bytes) {
    return op_fp8_gemm_workspace(M, N, K, bytes);
}

int compass_fp8_gemm(int M, int N, int K, const void *A, const void *A_scale, const void *W, const void *W_scale, void
                     *C, void *workspace, size_t workspace_bytes, void *stream) {
    return op_fp8_gemm(M, N, K, A, A_scale, W, W_scale, C, workspace, workspace_bytes, stream);
}

int compass_fp8_wgrad_workspace(int M, int N, int K, size_t *bytes) {
    return op_fp8_wgrad_workspace(M, N, K, bytes);
}

int compass_fp8_wgrad(int M, int N, int K, int gtype, const void *dY, const void *X8, const void *X_scale, void *dW, int
                      accumulate, void *workspace, size_t workspace_bytes, void *stream) {
    return op_fp8_wgrad(M, N, K, gtype, dY, X8, X_scale, dW, accumulate, workspace, workspace_bytes, stream);
}

int compass_sync(void) { return op_sync(); }

int compass_set_option(int key, long long value) { return op_set_option(key, value); }

int compass_kernel_times(double *us, int cap) { return op_kernel_times(us, cap); }

int compass_tile_trace(uint32_t *records, int cap) { return op_tile_trace(records, cap); }

int compass_probe_mfma(int iters, double *tflops, double *sclk_ghz) {
    return op_probe_mfma(iters, tflops, sclk_ghz);
}

int compass_pick_strategy(const compass_workload *w, const compass_topology *t, const compass_calib *cal,
                          compass_choice *out) {
    return pick(w, t, cal, out);
}

int compass_partition_layout(int pattern, int ring, int n, int rank, int M, const compass_links *l, int32_t *order,
                             int32_t *row0, int32_t *rows, int cap) {
    return op_partition_layout(pattern, ring, n, rank, M, l, order, row0, rows, cap);
}

int compass_ring_arrival_times(int n, int rank, double piece_bytes, const double *hop_Bps, int d, double *out,
                               int cap) {
    return ring_arrivals(n, rank, piece_bytes, hop_Bps, d, out, cap);
}

double compass_model_t_comm(const compass_workload *w, const compass_topology *t) {
    if (!w || !t || w->n < 1) return -1.0;
    const int r = t->ring;
    if (r != COMPASS_RING_SINGLE && r != COMPASS_RING_DOUBLE && r != COMPASS_RING_DOUBLE_SPLIT &&
        r != COMPASS_RING_ALLTOALL)
        return -1.0;
    if (r == COMPASS_RING_ALLTOALL && (w->pattern != COMPASS_AG_GEMM || w->n % 2)) return -1.0;
    if (!(t->fwd_Bps > 0) || (r != COMPASS_RING_SINGLE && !(t->bwd_Bps > 0))) return -1.0;
    return model_t_comm(*w, *t);
}

double compass_model_t_decomp(double t_comp, double t_comm, int d, double alpha, double beta) {
    return model_t_decomp(t_comp, t_comm, d, alpha, beta);
}

double compass_model_t_fusion(const compass_workload *w, double t_comp, double t_comm_step, double alpha_f,
                              double beta_f) {
    if (!w || w->n < 1) return -1.0;
    return model_t_fusion(*w, t_comp, t_comm_step, alpha_f, beta_f);
}

int compass_calibrate(const compass_sample *s, int count, compass_calib *inout) { return calibrate(s, count, inout); }

const char *compass_last_error(void) { return last_error(); }

const char *compass_version(void) { return "compass-mi355x 0.1 (gfx950)"; }

}  // extern "C"
