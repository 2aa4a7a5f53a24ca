// Internal declarations shared by the host-side translation units.
#pragma once
#include <stdint.h>

#include "compass.h"

namespace compass {

constexpr int kMaxRanks = 32;

int set_error(int code, const char *fmt, ...);
const char *last_error();

int schedule_fill(int pattern, int ring, int n, int rank, int32_t *out, int cap);
int pick(const compass_workload *w, const compass_topology *t, const compass_calib *cal, compass_choice *out);
int calibrate(const compass_sample *s, int count, compass_calib *inout);
double model_t_comm(const compass_workload &w, const compass_topology &t);
int ring_arrivals(int n, int rank, double piece_bytes, const double *hop_Bps, int d, double *out, int cap);
double model_t_decomp(double tc, double tm, int d, double alpha, double beta);
double model_t_fusion(const compass_workload &w, double tc, double tm_step, double af, double bf);

// runtime (GPU side)
int op_ag_gemm(const compass_problem *p, const compass_links *l, void *stream);
int op_gemm_rs(const compass_problem *p, const compass_links *l, void *stream);
int op_decomp(const compass_problem *p, int d, const compass_links *l, void *stream);
int op_gemm(int M, int N, int K, const void *A, const void *W, void *C, const float *P, void *stream);
int current_num_cu(int *out);
int op_gemm_noalloc(int M, int N, int K, const void *A, const void *W, void *C, const float *P, void *stream);
int op_transfer(const compass_problem *p, const compass_links *l, void *stream);
int op_partition_layout(int pattern, int ring, int n, int rank, int M, const compass_links *l, int32_t *order,
                        int32_t *row0, int32_t *rows, int cap);
int op_sequential(const compass_problem *p, const compass_links *l, void *stream);
int op_sync();
int op_set_option(int key, long long value);
int op_kernel_times(double *us, int cap);
int op_tile_trace(uint32_t *out, int cap);
int op_probe_mfma(int iters, double *tflops, double *sclk_ghz);


// the model's ends (operands as in compass.h); current_num_cu also refuses a
// device other than gfx950
int op_xent_workspace(int M, int V, int K, int backward, int piece, size_t *bytes);
int op_xent_forward(int M, int V, int K, const void *H, const void *W, const int64_t *target, int64_t v0, float *lse,
                    float *tlogit, float *loss, void *workspace, size_t workspace_bytes, void *stream);
int op_xent_join(int n, int M, const float *lse_parts, const float *tlogit_parts, const int64_t *target, float *lse,
                 float *loss, void *stream);
int op_xent_backward(int M, int V, int K, const void *H, const void *W, const int64_t *target, int64_t v0, const float
                     *lse, const float *grad, void *dH, void *dW, int piece, void *workspace, size_t workspace_bytes,
                     void *stream);
int op_norm_forward(int M, int N, int dtype, int ptype, const void *x, int64_t ldx, const void *gamma, const void
                    *beta, float eps, void *y, int64_t ldy, float *mean, float *rstd, void *stream);
int op_norm_workspace(int M, int N, size_t *bytes);
int op_norm_backward(int M, int N, int dtype, int ptype, const void *dy, int64_t lddy, const void *x, int64_t ldx,
                     const void *gamma, const float *mean, const float *rstd, void *dx, int64_t lddx, float *dgamma,
                     float *dbeta, void *workspace, size_t workspace_bytes, void *stream);
int op_embed_forward(int T, int V, int K, int dtype, const int64_t *ids, int64_t v0, const void *table, int64_t ldt,
                     float scale, void *y, int64_t ldy, void *stream);
int op_embed_workspace(int T, int V, int K, size_t *bytes);
int op_embed_backward(int T, int V, int K, int dtype, int gtype, const int64_t *ids, int64_t v0, const void *dy,
                      int64_t ldy, float scale, void *dtable, int64_t ldt, int accumulate, void *workspace, size_t
                      workspace_bytes, void *stream);

}  // namespace compass
