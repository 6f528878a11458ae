/*
 * prsgd_ops.h -- operators on replica sets exported by libprsgd beside the method's own calls (prsgd.h): the
 * orthogonalised update of every worker's weight matrix, and the root-mean-square norm of every worker's rows.
 *
 * Conventions are those of prsgd.h: a status is returned (PRSGD_OK == 0, negative on error; prsgd_last_error(NULL) has
 * the text), nothing throws or aborts, buffers are device addresses owned by the caller, nothing is allocated, and work is
 * enqueued on hip_stream alone (NULL = the default stream) without waiting for it.  No state is kept between calls, so
 * calls on different streams may run at once (with workspaces of their own), and calls may be recorded into a HIP graph.
 * Elements of a row are adjacent; distances between rows and between matrices are given in elements and may be larger
 * than the row or matrix.  Buffers need the alignment of their elements only, workspaces 256 bytes.
 * Results are the same from run to run.  Arguments are checked before anything is enqueued: PRSGD_EINVAL for a null
 * pointer, a size, distance or coefficient out of range, or a misaligned buffer; PRSGD_EHIP if a launch fails.
 */
#ifndef PRSGD_OPS_H
#define PRSGD_OPS_H

#include <stddef.h>
#include <stdint.h>

#include "prsgd.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Newton-Schulz orthogonalisation of `count` matrices G [rows][cols], one per worker:
 *   X_0 = G / (||G||_F + eps),
 *   A = X X^T,  X <- a X + (b A + c A A) X,   `steps` times,
 * so that every singular value sigma of X_0 becomes p(p(..p(sigma))), p(s) = a s + b s^3 + c s^5, and the singular
 * vectors stay.  (The products run on the shorter side: X^T X from the right where rows > cols, the same polynomial.)
 * The coefficients (3.4445, -4.7750, 2.0315) with 5 steps bring singular values from 0.0021 on to between 0.68 and 1.21 (the local extremes of p).
 * A zero matrix gives zeros; a NaN or an infinity makes its own matrix NaN and no other.
 *
 * dtype  PRSGD_F32: products of operands held to 22 bits, results to fp32 accuracy, also where ||G|| is small beside eps.
 *        PRSGD_BF16: products of operands held to 11 bits (fp16, scaled by a power of two), which leaves less error than
 *        the final rounding to bfloat16 does.  Either way products are accumulated in fp32, X itself is carried to 22
 *        bits between steps, and the norm is summed in 64.  A side of up to 64 is taken through its Gram matrix in 64 bits
 *        while steps are few (10 at these coefficients), by products beyond.
 * Coefficients have to keep singular values in [0, 1] below 2 and the middle factor |b s^2 + c s^4| below 7 at every
 * step (PRSGD_EINVAL otherwise): the range of the operands.
 */
typedef struct {
  int32_t dtype;                   /* PRSGD_F32 | PRSGD_BF16: type of G and of the result            */
  int32_t count;                   /* matrices, 0..65535 (0: nothing is done)                        */
  int32_t rows, cols;              /* 1..32768 each                                                  */
  int32_t steps;                   /* 1..64                                                          */
  float   a, b, c;                 /* coefficients                                                   */
  float   eps;                     /* added to the norm, >= 0                                        */
} prsgd_orth_config;

/* Bytes of workspace that either call below needs (0 if the configuration is invalid or count is 0). */
size_t prsgd_orthogonalize_workspace_bytes(const prsgd_orth_config* cfg);

/*
 * out <- the orthogonalised G.  Matrix k starts at g_dev + k * g_matrix elements, its row i at + i * g_row.
 * out_dev may be g_dev if both distances agree; otherwise the two may not overlap.
 */
int prsgd_orthogonalize(const prsgd_orth_config* cfg, const void* g_dev, int64_t g_matrix, int64_t g_row,
                        void* out_dev, int64_t out_matrix, int64_t out_row, void* workspace_dev, void* hip_stream);

/*
 * One step of momentum with an orthogonalised update on every worker's matrix X:
 *   M <- mu M + G,   U = G + mu M (nesterov != 0) or M,   O = orthogonalise(U),
 *   X <- (1 - lr * weight_decay) X - lr * scale * O.
 * x_dev and g_dev have cfg->dtype, which also says how many bits the products hold; momenta are fp32.  A scale of 0.2 sqrt(max(rows, cols)) gives updates of about the
 * RMS that an elementwise adaptive step has.  The three buffers may not overlap.
 */
int prsgd_muon_step(const prsgd_orth_config* cfg, void* x_dev, int64_t x_matrix, int64_t x_row,
                    const void* g_dev, int64_t g_matrix, int64_t g_row,
                    float* m_dev, int64_t m_matrix, int64_t m_row,
                    float lr, float mu, int32_t nesterov, float weight_decay, float scale,
                    void* workspace_dev, void* hip_stream);

/*
 * Root-mean-square norm of the workers' rows, with the residual's addition:
 *   s = x + res,   rstd = 1 / sqrt(mean(s^2) + eps),   y = s * rstd * w_i
 * for rows_per_worker rows of each of `workers` workers (worker i owns the i-th run of rows and the weights w_i).
 * Sums, statistics and products are fp32 and every output is rounded once; y and rstd go by s as summed, before it is rounded.
 * Rows whose squares overflow fp32, or vanish beside an eps as small, are summed again at another scale (below an RMS of 2.9e-39 under an
 * eps of 0 rstd itself overflows).  A row that holds a
 * NaN or an infinity gives NaN where that is (in 8 bits: everywhere), zeros with an eps of 0 too, and no other row notices.
 */
typedef struct {
  int32_t dtype;                   /* PRSGD_F32 | PRSGD_BF16: type of x, res, s, y and their gradients */
  int32_t workers;                 /* 1..65535                                                       */
  int64_t rows_per_worker;         /* >= 0; workers * rows_per_worker < 2^31                         */
  int32_t width;                   /* 1..16384                                                       */
  float   eps;                     /* >= 0                                                           */
} prsgd_norm_config;

/*
 * y_dev <- y, sum_dev <- s, rstd_dev [rows] <- rstd.  res_dev, sum_dev and rstd_dev may be NULL (no residual, not wanted).
 * w_dev is fp32, w_row elements from worker to worker (0: all share one).  sum_dev and y_dev may each be x_dev or res_dev, if
 * the distances agree; otherwise outputs may not overlap anything.
 */
int prsgd_rms_norm(const prsgd_norm_config* cfg, const void* x_dev, int64_t x_row, const void* res_dev, int64_t res_row,
                   const float* w_dev, int64_t w_row, void* sum_dev, int64_t sum_row, void* y_dev, int64_t y_row,
                   float* rstd_dev, void* hip_stream);

/*
 * The same with y in 8 bits: scale = max(max_j |y_j|, 2^-100) / 448 of each row, q = y / scale rounded to nearest even in
 * e4m3 (4 exponent bits, bias 7, largest 448, no infinities).  q_dev holds bytes, q_row bytes from row to row, and
 * overlaps nothing; scale_dev [rows].
 */
int prsgd_rms_norm_fp8(const prsgd_norm_config* cfg, const void* x_dev, int64_t x_row, const void* res_dev, int64_t res_row,
                       const float* w_dev, int64_t w_row, void* sum_dev, int64_t sum_row, uint8_t* q_dev, int64_t q_row,
                       float* scale_dev, void* hip_stream);

/*
 * Gradients of prsgd_rms_norm from dy (of y) and dsum (of s along the residual path, may be NULL), with sh = s * rstd:
 *   dx = rstd * (w dy - sh mean(w dy sh)) + dsum     (the gradient of x and of res alike)
 *   dw_i = sum over worker i's rows of dy * sh       (fp32, dw_row elements from worker to worker)
 * s_dev and rstd_dev are what the forward call wrote.  dx_dev may be dy_dev, dsum_dev or s_dev if the distances agree.
 * workspace_dev: prsgd_rms_norm_backward_workspace_bytes.  Without rows, dw is zeroed.
 */
size_t prsgd_rms_norm_backward_workspace_bytes(const prsgd_norm_config* cfg);
int prsgd_rms_norm_backward(const prsgd_norm_config* cfg, const void* dy_dev, int64_t dy_row, const void* dsum_dev,
                            int64_t dsum_row, const void* s_dev, int64_t s_row, const float* rstd_dev,
                            const float* w_dev, int64_t w_row, void* dx_dev, int64_t dx_row, float* dw_dev,
                            int64_t dw_row, void* workspace_dev, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* PRSGD_OPS_H */
