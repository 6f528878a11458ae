/*
 * prsgd_ops.h -- operators on replica sets exported by libprsgd beside the method's own calls (prsgd.h): the
 * orthogonalised update of every worker's weight matrix, the root-mean-square norm of every worker's rows, and what replicas of
 * a model over tokens need beside them: embedding, gated linear recurrence, dropout and the cross entropy of the last layer.
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

/*
 * Embedding: row r of worker i becomes scale times row token[r] of the worker's table T_i [classes][width], rounded once.  A
 * token below 0 or from `classes` on is padding: a row of zeros, and no gradient.
 */
typedef struct {
  int32_t dtype;                   /* PRSGD_F32 | PRSGD_BF16: type of tables, rows and gradients     */
  int32_t workers;                 /* 1..65535                                                       */
  int64_t rows_per_worker;         /* >= 0; workers * rows_per_worker < 2^31; backward: up to 2^24   */
  int32_t classes;                 /* 1..2^20                                                        */
  int32_t width;                   /* 1..32768                                                       */
  float   scale;                   /* finite                                                         */
} prsgd_embedding_config;

/* tokens_dev [workers * rows_per_worker]; worker i's table starts at + i * table_matrix elements (0: all share one). */
int prsgd_embedding(const prsgd_embedding_config* cfg, const int32_t* tokens_dev, const void* table_dev, int64_t table_matrix,
                    int64_t table_row, void* y_dev, int64_t y_row, void* hip_stream);

/*
 * dT_i[v] = scale * sum of the rows dy[r] of worker i whose token is v: fp32 sums in the order of the rows, in whole groups of them where
 * a token has many, rounded once.  Every row of dtable is written, with zeros where no token names it.
 */
size_t prsgd_embedding_backward_workspace_bytes(const prsgd_embedding_config* cfg);
int prsgd_embedding_backward(const prsgd_embedding_config* cfg, const int32_t* tokens_dev, const void* dy_dev, int64_t dy_row,
                             void* dtable_dev, int64_t dtable_matrix, int64_t dtable_row, void* workspace_dev, void* hip_stream);

/*
 * Gated linear recurrence along every sequence, channel by channel:
 *   f_t = 1 / (1 + exp(-gate_t)),   h_t = f_t h_{t-1} + (1 - f_t) v_t,
 * from `initial` (fp32, zeros if NULL) to `last` (fp32, behind the sequence's last row; `initial` if it has none).  States are fp32,
 * h is each rounded once.  starts_dev [sequences + 1] (int32, ascending): sequence s has the rows starts[s] .. starts[s + 1] - 1;
 * rows before the first and behind the last are not read, and written as `clear` says.  NULL: `sequences` equal runs of all rows, one behind
 * another (sequences of one row are a step of generation).  What starts_dev holds past 0 .. rows is taken as the nearest of these.
 * A NaN or an infinity stays in its channel of its sequence.
 */
typedef struct {
  int32_t dtype;                   /* PRSGD_F32 | PRSGD_BF16: type of v, gate, h and their gradients */
  int32_t sequences;               /* 1..2^24, and below 2^31 / ceil(width / 64)                     */
  int64_t rows;                    /* 0..2^30 in all; without starts a multiple of sequences         */
  int32_t width;                   /* 1..32768                                                       */
  int32_t clear;                   /* rows before the first sequence and behind the last: 0 left as they are; 1 zeros in h (backward: dv);
                                      2 zeros in dgate; 3 both                                       */
} prsgd_scan_config;

/* Bytes of workspace of either call below: 0 if they need none (few long sequences do) or the configuration is invalid. */
size_t prsgd_gated_scan_workspace_bytes(const prsgd_scan_config* cfg);

/*
 * last_dev may be NULL, and may be initial_dev if the distances agree.  No other buffers may overlap.  workspace_dev may be NULL
 * where none is needed.
 */
int prsgd_gated_scan(const prsgd_scan_config* cfg, const int32_t* starts_dev, const void* v_dev, int64_t v_row,
                     const void* gate_dev, int64_t gate_row, const float* initial_dev, int64_t initial_row, void* h_dev,
                     int64_t h_row, float* last_dev, int64_t last_row, void* workspace_dev, void* hip_stream);

/*
 * Gradients from dh and dlast (NULL: zeros), with g_t = dh_t + f_{t+1} g_{t+1} (behind the last row: dlast):
 *   dv_t = (1 - f_t) g_t,   dgate_t = f_t (1 - f_t) (h_{t-1} - v_t) g_t,   dinitial = f_1 g_1  (of an empty sequence: dlast)
 * h_dev is what the forward call wrote.  dinitial_dev may be NULL, and may be dlast_dev if the distances agree.
 */
int prsgd_gated_scan_backward(const prsgd_scan_config* cfg, const int32_t* starts_dev, const void* dh_dev, int64_t dh_row,
                              const void* v_dev, int64_t v_row, const void* gate_dev, int64_t gate_row, const void* h_dev,
                              int64_t h_row, const float* initial_dev, int64_t initial_row, const float* dlast_dev,
                              int64_t dlast_row, void* dv_dev, int64_t dv_row, void* dgate_dev, int64_t dgate_row,
                              float* dinitial_dev, int64_t dinitial_row, void* workspace_dev, void* hip_stream);

/*
 * Dropout: y = res + keep x / (1 - q), q = round(65536 p) / 65536, with a mask that is a function of (seed, step, layer, row, column):
 * eight elements j of a row share block = row * ceil(width / 8) + column / 8, and the words of
 *   Philox4x32-10(counter (block mod 2^32, step mod 2^32, step >> 32, (block >> 32) + 2^31 + 2^16 layer), key (seed mod 2^32, seed >> 32));
 * element j goes by 16 bits, the low (j even) or high half of word j / 2, and is dropped if they are below 65536 q.  What is dropped
 * adds nothing, also where it is no number.  The gradient of x is the same call on dy without a residual; that of res is dy.
 * (Minibatches are drawn from counters whose last word is below 2^31.)
 */
typedef struct {
  int32_t  dtype;                  /* PRSGD_F32 | PRSGD_BF16: type of x, res and y                   */
  int32_t  layer;                  /* 0..32767: calls of one step that differ in it have masks of their own */
  int64_t  rows;                   /* 0..2^31 - 1                                                    */
  int32_t  width;                  /* 1..32768                                                       */
  float    p;                      /* 0 <= p, round(65536 p) < 65536                                 */
  uint64_t seed;
  uint64_t step;
} prsgd_dropout_config;

/*
 * res_dev may be NULL.  step_dev (may be NULL): an int64 on the device that takes the place of cfg->step, read when the call
 * runs, so that replays of a captured call can have masks of their own.  y_dev may be x_dev or res_dev if the distances agree.
 */
int prsgd_dropout(const prsgd_dropout_config* cfg, const int64_t* step_dev, const void* x_dev, int64_t x_row, const void* res_dev,
                  int64_t res_row, void* y_dev, int64_t y_row, void* hip_stream);

/*
 * Softmax cross entropy of the workers' rows h through their last matrices W_i, whose logits are never stored whole:
 *   z = h W_i (classes_first: W_i is [classes][width] and z = h W_i^T),   lse = log sum exp z,   loss = lse - z[label].
 * A label below 0 or from `classes` on is padding: its row has a loss of 0 (and its lse).  Products of bf16 are summed in
 * fp32, products of fp32 are fp32; loss and lse are fp32.  A NaN or +infinity among a row's logits makes its loss and lse NaN.
 */
typedef struct {
  int32_t dtype;                   /* PRSGD_F32 | PRSGD_BF16: type of h, W and their gradients       */
  int32_t workers;                 /* 1..65535                                                       */
  int64_t rows_per_worker;         /* 0..2^31 - 256; workers * rows_per_worker < 2^31                */
  int32_t width;                   /* 1..32768                                                       */
  int32_t classes;                 /* 1..2^20                                                        */
  int32_t classes_first;           /* 0: W_i [width][classes]; 1: [classes][width], as a table of embeddings */
} prsgd_xent_config;

/*
 * labels_dev, loss_dev, lse_dev [workers * rows_per_worker]; w_matrix elements from worker to worker (0: all share one).  The workspace
 * holds 8 bytes a row for every tile of classes, 32 of them where products are small, 128 or 256 where they are large.
 */
size_t prsgd_linear_cross_entropy_workspace_bytes(const prsgd_xent_config* cfg);
int prsgd_linear_cross_entropy(const prsgd_xent_config* cfg, const void* h_dev, int64_t h_row, const void* w_dev,
                               int64_t w_matrix, int64_t w_row, const int32_t* labels_dev, float* loss_dev, float* lse_dev,
                               void* workspace_dev, void* hip_stream);

/*
 * Gradients from dloss [rows] (of every row's loss), with lse as the forward call wrote it:
 *   dz = dloss (exp(z - lse) - onehot(label)),   dh = dz W_i^T,   dW_i = sum over worker i's rows of h dz,
 * each rounded once from fp32 sums; dz itself, which the products take, is held in the rows' type.  Rows without a label get a dh of
 * zeros and are no part of dW, whatever h, lse and dloss hold there.  dw has W's layout; every worker has its own.  Without rows it is
 * zeros.  Classes are taken in pieces, of which the workspace holds one (256 MiB, or 256 classes if those are more).
 */
size_t prsgd_linear_cross_entropy_backward_workspace_bytes(const prsgd_xent_config* cfg);
int prsgd_linear_cross_entropy_backward(const prsgd_xent_config* cfg, const float* dloss_dev, const void* h_dev, int64_t h_row,
                                        const void* w_dev, int64_t w_matrix, int64_t w_row, const int32_t* labels_dev,
                                        const float* lse_dev, void* dh_dev, int64_t dh_row, void* dw_dev, int64_t dw_matrix,
                                        int64_t dw_row, void* workspace_dev, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* PRSGD_OPS_H */
