// C ABI of the operators on replica sets (prsgd_ops.h): argument checks, workspace layout and launch order.
#include <math.h>
#include <stdio.h>

#include <algorithm>
#include <utility>

#include "prsgd_internal.h"
#include "prsgd_ops_internal.h"

using namespace prsgd;

namespace {

int bad(const char* text) { return op_error(PRSGD_EINVAL, text); }
int hip_result(hipError_t e, const char* what) {
  if (e == hipSuccess) return PRSGD_OK;
  char buf[200];
  snprintf(buf, sizeof(buf), "%s: %s", what, hipGetErrorString(e));
  return op_error(PRSGD_EHIP, buf);
}
size_t align256(size_t v) { return (v + 255) / 256 * 256; }
int element_bytes(int dtype) { return dtype == PRSGD_BF16 ? 2 : 4; }
bool misaligned(const void* p, int bytes) { return (uintptr_t)p % (uintptr_t)bytes != 0; }
// distances between rows (and matrices) whose products with the counts, 2^16 matrices of 2^15 rows, stay far inside 64 bits; rows of norms,
// up to 2^31 of them, are checked against their own number
constexpr int64_t kMaxDistance = (int64_t)1 << 40;
constexpr int64_t kMaxRowSpan = (int64_t)1 << 60;
bool distance_ok(int64_t d, int64_t least) { return d >= least && d <= kMaxDistance; }

// ---- norm ------------------------------------------------------------------------------------

const char* norm_config_error(const prsgd_norm_config* c) {
  if (c == nullptr) return "norm: config is null";
  if (c->dtype != PRSGD_F32 && c->dtype != PRSGD_BF16) return "norm: unknown dtype";
  if (c->workers < 1 || c->workers > 65535) return "norm: workers out of range (1..65535)";
  if (c->rows_per_worker < 0 || c->rows_per_worker >= (1LL << 31) / c->workers) return "norm: rows out of range (below 2^31 in all)";
  if (c->width < 1 || c->width > kMaxNormWidth) return "norm: width out of range (1..16384)";
  if (!(c->eps >= 0.0f) || isinf(c->eps)) return "norm: eps must be finite and not negative";
  return nullptr;
}
// inputs may repeat a row (distance 0), outputs may not
bool rows_ok(const prsgd_norm_config* c, int64_t distance, bool output) {
  if (!distance_ok(distance, output ? c->width : 0) || (distance != 0 && distance < c->width)) return false;
  return distance <= kMaxRowSpan / std::max<int64_t>(1, c->workers * c->rows_per_worker);
}

int norm_forward(const prsgd_norm_config* c, const void* x, int64_t x_row, const void* res, int64_t res_row, const float* w,
                 int64_t w_row, void* sum, int64_t sum_row, void* y, int64_t y_row, float* stat, bool fp8, void* stream) {
  if (const char* e = norm_config_error(c)) return bad(e);
  const int es = element_bytes(c->dtype);
  if (w == nullptr || misaligned(w, 4) || !rows_ok(c, w_row, false)) return bad("norm: weights null, misaligned or overlapping");
  if (c->rows_per_worker == 0) return PRSGD_OK;
  if (x == nullptr || y == nullptr || (fp8 && stat == nullptr)) return bad("norm: null buffer");
  if (misaligned(x, es) || misaligned(res, es) || misaligned(sum, es) || (!fp8 && misaligned(y, es)) || misaligned(stat, 4))
    return bad("norm: misaligned buffer");
  if (!rows_ok(c, x_row, false) || (res != nullptr && !rows_ok(c, res_row, false)) || (sum != nullptr && !rows_ok(c, sum_row, true)) ||
      !rows_ok(c, y_row, true))
    return bad("norm: distance between rows out of range");
  // 8-bit rows lie otherwise than what they would replace
  if (y == sum || (fp8 && (y == x || y == res))) return bad("norm: buffers overlap");
  auto elsewhere = [](const void* out, int64_t out_row, const void* in, int64_t in_row) { return out != nullptr && out == in && out_row != in_row; };
  if (elsewhere(sum, sum_row, x, x_row) || elsewhere(sum, sum_row, res, res_row) || elsewhere(y, y_row, x, x_row) || elsewhere(y, y_row, res, res_row))
    return bad("norm: in place with another distance between rows");
  NormArgs p{};
  p.x = x;
  p.x_row = x_row;
  p.res = res;
  p.res_row = res_row;
  p.w = w;
  p.w_row = w_row;
  p.sum = sum;
  p.sum_row = sum_row;
  p.y = y;
  p.y_row = y_row;
  p.stat = stat;
  p.rows_per_worker = (uint32_t)c->rows_per_worker;
  p.rows = (uint32_t)(c->rows_per_worker * c->workers);
  p.width = c->width;
  p.eps = c->eps;
  return hip_result(launch_rms_norm(p, c->dtype == PRSGD_BF16, fp8, reinterpret_cast<hipStream_t>(stream)), "norm");
}

// ---- orthogonalised updates --------------------------------------------------------------------

// What the polynomial does over the steps, on a grid over where the singular values are (they start in [0, 1]).
struct OrthBounds {
  float gram_growth;                           // product over the steps of the largest slope of A -> Q A Q in an eigenvalue of A
  uint8_t grown[kMaxOrthSteps];                // X in front of step k is below 2^grown[k] |X_0| (or 255)
};
const char* orth_config_error(const prsgd_orth_config* c, OrthBounds* bounds) {
  if (c == nullptr) return "orthogonalize: config is null";
  if (c->dtype != PRSGD_F32 && c->dtype != PRSGD_BF16) return "orthogonalize: unknown dtype";
  if (c->count < 0 || c->count > 65535) return "orthogonalize: count out of range (0..65535)";
  if (c->rows < 1 || c->rows > kMaxOrthSide || c->cols < 1 || c->cols > kMaxOrthSide) return "orthogonalize: sides out of range (1..32768)";
  if (c->steps < 1 || c->steps > kMaxOrthSteps) return "orthogonalize: steps out of range (1..64)";
  if (!(c->eps >= 0.0f) || isinf(c->eps)) return "orthogonalize: eps must be finite and not negative";
  bounds->gram_growth = 1.0f;
  float top = 1.0f, slope = 0.0f, factor = 0.0f, x_growth = 1.0f;
  bool settled = false;                        // steps to come are like the last one
  for (int k = 0; k < c->steps; ++k) {
    int e = 0;
    if (k > 0) (void)frexpf(x_growth, &e);
    bounds->grown[k] = (uint8_t)std::min(e, 255);
    if (!settled) {
      float next = 0.0f;
      slope = c->a * c->a;
      factor = fabsf(c->a);
      for (int i = 1; i <= 32; ++i) {
        const float s = top * (float)i / 32.0f, l = s * s, q = l * (c->b + c->c * l), f = c->a + q, v = fabsf(s * f);
        if (!(fabsf(q) < 7.0f) || !(v < 2.0f)) return "orthogonalize: coefficients leave the range of the products";
        next = std::max(next, v);
        factor = std::max(factor, fabsf(f));
        slope = std::max(slope, fabsf(f * (f + 2.0f * l * (c->b + 2.0f * c->c * l))));
      }
      settled = next == top;
      top = next;
    }
    bounds->gram_growth *= slope;
    x_growth = std::min(x_growth * std::max(factor, 1.0f), 0x1p120f);
  }
  return nullptr;
}

// Workspace of the products' path: halves of every matrix, then the partial sums of squares.
struct OrthPlan {
  bool split;
  int r, longer, ld_x, ld_a;
  size_t x, x_lo, a, b, diag, room, parts, total;    // byte offsets
  int64_t x_gs, a_gs;                          // halves per matrix
};
OrthPlan orth_plan(const prsgd_orth_config* c) {
  OrthPlan p{};
  p.split = c->dtype == PRSGD_F32;
  p.r = c->rows < c->cols ? c->rows : c->cols;
  p.longer = c->rows < c->cols ? c->cols : c->rows;
  p.ld_x = half_ld(p.longer, p.split);
  p.ld_a = half_ld(p.r, p.split);
  p.x_gs = (int64_t)half_rows(p.r) * p.ld_x;
  p.a_gs = (int64_t)p.r * p.ld_a;
  const size_t n = (size_t)c->count;
  size_t at = 0;
  auto take = [&](size_t bytes) { const size_t v = at; at += align256(bytes); return v; };
  p.x = take(2 * n * p.x_gs * 2);
  p.x_lo = p.split ? 0 : take(n * p.x_gs * 2);
  p.a = take(n * p.a_gs * 2);
  p.b = take(n * p.a_gs * 2);
  p.diag = p.split ? 0 : take(n * p.r * 2 * sizeof(float));
  p.room = take(n * sizeof(int));
  p.parts = take(n * norm_parts(c->rows, c->cols) * sizeof(double));
  p.total = at;
  return p;
}
// A short side goes through its Gram matrix while that holds.  An eigenvalue of it that is zero comes out as 2^-52 of the trace, of either
// sign, and grows by the slope at 0, a^2, per step; a negative one leaves every bound once it is about -1 (NaN from 20 default steps on).  Up
// to 2^36 it stays below 2^-16, and errors below those of products of X in fp32: 10 default steps (2e-3 to 6e-3 of the result
// where the side is of lower rank, against 5e-3 to 1e-2), 18 of (2, -1.5, 0.5), 30 of (1.5, -0.5, 0).  Products carry X itself, which any number leaves
// in its range.
bool is_short(const prsgd_orth_config* c, const OrthBounds& b) {
  return (c->rows <= kShortSide || c->cols <= kShortSide) && b.gram_growth <= 0x1p36f;
}
size_t short_bytes(const prsgd_orth_config* c) {
  const int r = c->rows < c->cols ? c->rows : c->cols, longer = c->rows < c->cols ? c->cols : c->rows;
  const int slices = orth_short_slices(c->count, r, longer);
  return align256(slices == 1 ? 256 : (size_t)c->count * slices * orth_short_doubles(r) * sizeof(double));
}

hipError_t run_squares(const prsgd_orth_config* c, const OrthBounds& bounds, const OrthMatrices& m, char* ws, hipStream_t s) {
  const OrthPlan p = orth_plan(c);
  auto halves = [&](size_t offset) { return reinterpret_cast<uint16_t*>(ws + offset); };
  double* parts = reinterpret_cast<double*>(ws + p.parts);
  uint16_t* x = halves(p.x);                   // every product reads all of X while the next one is written
  uint16_t* y = x + (size_t)c->count * p.x_gs;
  uint16_t* x_lo = p.split ? nullptr : halves(p.x_lo);
  uint16_t* a = halves(p.a);
  uint16_t* b = halves(p.b);
  int* room = reinterpret_cast<int*>(ws + p.room);
  const float inv = 1.0f / kHalfScale;

  hipError_t e = launch_orth_squares(m, parts, s);
  if (e != hipSuccess) return e;
  e = launch_orth_load(m, parts, OrthHalves{x, x_lo, y, p.x_gs, p.ld_x, room}, s);
  for (int k = 0; k < c->steps && e == hipSuccess; ++k) {
    SquareArgs q{};
    q.count = c->count;
    q.room = room;
    q.grown = bounds.grown[k];
    q.grown_next = bounds.grown[std::min(k + 1, c->steps - 1)];
    if (!p.split) q.diag = reinterpret_cast<float*>(ws + p.diag);
    // A = X X^T
    q.a = q.b = x;
    q.a_gs = q.b_gs = p.x_gs;
    q.lda = q.ldb = p.ld_x;
    q.M = q.N = p.r;
    q.out = q.out_t = a;
    q.out_gs = q.t_gs = p.a_gs;
    q.ldo = q.ldt = p.ld_a;
    q.beta = inv;
    if ((e = launch_square(q, SQ_GRAM, p.split, s)) != hipSuccess) break;
    // B = b A + c A A
    q.a = q.b = q.lin = a;
    q.a_gs = q.b_gs = q.lin_gs = p.a_gs;
    q.lda = q.ldb = q.ld_lin = p.ld_a;
    q.out = q.out_t = b;
    q.alpha = c->b;
    q.beta = c->c * inv;
    if ((e = launch_square(q, SQ_POLY, p.split, s)) != hipSuccess) break;
    // X <- a X + B X
    q.a = b;
    q.b = x;
    q.b_gs = p.x_gs;
    q.ldb = p.ld_x;
    q.N = p.longer;
    q.lin = x;
    q.lin_lo = x_lo;
    q.lin_gs = p.x_gs;
    q.ld_lin = p.ld_x;
    if (k + 1 < c->steps) {
      q.out = y;
      q.out_lo = x_lo;
      q.out_gs = p.x_gs;
      q.ldo = p.ld_x;
      q.alpha = c->a;
      q.beta = inv;
      q.diag_scale = 1.0f;
      e = launch_square(q, SQ_NEXT, p.split, s);
      std::swap(x, y);
    } else {
      q.user = m;
      q.transposed = c->rows > c->cols;
      q.alpha = c->a * inv;
      q.beta = inv * inv;
      q.diag_scale = inv;
      e = launch_square(q, SQ_LAST, p.split, s);
    }
  }
  return e;
}

int run_orth(const prsgd_orth_config* c, const OrthBounds& bounds, OrthMatrices m, void* ws, void* stream, const char* what) {
  m.count = c->count;
  m.rows = c->rows;
  m.cols = c->cols;
  m.bf16 = c->dtype == PRSGD_BF16;
  m.eps = c->eps;
  m.a = c->a;
  m.b = c->b;
  m.c = c->c;
  m.steps = c->steps;
  const hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  if (is_short(c, bounds)) {
    const int slices = c->rows < c->cols ? orth_short_slices(c->count, c->rows, c->cols) : orth_short_slices(c->count, c->cols, c->rows);
    return hip_result(launch_orth_short(m, reinterpret_cast<double*>(ws), slices, s), what);
  }
  return hip_result(run_squares(c, bounds, m, reinterpret_cast<char*>(ws), s), what);
}

// matrices of a caller: rows apart by at least a row, matrices by at least a matrix (inputs and outputs alike)
bool matrices_ok(const prsgd_orth_config* c, int64_t matrix, int64_t row) {
  if (!distance_ok(row, c->rows > 1 ? c->cols : 0)) return false;
  return distance_ok(matrix, c->count > 1 ? (int64_t)(c->rows - 1) * row + c->cols : 0);
}

}  // namespace

extern "C" {

size_t prsgd_orthogonalize_workspace_bytes(const prsgd_orth_config* cfg) {
  OrthBounds bounds;
  if (const char* e = orth_config_error(cfg, &bounds)) {
    bad(e);
    return 0;
  }
  if (cfg->count == 0) return 0;
  return is_short(cfg, bounds) ? short_bytes(cfg) : orth_plan(cfg).total;
}

int prsgd_orthogonalize(const prsgd_orth_config* cfg, const void* g_dev, int64_t g_matrix, int64_t g_row, void* out_dev,
                        int64_t out_matrix, int64_t out_row, void* workspace_dev, void* hip_stream) {
  OrthBounds bounds;
  if (const char* e = orth_config_error(cfg, &bounds)) return bad(e);
  if (cfg->count == 0) return PRSGD_OK;
  if (g_dev == nullptr || out_dev == nullptr || workspace_dev == nullptr) return bad("orthogonalize: null buffer");
  const int es = element_bytes(cfg->dtype);
  if (misaligned(g_dev, es) || misaligned(out_dev, es) || misaligned(workspace_dev, 256)) return bad("orthogonalize: misaligned buffer");
  if (!matrices_ok(cfg, g_matrix, g_row) || !matrices_ok(cfg, out_matrix, out_row)) return bad("orthogonalize: distance between rows or matrices out of range");
  if (g_dev == out_dev && (g_row != out_row || g_matrix != out_matrix)) return bad("orthogonalize: in place with other distances");
  OrthMatrices m{};
  m.g = g_dev;
  m.g_matrix = g_matrix;
  m.g_row = g_row;
  m.out = out_dev;
  m.out_matrix = out_matrix;
  m.out_row = out_row;
  return run_orth(cfg, bounds, m, workspace_dev, hip_stream, "orthogonalize");
}

int prsgd_muon_step(const prsgd_orth_config* cfg, void* x_dev, int64_t x_matrix, int64_t x_row, const void* g_dev, int64_t g_matrix,
                    int64_t g_row, float* m_dev, int64_t m_matrix, int64_t m_row, float lr, float mu, int32_t nesterov,
                    float weight_decay, float scale, void* workspace_dev, void* hip_stream) {
  OrthBounds bounds;
  if (const char* e = orth_config_error(cfg, &bounds)) return bad(e);
  if (!(mu >= 0.0f && mu < 1.0f)) return bad("muon_step: momentum must be in [0, 1)");
  if (!isfinite(lr) || !isfinite(weight_decay) || !isfinite(scale)) return bad("muon_step: rate, decay or scale is not finite");
  if (cfg->count == 0) return PRSGD_OK;
  if (x_dev == nullptr || g_dev == nullptr || m_dev == nullptr || workspace_dev == nullptr) return bad("muon_step: null buffer");
  const int es = element_bytes(cfg->dtype);
  if (misaligned(x_dev, es) || misaligned(g_dev, es) || misaligned(m_dev, 4) || misaligned(workspace_dev, 256)) return bad("muon_step: misaligned buffer");
  if (!matrices_ok(cfg, x_matrix, x_row) || !matrices_ok(cfg, g_matrix, g_row) || !matrices_ok(cfg, m_matrix, m_row))
    return bad("muon_step: distance between rows or matrices out of range");
  if (x_dev == g_dev || x_dev == (void*)m_dev || g_dev == (const void*)m_dev) return bad("muon_step: buffers overlap");
  OrthMatrices m{};
  m.g = g_dev;
  m.g_matrix = g_matrix;
  m.g_row = g_row;
  m.out = x_dev;
  m.out_matrix = x_matrix;
  m.out_row = x_row;
  m.m = m_dev;
  m.m_matrix = m_matrix;
  m.m_row = m_row;
  m.mu = mu;
  m.g_part = nesterov != 0 ? 1.0f : 0.0f;
  m.m_part = nesterov != 0 ? mu : 1.0f;
  m.keep = 1.0f - lr * weight_decay;
  m.step = lr * scale;
  return run_orth(cfg, bounds, m, workspace_dev, hip_stream, "muon_step");
}

int prsgd_rms_norm(const prsgd_norm_config* cfg, const void* x_dev, int64_t x_row, const void* res_dev, int64_t res_row,
                   const float* w_dev, int64_t w_row, void* sum_dev, int64_t sum_row, void* y_dev, int64_t y_row,
                   float* rstd_dev, void* hip_stream) {
  return norm_forward(cfg, x_dev, x_row, res_dev, res_row, w_dev, w_row, sum_dev, sum_row, y_dev, y_row, rstd_dev, false, hip_stream);
}

int prsgd_rms_norm_fp8(const prsgd_norm_config* cfg, const void* x_dev, int64_t x_row, const void* res_dev, int64_t res_row,
                       const float* w_dev, int64_t w_row, void* sum_dev, int64_t sum_row, uint8_t* q_dev, int64_t q_row,
                       float* scale_dev, void* hip_stream) {
  return norm_forward(cfg, x_dev, x_row, res_dev, res_row, w_dev, w_row, sum_dev, sum_row, q_dev, q_row, scale_dev, true, hip_stream);
}

size_t prsgd_rms_norm_backward_workspace_bytes(const prsgd_norm_config* cfg) {
  if (const char* e = norm_config_error(cfg)) {
    bad(e);
    return 0;
  }
  const size_t floats = norm_back_share_floats(cfg->workers, cfg->rows_per_worker, cfg->width, cfg->dtype == PRSGD_BF16);
  return floats == 0 ? 256 : align256(floats * sizeof(float));
}

int prsgd_rms_norm_backward(const prsgd_norm_config* cfg, const void* dy_dev, int64_t dy_row, const void* dsum_dev, int64_t dsum_row,
                            const void* s_dev, int64_t s_row, const float* rstd_dev, const float* w_dev, int64_t w_row, void* dx_dev,
                            int64_t dx_row, float* dw_dev, int64_t dw_row, void* workspace_dev, void* hip_stream) {
  if (const char* e = norm_config_error(cfg)) return bad(e);
  const int es = element_bytes(cfg->dtype);
  if (w_dev == nullptr || misaligned(w_dev, 4) || !rows_ok(cfg, w_row, false)) return bad("norm: weights null, misaligned or overlapping");
  if (dw_dev == nullptr || misaligned(dw_dev, 4) || !distance_ok(dw_row, cfg->workers > 1 ? cfg->width : 0))
    return bad("norm: weight gradients null, misaligned or overlapping");
  NormArgs p{};
  if (cfg->rows_per_worker > 0) {
    if (dy_dev == nullptr || s_dev == nullptr || rstd_dev == nullptr || dx_dev == nullptr || workspace_dev == nullptr) return bad("norm: null buffer");
    if (misaligned(dy_dev, es) || misaligned(dsum_dev, es) || misaligned(s_dev, es) || misaligned(dx_dev, es) || misaligned(rstd_dev, 4) ||
        misaligned(workspace_dev, 256))
      return bad("norm: misaligned buffer");
    if (!rows_ok(cfg, dy_row, false) || (dsum_dev != nullptr && !rows_ok(cfg, dsum_row, false)) || !rows_ok(cfg, s_row, false) ||
        !rows_ok(cfg, dx_row, true))
      return bad("norm: distance between rows out of range");
    if ((dx_dev == dy_dev && dx_row != dy_row) || (dx_dev == dsum_dev && dx_row != dsum_row) || (dx_dev == s_dev && dx_row != s_row))
      return bad("norm: in place with another distance between rows");
  }
  p.x = dy_dev;
  p.x_row = dy_row;
  p.res = dsum_dev;
  p.res_row = dsum_row;
  p.sum = const_cast<void*>(s_dev);
  p.sum_row = s_row;
  p.stat = const_cast<float*>(rstd_dev);
  p.w = w_dev;
  p.w_row = w_row;
  p.y = dx_dev;
  p.y_row = dx_row;
  p.dw = dw_dev;
  p.dw_row = dw_row;
  p.rows_per_worker = (uint32_t)cfg->rows_per_worker;
  p.rows = (uint32_t)(cfg->rows_per_worker * cfg->workers);
  p.width = cfg->width;
  return hip_result(launch_rms_norm_backward(p, reinterpret_cast<float*>(workspace_dev), cfg->workers, cfg->dtype == PRSGD_BF16,
                                             reinterpret_cast<hipStream_t>(hip_stream)), "norm backward");
}

}  // extern "C"
