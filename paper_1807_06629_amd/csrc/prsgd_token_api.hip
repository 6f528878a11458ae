// C ABI of the operators of replicas of a model over tokens (prsgd_ops.h): argument checks and workspace layout.
#include <math.h>
#include <stdio.h>

#include <algorithm>

#include "prsgd_ops_internal.h"
#include "prsgd_token_internal.h"

using namespace prsgd;

namespace {

int bad(const char* text) { return op_error(PRSGD_EINVAL, text); }
int hip_result(hipError_t e, const char* what) {
  if (e == hipSuccess) return PRSGD_OK;
  char buf[200];
  snprintf(buf, sizeof(buf), "%s: %s", what, hipGetErrorString(e));
  return op_error(PRSGD_EHIP, buf);
}
int element_bytes(int dtype) { return dtype == PRSGD_BF16 ? 2 : 4; }
bool type_ok(int dtype) { return dtype == PRSGD_F32 || dtype == PRSGD_BF16; }
bool misaligned(const void* p, int bytes) { return (uintptr_t)p % (uintptr_t)bytes != 0; }

// The last element of `count` rows (or matrices) that lie d elements apart is within 2^60 elements of the first; inputs may repeat a row (distance 0).
constexpr int64_t kMaxDistance = (int64_t)1 << 40, kMaxSpan = (int64_t)1 << 60;
bool rows_ok(int64_t count, int64_t width, int64_t d, bool output) {
  if (count <= 1) return d >= 0 && d <= kMaxDistance;
  return d <= kMaxDistance && d <= kMaxSpan / count && (d >= width || (d == 0 && !output));
}
// matrices [rows][cols] of `count` workers; inputs may share one (distance 0)
bool matrices_ok(int64_t count, int64_t rows, int64_t cols, int64_t matrix, int64_t row, bool output) {
  if (!rows_ok(rows, cols, row, true)) return false;
  return rows_ok(count, (rows - 1) * row + cols, matrix, output);
}
constexpr int64_t kMaxRows = ((int64_t)1 << 31) - 1;
bool rows_of_workers_ok(int workers, int64_t rows) { return workers >= 1 && workers <= 65535 && rows >= 0 && rows <= kMaxRows / workers; }
bool width_ok(int width) { return width >= 1 && width <= kMaxTokenWidth; }
bool classes_ok(int classes) { return classes >= 1 && classes <= kMaxClasses; }

// ---- embedding ---------------------------------------------------------------------------------

constexpr int64_t kMaxSortedRows = (int64_t)1 << 24;
const char* embedding_error(const prsgd_embedding_config* c, bool backward) {
  if (c == nullptr) return "embedding: config is null";
  if (!type_ok(c->dtype)) return "embedding: unknown dtype";
  if (!rows_of_workers_ok(c->workers, c->rows_per_worker)) return "embedding: workers (1..65535) or rows (below 2^31 in all) out of range";
  if (backward && c->rows_per_worker > kMaxSortedRows) return "embedding: more than 2^24 rows of a worker";
  if (!classes_ok(c->classes)) return "embedding: classes out of range (1..2^20)";
  if (!width_ok(c->width)) return "embedding: width out of range (1..32768)";
  if (!isfinite(c->scale)) return "embedding: scale must be finite";
  return nullptr;
}
EmbeddingArgs embedding_args(const prsgd_embedding_config* c) {
  EmbeddingArgs p{};
  p.workers = c->workers;
  p.rows = c->rows_per_worker;
  p.classes = c->classes;
  p.width = c->width;
  p.scale = c->scale;
  return p;
}

// ---- scan --------------------------------------------------------------------------------------

constexpr int64_t kMaxScanRows = (int64_t)1 << 30;
const char* scan_error(const prsgd_scan_config* c, const int32_t* starts, int clear) {
  if (c == nullptr) return "gated_scan: config is null";
  if (!type_ok(c->dtype)) return "gated_scan: unknown dtype";
  if (c->sequences < 1 || c->sequences > (1 << 24)) return "gated_scan: sequences out of range (1..2^24)";
  if (c->rows < 0 || c->rows > kMaxScanRows) return "gated_scan: rows out of range (0..2^30)";
  if (!width_ok(c->width)) return "gated_scan: width out of range (1..32768)";
  if ((int64_t)c->sequences * ((c->width + 63) / 64) > kMaxRows - 64) return "gated_scan: sequences times width out of range";
  if (c->clear < 0 || c->clear > clear) return "gated_scan: clear out of range";
  if (starts == nullptr && c->rows % c->sequences != 0) return "gated_scan: rows must be a multiple of the sequences where these have no starts";
  if (misaligned(starts, 4)) return "gated_scan: misaligned buffer";
  return nullptr;
}
int parts_of(const prsgd_scan_config* c, const int32_t* starts, bool backward) {
  return scan_parts(c->sequences, c->rows, c->width, element_bytes(c->dtype), starts != nullptr, backward);
}
size_t joint_bytes(const prsgd_scan_config* c, int parts) { return ((size_t)parts * c->width * sizeof(float2) + 255) / 256 * 256; }
size_t scan_bytes(const prsgd_scan_config* c) {
  // of any of the calls that the configuration allows
  int most = 1;
  for (int k = 0; k < 4; ++k) most = std::max(most, scan_parts(c->sequences, c->rows, c->width, element_bytes(c->dtype), (k & 1) != 0, (k & 2) != 0));
  return most > 1 ? joint_bytes(c, most) + (size_t)c->sequences * c->width * sizeof(float) : 0;
}
void set_parts(ScanArgs& p, const prsgd_scan_config* c, bool backward, void* workspace) {
  p.parts = parts_of(c, p.starts, backward);
  if (p.parts <= 1) return;
  p.joint = reinterpret_cast<float2*>(workspace);
  p.aside = reinterpret_cast<float*>(reinterpret_cast<char*>(workspace) + joint_bytes(c, p.parts));
}
struct ScanBuffer { const void* at; int64_t row; bool output, needed; };
// Rows in the sequences' type and states in fp32: present, aligned, distances, and outputs nowhere else.
const char* scan_buffers_error(const prsgd_scan_config* c, const ScanBuffer* rows, int n_rows, const ScanBuffer* states, int n_states, const void* workspace) {
  if ((workspace == nullptr && scan_bytes(c) > 0) || misaligned(workspace, 256)) return "gated_scan: null or misaligned workspace";
  const int es = element_bytes(c->dtype);
  for (int i = 0; i < n_rows; ++i) {
    if (c->rows == 0) break;
    if (rows[i].at == nullptr) return "gated_scan: null buffer";
    if (misaligned(rows[i].at, es)) return "gated_scan: misaligned buffer";
    if (!rows_ok(c->rows, c->width, rows[i].row, rows[i].output)) return "gated_scan: distance between rows out of range";
    for (int j = 0; j < n_rows; ++j)
      if (j != i && rows[i].output && rows[i].at == rows[j].at) return "gated_scan: buffers overlap";
  }
  for (int i = 0; i < n_states; ++i) {
    if (states[i].at == nullptr) {
      if (states[i].needed) return "gated_scan: null buffer";
      continue;
    }
    if (misaligned(states[i].at, 4)) return "gated_scan: misaligned buffer";
    if (!rows_ok(c->sequences, c->width, states[i].row, states[i].output)) return "gated_scan: distance between states out of range";
    for (int j = 0; j < n_rows && c->rows > 0; ++j)
      if ((states[i].output || rows[j].output) && states[i].at == rows[j].at) return "gated_scan: buffers overlap";
  }
  return nullptr;
}

// ---- cross entropy -----------------------------------------------------------------------------

// Tiles of up to 256 rows are counted in 32 bits.
constexpr int64_t kMaxTiledRows = ((int64_t)1 << 31) - 256;
const char* xent_error(const prsgd_xent_config* c) {
  if (c == nullptr) return "linear_cross_entropy: config is null";
  if (!type_ok(c->dtype)) return "linear_cross_entropy: unknown dtype";
  if (!rows_of_workers_ok(c->workers, c->rows_per_worker)) return "linear_cross_entropy: workers (1..65535) or rows (below 2^31 in all) out of range";
  if (c->rows_per_worker > kMaxTiledRows) return "linear_cross_entropy: more than 2^31 - 256 rows of a worker";
  if (!classes_ok(c->classes)) return "linear_cross_entropy: classes out of range (1..2^20)";
  if (!width_ok(c->width)) return "linear_cross_entropy: width out of range (1..32768)";
  if (c->classes_first != 0 && c->classes_first != 1) return "linear_cross_entropy: classes_first must be 0 or 1";
  // workgroups of a launch
  auto tiles = [](int64_t n) { return (n + 31) / 32; };
  const int64_t r = tiles(c->rows_per_worker), w = tiles(c->width), k = tiles(c->classes), most = kMaxRows / c->workers;
  if (r > 0 && (w > most / r || k > most / r)) return "linear_cross_entropy: rows times classes or width out of range";
  if (w > most / k) return "linear_cross_entropy: width times classes out of range";
  return nullptr;
}
int64_t matrix_rows(const prsgd_xent_config* c) { return c->classes_first != 0 ? c->classes : c->width; }
int64_t matrix_cols(const prsgd_xent_config* c) { return c->classes_first != 0 ? c->width : c->classes; }
XentArgs xent_args(const prsgd_xent_config* c) {
  XentArgs p{};
  p.workers = c->workers;
  p.rows = c->rows_per_worker;
  p.width = c->width;
  p.classes = c->classes;
  p.classes_first = c->classes_first != 0;
  return p;
}
XentPlan plan_of(const prsgd_xent_config* c, bool backward) {
  return xent_plan(c->workers, c->rows_per_worker, c->width, c->classes, c->classes_first != 0, c->dtype == PRSGD_BF16, backward);
}
size_t xent_bytes(const prsgd_xent_config* c, bool backward) {
  if (const char* e = xent_error(c)) {
    bad(e);
    return 0;
  }
  return std::max<size_t>(plan_of(c, backward).total, 256);
}

}  // namespace

extern "C" {

int prsgd_embedding(const prsgd_embedding_config* cfg, const int32_t* tokens_dev, const void* table_dev, int64_t table_matrix,
                    int64_t table_row, void* y_dev, int64_t y_row, void* hip_stream) {
  if (const char* e = embedding_error(cfg, false)) return bad(e);
  if (cfg->rows_per_worker == 0) return PRSGD_OK;
  const int es = element_bytes(cfg->dtype);
  if (tokens_dev == nullptr || table_dev == nullptr || y_dev == nullptr) return bad("embedding: null buffer");
  if (misaligned(tokens_dev, 4) || misaligned(table_dev, es) || misaligned(y_dev, es)) return bad("embedding: misaligned buffer");
  if (!matrices_ok(cfg->workers, cfg->classes, cfg->width, table_matrix, table_row, false)) return bad("embedding: distance between tables or their rows out of range");
  if (!rows_ok(cfg->rows_per_worker * cfg->workers, cfg->width, y_row, true)) return bad("embedding: distance between rows out of range");
  if (y_dev == table_dev || (const void*)tokens_dev == y_dev) return bad("embedding: buffers overlap");
  EmbeddingArgs p = embedding_args(cfg);
  p.tokens = tokens_dev;
  p.table = table_dev;
  p.table_gs = table_matrix;
  p.table_row = table_row;
  p.y = y_dev;
  p.y_row = y_row;
  return hip_result(launch_embedding(p, cfg->dtype == PRSGD_BF16, reinterpret_cast<hipStream_t>(hip_stream)), "embedding");
}

size_t prsgd_embedding_backward_workspace_bytes(const prsgd_embedding_config* cfg) {
  if (const char* e = embedding_error(cfg, true)) {
    bad(e);
    return 0;
  }
  return embedding_plan(cfg->workers, cfg->rows_per_worker, cfg->width).total;
}

int prsgd_embedding_backward(const prsgd_embedding_config* cfg, const int32_t* tokens_dev, const void* dy_dev, int64_t dy_row,
                             void* dtable_dev, int64_t dtable_matrix, int64_t dtable_row, void* workspace_dev, void* hip_stream) {
  if (const char* e = embedding_error(cfg, true)) return bad(e);
  const int es = element_bytes(cfg->dtype);
  if (dtable_dev == nullptr || workspace_dev == nullptr) return bad("embedding: null buffer");
  if (misaligned(dtable_dev, es) || misaligned(workspace_dev, 256)) return bad("embedding: misaligned buffer");
  if (!matrices_ok(cfg->workers, cfg->classes, cfg->width, dtable_matrix, dtable_row, true)) return bad("embedding: distance between tables or their rows out of range");
  if (cfg->rows_per_worker > 0) {
    if (tokens_dev == nullptr || dy_dev == nullptr) return bad("embedding: null buffer");
    if (misaligned(tokens_dev, 4) || misaligned(dy_dev, es)) return bad("embedding: misaligned buffer");
    if (!rows_ok(cfg->rows_per_worker * cfg->workers, cfg->width, dy_row, false)) return bad("embedding: distance between rows out of range");
    if (dy_dev == dtable_dev || (const void*)tokens_dev == dtable_dev) return bad("embedding: buffers overlap");
  }
  EmbeddingArgs p = embedding_args(cfg);
  p.tokens = tokens_dev;
  p.y = const_cast<void*>(dy_dev);
  p.y_row = dy_row;
  p.dtable = dtable_dev;
  p.dtable_gs = dtable_matrix;
  p.dtable_row = dtable_row;
  return hip_result(launch_embedding_backward(p, embedding_plan(cfg->workers, cfg->rows_per_worker, cfg->width),
                                              reinterpret_cast<char*>(workspace_dev), cfg->dtype == PRSGD_BF16,
                                              reinterpret_cast<hipStream_t>(hip_stream)), "embedding backward");
}

size_t prsgd_gated_scan_workspace_bytes(const prsgd_scan_config* cfg) {
  // sequences that are given no starts have to be equal in the call itself
  const int32_t* const some = reinterpret_cast<const int32_t*>(sizeof(int32_t));
  if (const char* e = scan_error(cfg, some, 3)) {
    bad(e);
    return 0;
  }
  return scan_bytes(cfg);
}

int prsgd_gated_scan(const prsgd_scan_config* cfg, const int32_t* starts_dev, const void* v_dev, int64_t v_row, const void* gate_dev,
                     int64_t gate_row, const float* initial_dev, int64_t initial_row, void* h_dev, int64_t h_row, float* last_dev,
                     int64_t last_row, void* workspace_dev, void* hip_stream) {
  if (const char* e = scan_error(cfg, starts_dev, 1)) return bad(e);
  const ScanBuffer rows[] = {{v_dev, v_row, false, true}, {gate_dev, gate_row, false, true}, {h_dev, h_row, true, true}};
  const ScanBuffer states[] = {{initial_dev, initial_row, false, false}, {last_dev, last_row, true, false}};
  if (const char* e = scan_buffers_error(cfg, rows, 3, states, 2, workspace_dev)) return bad(e);
  if (last_dev != nullptr && last_dev == initial_dev && last_row != initial_row) return bad("gated_scan: state in place with another distance");
  ScanArgs p{};
  p.starts = starts_dev;
  p.v = v_dev;
  p.v_row = v_row;
  p.gate = gate_dev;
  p.gate_row = gate_row;
  p.initial = initial_dev;
  p.initial_row = initial_row;
  p.h = h_dev;
  p.h_row = h_row;
  p.last = last_dev;
  p.last_row = last_row;
  p.sequences = cfg->sequences;
  p.clear = cfg->clear;
  p.rows = cfg->rows;
  p.width = cfg->width;
  set_parts(p, cfg, false, workspace_dev);
  return hip_result(launch_gated_scan(p, cfg->dtype == PRSGD_BF16, false, reinterpret_cast<hipStream_t>(hip_stream)), "gated_scan");
}

int prsgd_gated_scan_backward(const prsgd_scan_config* cfg, const int32_t* starts_dev, const void* dh_dev, int64_t dh_row, const void* v_dev,
                              int64_t v_row, const void* gate_dev, int64_t gate_row, const void* h_dev, int64_t h_row,
                              const float* initial_dev, int64_t initial_row, const float* dlast_dev, int64_t dlast_row, void* dv_dev,
                              int64_t dv_row, void* dgate_dev, int64_t dgate_row, float* dinitial_dev, int64_t dinitial_row, void* workspace_dev,
                              void* hip_stream) {
  if (const char* e = scan_error(cfg, starts_dev, 3)) return bad(e);
  const ScanBuffer rows[] = {{dh_dev, dh_row, false, true}, {v_dev, v_row, false, true},   {gate_dev, gate_row, false, true},
                             {h_dev, h_row, false, true},   {dv_dev, dv_row, true, true}, {dgate_dev, dgate_row, true, true}};
  const ScanBuffer states[] = {{initial_dev, initial_row, false, false}, {dlast_dev, dlast_row, false, false}, {dinitial_dev, dinitial_row, true, false}};
  if (const char* e = scan_buffers_error(cfg, rows, 6, states, 3, workspace_dev)) return bad(e);
  if (dinitial_dev != nullptr && dinitial_dev == initial_dev) return bad("gated_scan: buffers overlap");
  if (dinitial_dev != nullptr && dinitial_dev == dlast_dev && dinitial_row != dlast_row) return bad("gated_scan: state in place with another distance");
  ScanArgs p{};
  p.starts = starts_dev;
  p.v = v_dev;
  p.v_row = v_row;
  p.gate = gate_dev;
  p.gate_row = gate_row;
  p.h_in = h_dev;
  p.h_in_row = h_row;
  p.dh = dh_dev;
  p.dh_row = dh_row;
  p.initial = initial_dev;
  p.initial_row = initial_row;
  p.dlast = dlast_dev;
  p.dlast_row = dlast_row;
  p.h = dv_dev;
  p.h_row = dv_row;
  p.dgate = dgate_dev;
  p.dgate_row = dgate_row;
  p.last = dinitial_dev;
  p.last_row = dinitial_row;
  p.sequences = cfg->sequences;
  p.clear = cfg->clear;
  p.rows = cfg->rows;
  p.width = cfg->width;
  set_parts(p, cfg, true, workspace_dev);
  return hip_result(launch_gated_scan(p, cfg->dtype == PRSGD_BF16, true, reinterpret_cast<hipStream_t>(hip_stream)), "gated_scan backward");
}

int prsgd_dropout(const prsgd_dropout_config* cfg, const int64_t* step_dev, const void* x_dev, int64_t x_row, const void* res_dev,
                  int64_t res_row, void* y_dev, int64_t y_row, void* hip_stream) {
  if (cfg == nullptr) return bad("dropout: config is null");
  if (!type_ok(cfg->dtype)) return bad("dropout: unknown dtype");
  if (cfg->layer < 0 || cfg->layer >= kDropLayers) return bad("dropout: layer out of range (0..32767)");
  if (cfg->rows < 0 || cfg->rows > kMaxRows) return bad("dropout: rows out of range (below 2^31)");
  if (!width_ok(cfg->width)) return bad("dropout: width out of range (1..32768)");
  if (!(cfg->p >= 0.0f) || !(floor((double)cfg->p * 65536.0 + 0.5) < 65536.0)) return bad("dropout: p out of range (0 up to 1 - 2^-17)");
  if (cfg->rows == 0) return PRSGD_OK;
  const int es = element_bytes(cfg->dtype);
  if (x_dev == nullptr || y_dev == nullptr) return bad("dropout: null buffer");
  if (misaligned(x_dev, es) || misaligned(res_dev, es) || misaligned(y_dev, es) || misaligned(step_dev, 8)) return bad("dropout: misaligned buffer");
  if (!rows_ok(cfg->rows, cfg->width, x_row, false) || (res_dev != nullptr && !rows_ok(cfg->rows, cfg->width, res_row, false)) ||
      !rows_ok(cfg->rows, cfg->width, y_row, true))
    return bad("dropout: distance between rows out of range");
  if ((y_dev == x_dev && y_row != x_row) || (y_dev == res_dev && y_row != res_row)) return bad("dropout: in place with another distance between rows");
  if ((const void*)step_dev == y_dev) return bad("dropout: buffers overlap");
  DropoutArgs p{};
  p.x = x_dev;
  p.x_row = x_row;
  p.res = res_dev;
  p.res_row = res_row;
  p.y = y_dev;
  p.y_row = y_row;
  p.step_at = step_dev;
  p.seed = cfg->seed;
  p.step = cfg->step;
  p.rows = cfg->rows;
  p.width = cfg->width;
  p.layer = (uint32_t)cfg->layer;
  p.dropped = (uint32_t)floor((double)cfg->p * 65536.0 + 0.5);
  return hip_result(launch_dropout(p, cfg->dtype == PRSGD_BF16, reinterpret_cast<hipStream_t>(hip_stream)), "dropout");
}

size_t prsgd_linear_cross_entropy_workspace_bytes(const prsgd_xent_config* cfg) { return xent_bytes(cfg, false); }
size_t prsgd_linear_cross_entropy_backward_workspace_bytes(const prsgd_xent_config* cfg) { return xent_bytes(cfg, true); }

int prsgd_linear_cross_entropy(const prsgd_xent_config* cfg, const void* h_dev, int64_t h_row, const void* w_dev, int64_t w_matrix,
                               int64_t w_row, const int32_t* labels_dev, float* loss_dev, float* lse_dev, void* workspace_dev,
                               void* hip_stream) {
  if (const char* e = xent_error(cfg)) return bad(e);
  if (cfg->rows_per_worker == 0) return PRSGD_OK;
  const int es = element_bytes(cfg->dtype);
  if (h_dev == nullptr || w_dev == nullptr || labels_dev == nullptr || loss_dev == nullptr || lse_dev == nullptr || workspace_dev == nullptr)
    return bad("linear_cross_entropy: null buffer");
  if (misaligned(h_dev, es) || misaligned(w_dev, es) || misaligned(labels_dev, 4) || misaligned(loss_dev, 4) || misaligned(lse_dev, 4) ||
      misaligned(workspace_dev, 256))
    return bad("linear_cross_entropy: misaligned buffer");
  if (!rows_ok(cfg->rows_per_worker * cfg->workers, cfg->width, h_row, false)) return bad("linear_cross_entropy: distance between rows out of range");
  if (!matrices_ok(cfg->workers, matrix_rows(cfg), matrix_cols(cfg), w_matrix, w_row, false))
    return bad("linear_cross_entropy: distance between matrices or their rows out of range");
  const void* ins[] = {h_dev, w_dev, labels_dev};
  for (const void* in : ins)
    if (in == loss_dev || in == lse_dev) return bad("linear_cross_entropy: buffers overlap");
  if (loss_dev == lse_dev) return bad("linear_cross_entropy: buffers overlap");
  XentArgs p = xent_args(cfg);
  p.h = h_dev;
  p.h_row = h_row;
  p.w = w_dev;
  p.w_gs = w_matrix;
  p.w_row = w_row;
  p.labels = labels_dev;
  p.loss = loss_dev;
  p.lse = lse_dev;
  return hip_result(launch_xent(p, plan_of(cfg, false), reinterpret_cast<char*>(workspace_dev), cfg->dtype == PRSGD_BF16,
                                reinterpret_cast<hipStream_t>(hip_stream)), "linear_cross_entropy");
}

int prsgd_linear_cross_entropy_backward(const prsgd_xent_config* cfg, const float* dloss_dev, const void* h_dev, int64_t h_row,
                                        const void* w_dev, int64_t w_matrix, int64_t w_row, const int32_t* labels_dev, const float* lse_dev,
                                        void* dh_dev, int64_t dh_row, void* dw_dev, int64_t dw_matrix, int64_t dw_row, void* workspace_dev,
                                        void* hip_stream) {
  if (const char* e = xent_error(cfg)) return bad(e);
  const int es = element_bytes(cfg->dtype);
  if (dw_dev == nullptr || misaligned(dw_dev, es)) return bad("linear_cross_entropy: null or misaligned buffer");
  if (!matrices_ok(cfg->workers, matrix_rows(cfg), matrix_cols(cfg), dw_matrix, dw_row, true))
    return bad("linear_cross_entropy: distance between matrices or their rows out of range");
  if (cfg->rows_per_worker > 0) {
    if (dloss_dev == nullptr || h_dev == nullptr || w_dev == nullptr || labels_dev == nullptr || lse_dev == nullptr || dh_dev == nullptr ||
        workspace_dev == nullptr)
      return bad("linear_cross_entropy: null buffer");
    if (misaligned(dloss_dev, 4) || misaligned(h_dev, es) || misaligned(w_dev, es) || misaligned(labels_dev, 4) || misaligned(lse_dev, 4) ||
        misaligned(dh_dev, es) || misaligned(workspace_dev, 256))
      return bad("linear_cross_entropy: misaligned buffer");
    const int64_t rows = cfg->rows_per_worker * cfg->workers;
    if (!rows_ok(rows, cfg->width, h_row, false) || !rows_ok(rows, cfg->width, dh_row, true)) return bad("linear_cross_entropy: distance between rows out of range");
    if (!matrices_ok(cfg->workers, matrix_rows(cfg), matrix_cols(cfg), w_matrix, w_row, false))
      return bad("linear_cross_entropy: distance between matrices or their rows out of range");
    const void* ins[] = {dloss_dev, h_dev, w_dev, labels_dev, lse_dev};
    for (const void* in : ins)
      if (in == dh_dev || in == dw_dev) return bad("linear_cross_entropy: buffers overlap");
    if (dh_dev == dw_dev) return bad("linear_cross_entropy: buffers overlap");
  }
  XentArgs p = xent_args(cfg);
  p.dloss = dloss_dev;
  p.h = h_dev;
  p.h_row = h_row;
  p.w = w_dev;
  p.w_gs = w_matrix;
  p.w_row = w_row;
  p.labels = labels_dev;
  p.lse_in = lse_dev;
  p.dh = dh_dev;
  p.dh_row = dh_row;
  p.dw = dw_dev;
  p.dw_gs = dw_matrix;
  p.dw_row = dw_row;
  return hip_result(launch_xent_backward(p, plan_of(cfg, true), reinterpret_cast<char*>(workspace_dev), cfg->dtype == PRSGD_BF16,
                                         reinterpret_cast<hipStream_t>(hip_stream)), "linear_cross_entropy backward");
}

}  // extern "C"
