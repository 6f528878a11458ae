// Internal declarations of the operators of replicas of a model over tokens (prsgd_ops.h, second half).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "prsgd_ops.h"

namespace prsgd {

constexpr int kMaxTokenWidth = 32768;    // embeddings, scans, dropout and the loss
constexpr int kMaxClasses = 1 << 20;     // of a table or a last matrix

// Lanes that share a row, eight elements each: their logarithm, at most that of a workgroup of 256.
constexpr int lanes_for_row(int width) {
  int log2 = 0;
  while (log2 < 8 && (8 << log2) < width) ++log2;
  return log2;
}

// ---- dropout -----------------------------------------------------------------------------------

constexpr int kDropLayers = 1 << 15;
struct DropoutArgs {
  const void* x; int64_t x_row;
  const void* res; int64_t res_row;      // nullptr: none
  void* y; int64_t y_row;
  const int64_t* step_at;                // nullptr: `step`
  uint64_t seed, step;
  int64_t rows;
  int width;
  uint32_t layer, dropped;               // of 65536 equally likely values, how many drop an element
};
hipError_t launch_dropout(const DropoutArgs& p, bool bf16, hipStream_t s);

// ---- embedding ---------------------------------------------------------------------------------

constexpr int kSortTile = 2048;          // tokens that a workgroup sorts
struct EmbeddingArgs {
  const int32_t* tokens;                 // [workers][rows]
  const void* table; int64_t table_gs, table_row;    // backward: not read
  void* y; int64_t y_row;                // backward: dy, read
  void* dtable; int64_t dtable_gs, dtable_row;
  int workers;
  int64_t rows;                          // of a worker
  int classes, width;
  float scale;
};
hipError_t launch_embedding(const EmbeddingArgs& p, bool bf16, hipStream_t s);
// Sorted order of every worker's tokens, runs of equal ones, and partial sums of runs that pass a chunk's end.
struct EmbeddingPlan {
  int tiles;                             // of kSortTile tokens, per worker
  int chunk, chunks;                     // sorted tokens whose sums some lanes take; per worker
  size_t keys, order, sorted, parts, total;    // byte offsets
};
EmbeddingPlan embedding_plan(int workers, int64_t rows, int width);
hipError_t launch_embedding_backward(const EmbeddingArgs& p, const EmbeddingPlan& plan, char* ws, bool bf16, hipStream_t s);

// ---- gated scan --------------------------------------------------------------------------------

struct ScanArgs {
  const int32_t* starts;                 // nullptr: rows are dealt evenly
  const void* v; int64_t v_row;
  const void* gate; int64_t gate_row;
  const void* h_in; int64_t h_in_row;    // backward: what the forward pass wrote
  const void* dh; int64_t dh_row;        // backward
  const float* initial; int64_t initial_row;         // nullptr: zeros
  const float* dlast; int64_t dlast_row;             // backward; nullptr: zeros
  void* h; int64_t h_row;                // backward: dv
  void* dgate; int64_t dgate_row;        // backward
  float* last; int64_t last_row;         // nullptr: not wanted; backward: dinitial
  int sequences;
  int64_t rows;
  int width;
  int parts; float2* joint; float* aside;
  int clear;                             // 1: h, 2: dgate hold zeros in rows before the first sequence and behind the last
};
// Parts that the rows are cut into (1: they are not); their compositions lie in `joint` [parts][width], the sequences' states at their start in `aside`
// [sequences][width].
int scan_parts(int sequences, int64_t rows, int width, int element_bytes, bool packed, bool backward);
hipError_t launch_gated_scan(const ScanArgs& p, bool bf16, bool backward, hipStream_t s);

// ---- cross entropy of a last layer ---------------------------------------------------------------

struct XentArgs {
  const void* h; int64_t h_row;
  const void* w; int64_t w_gs, w_row;
  const int32_t* labels;
  const float* dloss; const float* lse_in;           // backward
  float* loss; float* lse;               // forward
  void* dh; int64_t dh_row;
  void* dw; int64_t dw_gs, dw_row;
  int workers;
  int64_t rows;                          // of a worker
  int width, classes;
  bool classes_first;
};
struct XentPlan {
  int piece, pieces;                     // classes of a piece
  int tiles;                             // forward: of a piece, at most
  bool align_h, align_w;                 // h, a piece of W: copied, each row to a multiple of 16 bytes
  size_t stats, picked, dz, sums, parts, real, h, w, total;         // byte offsets
};
XentPlan xent_plan(int workers, int64_t rows, int width, int classes, bool classes_first, bool bf16, bool backward);
hipError_t launch_xent(const XentArgs& p, const XentPlan& plan, char* ws, bool bf16, hipStream_t s);
hipError_t launch_xent_backward(const XentArgs& p, const XentPlan& plan, char* ws, bool bf16, hipStream_t s);

}  // namespace prsgd
