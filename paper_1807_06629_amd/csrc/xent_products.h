// The products of the cross entropy and its gradients, with what each does with its tiles.
//   PX_STATS  z^T = W^T h^T    a tile of logits becomes the maximum, the sum of exponentials and the label's logit of each of its rows
//   PX_DZ     z = h W          ... becomes dz, in the rows' type
//   PX_DH     dh = dz W^T      summed over the pieces of the classes in fp32
//   PX_DW     dW = h^T dz
// (PX_STATS has the classes along the accumulators' rows, 16 of them a lane, so that most of a row's reduction stays in registers.)
#pragma once

#include <math.h>

#include <algorithm>
#include <atomic>
#include <type_traits>

#include "gemm_tile.h"
#include "orth_rows.h"
#include "prsgd_token_internal.h"

namespace prsgd {

// One matrix of every worker: element (i, c), c the contraction index, at p + g * gs + i * ld + c, or (transposed) + c * ld + i.
// padded: rows as they lie in memory go on with zeros up to a multiple of eight.
struct Operand { const void* p; int64_t gs, ld; bool padded; };
struct ProductArgs {
  Operand a, b;
  int M, N, K;                           // rows of A, rows of B, contraction
  int groups;
  int splits; float* parts;              // wished for: parts of the contraction, each to its own fp32 [groups][M][parts_row(N)] of `parts` (1: none)
  int tiles_m, tiles_n, split_steps;     // filled in by the launcher: tiles, and steps of the contraction in a part
  unsigned first;                        // ... and the launch's first workgroup of all
  // of the rows, `rows` in every worker
  const int32_t* labels;
  const float* lse; const float* dloss;
  int64_t rows;
  int class0, classes;                   // first class of the piece; of all
  float2* stats; float* picked;          // PX_STATS: [rows of all workers][tiles_m]
  int most_tiles;                        // ... of which there is room for that many
  float* loss_out; float* lse_out;       // PX_STATS of all classes in one tile: what comes of its statistics (nullptr: these alone)
  void* out; int64_t out_gs, out_ld;     // the others
  float* sums;                           // PX_DH over several pieces: [groups][M][N] fp32
  bool first_piece, last_piece;
  uint32_t* real;                        // rows with a label, 32 to a word, (rows + 63) / 64 * 2 words a worker: PX_DZ of the first piece writes them
};
enum ProductEpilogue { PX_STATS = 0, PX_DZ = 1, PX_DH = 2, PX_DW = 3 };

template <typename T> constexpr bool kIsBf16 = std::is_same_v<T, uint16_t>;
__host__ __device__ constexpr int64_t parts_row(int64_t n) { return (n + 7) / 8 * 8; }
__host__ __device__ constexpr int64_t real_words(int64_t rows) { return (rows + 63) / 64 * 2; }

// exp of what is at most about zero.  bf16: on the hardware's base 2, which leaves |x| 2^-24 of the result, at most 2^-24 of the largest term.
template <typename T> __device__ __forceinline__ float exp_of(float x) {
  if constexpr (kIsBf16<T>) return __builtin_amdgcn_exp2f(x * 1.44269504f);
  else return expf(x);
}

// (m, s) of the union of two sets of logits, s the sum of exp(z - m)
__device__ __forceinline__ void join_stats(float& m, float& s, float m2, float s2) {
  const float top = fmaxf(m, m2);
  // a set without logits, or of logits of -infinity alone, has no sum
  s = (s == 0.0f ? 0.0f : s * expf(m - top)) + (s2 == 0.0f ? 0.0f : s2 * expf(m2 - top));
  m = top;
}

// Rows of the accumulators: element e of a 32 x 32 block lies at row acc_row(e, lane), column lane % 32.
__device__ __forceinline__ int acc_row(int e, int lane) { return 8 * (e / 4) + 4 * (lane >> 5) + (e & 3); }

// Consecutive workgroups go to the XCDs in turn; each gets a contiguous range of the tiles, so that what neighbours share stays in its L2.
struct TilePosition { int g, ti, tj, split; };
__device__ __forceinline__ TilePosition tile_of_workgroup(const ProductArgs& p, unsigned block) {
  const int tiles = p.tiles_m * p.tiles_n, total = tiles * p.groups * p.splits, xcd = block & 7;
  const int idx = xcd * (total >> 3) + min(xcd, total & 7) + (int)(block >> 3), part = idx / tiles, in = idx - part * tiles, g = part % p.groups;
  // strips four tiles high, column by column
  constexpr int kHigh = 4;
  const int strip = in / (kHigh * p.tiles_n), first = strip * kHigh, high = min(kHigh, p.tiles_m - first), rest = in - first * p.tiles_n;
  return {g, first + rest % high, rest / high, part / p.groups};
}

constexpr int kStripPad = 8;             // floats: the four rows between a register's two halves lie 32 banks apart
template <int BM, int BN, int WM, int WN, int EPI> constexpr int epilogue_lds_bytes() {
  return EPI == PX_STATS ? (WM * (int)sizeof(float2) + (int)sizeof(float)) * BN : WM * WN * 32 * (BN / WN + kStripPad) * 4;
}

// The loss goes from the row's maximum, not from lse, which is rounded at the logits' size: of a label whose logit is the maximum it is log s itself.
__device__ __forceinline__ void write_loss(float* loss, float* lse_out, int64_t row, float m, float s, bool real, float picked) {
  const float log_s = logf(s);
  lse_out[row] = m + log_s;
  loss[row] = real ? (m - picked) + log_s : 0.0f;
}

// Eight columns of a row of dz, dh or dW, n of which exist.
template <typename T, int EPI> __device__ __forceinline__ void finish(const ProductArgs& p, int g, int r, int c, int n, float (&v)[8]) {
  if constexpr (EPI == PX_DZ) {
    const int64_t row = g * p.rows + r;
    const int label = p.labels[row];
    const bool real = (unsigned)label < (unsigned)p.classes;
    const float lse = p.lse[row], weight = p.dloss[row];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = real && e < n ? weight * (exp_of<T>(v[e] - lse) - (p.class0 + c + e == label ? 1.0f : 0.0f)) : 0.0f;
    // zeros behind the last class
    store8(reinterpret_cast<T*>(p.out) + g * p.out_gs + (int64_t)r * p.out_ld + c, 8, v);
    return;
  }
  if constexpr (EPI == PX_DH) {
    const bool real = (unsigned)p.labels[g * p.rows + r] < (unsigned)p.classes;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = real ? v[e] : 0.0f;
    if (p.sums != nullptr) {
      float* sum = p.sums + ((int64_t)g * p.M + r) * p.N + c;
      if (!p.first_piece) {
        float before[8];
        load8(sum, n, before);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += before[e];
      }
      if (!p.last_piece) {
        store8(sum, n, v);
        return;
      }
    }
  }
  store8(reinterpret_cast<T*>(p.out) + g * p.out_gs + (int64_t)r * p.out_ld + c, n, v);
}

// Workgroup-wide: the last reads of the operands' tiles in smem are over.  sums: this wavefront's accumulators are whole (of WK at a place one).
template <typename T, int EPI, int BM, int BN, int WM, int WN, int WK>
__device__ __forceinline__ void product_epilogue(const ProductArgs& p, const f32x16_t (&acc)[BM / WM / 32][BN / WN / 32], TilePosition at, int m0, int n0,
                                                 int wm, int wn, int lane, bool sums, unsigned char* smem) {
  constexpr int TM = BM / WM / 32, TN = BN / WN / 32;
  const int g = at.g;
  if constexpr (EPI == PX_STATS) {
    float2* shared = reinterpret_cast<float2*>(smem);        // [WM][BN], and the labels' logits
    float* shared_picked = reinterpret_cast<float*>(shared + WM * BN);
    const bool whole = p.loss_out != nullptr && p.tiles_m == 1;
#pragma unroll
    for (int j = 0; j < TN; ++j) {
      if (!sums) break;
      const int col = (wn * TN + j) * 32 + (lane & 31), row = n0 + col;
      const bool live = row < p.N;
      const int label = live ? p.labels[g * p.rows + row] : -1;
      float m = -INFINITY, s = 0.0f;
      bool odd = false;
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int c = m0 + (wm * TM + i) * 32 + acc_row(e, lane);
          if (c < p.M) {
            m = fmaxf(m, acc[i][j][e]);
            odd = odd || !(acc[i][j][e] <= INFINITY);          // fmaxf passes over what is no number
            if (p.class0 + c == label) {
              if (whole) shared_picked[col] = acc[i][j][e];
              else p.picked[g * p.rows + row] = acc[i][j][e];
            }
          }
        }
      const float top = m == -INFINITY ? 0.0f : m;
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int c = m0 + (wm * TM + i) * 32 + acc_row(e, lane);
          if (c < p.M) s += exp_of<T>(acc[i][j][e] - top);
        }
      if (odd) s = NAN;
      join_stats(m, s, __shfl_xor(m, 32), __shfl_xor(s, 32));
      if (lane < 32) shared[wm * BN + col] = make_float2(m, s);
    }
    __syncthreads();
    for (int col = threadIdx.x; col < BN; col += WM * WN * WK * kWave) {
      if (n0 + col >= p.N) continue;
      float2 v = shared[col];
#pragma unroll
      for (int w = 1; w < WM; ++w) {
        const float2 o = shared[w * BN + col];
        join_stats(v.x, v.y, o.x, o.y);
      }
      const int64_t row = g * p.rows + n0 + col;
      if (whole) write_loss(p.loss_out, p.lse_out, row, v.x, v.y, (unsigned)p.labels[row] < (unsigned)p.classes, shared_picked[col]);
      else p.stats[row * p.tiles_m + at.ti] = v;
    }
  } else {
    // a wavefront passes strips of 32 rows through LDS, from where a lane takes eight columns of a row at a time
    if (!sums) return;
    constexpr int W = BN / WN, P = W + kStripPad, VPR = W / 8, RPP = kWave / VPR, PASSES = 32 / RPP;
    float* strip = reinterpret_cast<float*>(smem) + (wm * WN + wn) * 32 * P;
    const int c = n0 + wn * W + lane % VPR * 8, n = p.N - c;
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      const int r0 = m0 + (wm * TM + i) * 32;
#pragma unroll
      for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) strip[acc_row(e, lane) * P + j * 32 + (lane & 31)] = acc[i][j][e];
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int q = 0; q < PASSES; ++q) {
        const int lr = q * RPP + lane / VPR, r = r0 + lr;
        const float* from = strip + lr * P + lane % VPR * 8;
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = from[e];
        const bool live = r < p.M;
        if (!live || n <= 0) continue;
        if (p.splits > 1) store8(p.parts + (((int64_t)at.split * p.groups + g) * p.M + r) * parts_row(p.N) + c, 8, v);
        else finish<T, EPI>(p, g, r, c, n, v);
      }
      __builtin_amdgcn_wave_barrier();
    }
    if constexpr (EPI == PX_DZ) {
      if (p.first_piece && n0 == 0 && wn == 0 && at.split == 0) {
        // rows of this wavefront: words of 32, of which behind the last row there may be one more, so that they are pairs
#pragma unroll
        for (int i = 0; i < TM; ++i) {
          const int r0 = m0 + (wm * TM + i) * 32, r = r0 + (lane & 31);
          const bool real = r < p.M && (unsigned)p.labels[g * p.rows + r] < (unsigned)p.classes;
          const uint64_t bits = __ballot(real);
          uint32_t* words = p.real + g * real_words(p.M) + r0 / 32;
          if (lane == 0 && r0 < p.M) words[0] = (uint32_t)bits;
          if (lane == 0 && r0 < p.M && r0 + 32 >= p.M && r0 / 32 % 2 == 0) words[1] = 0;
        }
      }
    }
  }
}

// Limit of a kernel's dynamic LDS, raised once on every device (twice is harmless).
template <auto KERNEL> hipError_t allow_lds(int bytes) {
  if (bytes <= 64 * 1024) return hipSuccess;
  static std::atomic<uint64_t> configured{0};
  int device = 0;
  if (const hipError_t e = hipGetDevice(&device); e != hipSuccess) return e;
  const uint64_t bit = device < 64 ? (uint64_t)1 << device : 0;
  if ((configured.load(std::memory_order_acquire) & bit) != 0) return hipSuccess;
  const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(KERNEL), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == hipSuccess) configured.fetch_or(bit, std::memory_order_release);
  return e;
}

// Tiles of B x B, and those of all parts of the contraction.
inline int64_t tiles_of(const ProductArgs& p, int64_t b) { return (p.M + b - 1) / b * ((p.N + b - 1) / b) * p.groups * p.splits; }
// How a launch of tiles of bm x bn, `depth` a step, cuts the product: its grid.  No part of the contraction is empty.
struct Cut { int tiles_m, splits; };
inline unsigned cut_product(ProductArgs& p, int bm, int bn, int depth, Cut* cut) {
  cut->tiles_m = p.tiles_m = (p.M + bm - 1) / bm;
  p.tiles_n = (p.N + bn - 1) / bn;
  const int steps = std::max((p.K + depth - 1) / depth, 1);
  p.split_steps = (steps + p.splits - 1) / p.splits;
  cut->splits = p.splits = (steps + p.split_steps - 1) / p.split_steps;
  return (unsigned)p.tiles_m * (unsigned)p.tiles_n * (unsigned)p.groups * (unsigned)p.splits;
}
// An axis of a grid holds fewer than 2^32 threads, and a launch of more is cut without an error: 2^22 workgroups a launch.
template <typename F> hipError_t in_turn(ProductArgs& p, unsigned grid, const F& launch) {
  constexpr unsigned kMost = 1u << 22;
  for (p.first = 0; p.first < grid; p.first += kMost) {
    launch(std::min(grid - p.first, kMost));
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  }
  return hipSuccess;
}

// transposed: (A, B) as (element (i, c) at c * ld + i).  Operands of any alignment and size (kernels_xent_any.hip) ...
// cut: how the product was cut
hipError_t launch_product_any(const ProductArgs& p, int epi, bool a_transposed, bool b_transposed, bool bf16, Cut* cut, hipStream_t s);
// Rows of the tiles that PX_STATS of this size gets, by its sizes and by which operands are padded alone.
int stats_rows_any(const ProductArgs& p, bool a_transposed, bool bf16);
int stats_rows_bf16(const ProductArgs& p);
// The gradients' three products one after another, by a workgroup a worker, where that takes less than their launches.
bool small_gradients(int64_t rows, int width, int classes, bool bf16);
hipError_t launch_small_gradients(ProductArgs dz, ProductArgs dh, ProductArgs dw, bool classes_first, bool bf16, hipStream_t s);
// dh and dW in one launch, where they are small (splits is set as wished in both).
bool pair_gradients(const ProductArgs& dh, const ProductArgs& dw, int classes, int width, bool bf16);
hipError_t launch_pair_any(const ProductArgs& dh, const ProductArgs& dw, bool classes_first, bool bf16, hipStream_t s);
hipError_t launch_pair_bf16(const ProductArgs& dh, const ProductArgs& dw, bool classes_first, hipStream_t s);
// ... and bf16 operands whose rows start at 16 bytes and are as long in whole (kernels_xent_bf16.hip).
bool product_aligned(const ProductArgs& p, bool a_transposed, bool b_transposed);
hipError_t launch_product_bf16(const ProductArgs& p, int epi, bool a_transposed, bool b_transposed, Cut* cut, hipStream_t s);

}  // namespace prsgd
