// Softmax cross entropy of the workers' rows through their last matrices, in pieces of the classes; the logits are never stored whole.
//   z = W^T h,  lse = log sum exp z,  loss = lse - z[label]
//   dz = dloss (exp(z - lse) - onehot(label)),  dh = W dz,  dW = h dz^T
// Forward: a tile of logits is reduced to the maximum, the sum of exponentials and the label's logit of each of its rows; a second launch joins the tiles'.
// Backward, piece by piece: a tile of logits becomes dz (in the rows' type, which is what the products take: for bf16 8 bits, an error that the
// sums over rows or classes average to about that of the result's own rounding), two products follow.  Rows without a label have dz = 0, take no part in dW, also where they are
// no numbers, and get zeros.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "gemm_tile.h"
#include "orth_rows.h"
#include "prsgd_token_internal.h"

namespace prsgd {

namespace {

// One matrix of every worker: element (i, c), c the contraction index, at p + g * gs + i * ld + c, or (transposed) + c * ld + i.
struct Operand { const void* p; int64_t gs, ld; };
struct ProductArgs {
  Operand a, b;
  int M, N, K;                           // rows of A, rows of B, contraction
  int tiles_m, tiles_n, groups;          // filled in by the launcher
  // rows of the set in every worker, of which the first is this worker's: labels, lse, dloss, stats
  const int32_t* labels;
  const float* lse; const float* dloss;
  int64_t rows;
  int class0, classes;                   // first class of the piece; of all
  float2* stats; int stat_tiles; float* picked;      // PX_STATS
  void* out; int64_t out_gs, out_ld;     // the others
  float* sums;                           // PX_DH over several pieces: [groups][M][N] fp32
  bool first_piece, last_piece;
};
enum ProductEpilogue {
  PX_STATS = 0,   // M classes, N rows
  PX_DZ = 1,      // M classes, N rows: out [row][class of the piece]
  PX_DH = 2,      // M rows, N columns
  PX_DW = 3,      // contraction over the rows; those without a label take no part
};

template <typename T> constexpr bool kIsBf16 = std::is_same_v<T, uint16_t>;
template <typename T> using Tag = std::conditional_t<kIsBf16<T>, TBF16, TF32>;

// n elements from p on (0 .. 16 bytes' worth)
template <typename T> __device__ __forceinline__ u32x4_t load16(const T* p, int n) {
  constexpr int V = 16 / (int)sizeof(T);
  u32x4_t v = {0, 0, 0, 0};
  if (n >= V) return reinterpret_cast<const Packed16<(int)sizeof(T)>*>(p)->v;
#pragma unroll
  for (int e = 0; e < V; ++e)
    if (e < n) {
      if constexpr (sizeof(T) == 4) v[e] = __float_as_uint(p[e]);
      else v[e / 2] |= (uint32_t)p[e] << (16 * (e & 1));
    }
  return v;
}

// ---- products of operands of any alignment and size --------------------------------------------
// Tiles pass through registers into LDS, [row][contraction] either way: 32 deep, rows padded by 16 bytes.  Fragments are those of the grouped products.
constexpr int kDepth = 32;
template <typename T, int ROWS, bool TRANS> struct Stage {
  static constexpr int ES = (int)sizeof(T), V = 16 / ES, LD = kDepth * ES + 16, BYTES = ROWS * LD;
  // transposed: a thread has a block of 4 / ES contraction elements ... of 16 bytes of rows
  static constexpr int BK = TRANS ? 4 / ES * (ES == 4 ? 4 : 1) : 1;            // fp32 4 x 4, bf16 2 x 8
  static constexpr int UNITS = TRANS ? kDepth / BK * (ROWS / V) : ROWS * kDepth / V;
  static constexpr int NPT = (UNITS + kThreads - 1) / kThreads;
  u32x4_t reg[NPT][BK];
  // rows, depth: what is left of the operand from the tile's first element on; labels: of the contraction index (PX_DW)
  __device__ __forceinline__ void load(const T* base, int64_t ld, int rows, int depth, const int32_t* labels, int classes) {
#pragma unroll
    for (int q = 0; q < NPT; ++q) {
      const int u = q * kThreads + (int)threadIdx.x;
#pragma unroll
      for (int k = 0; k < BK; ++k) reg[q][k] = (u32x4_t){0, 0, 0, 0};
      if (UNITS % kThreads != 0 && u >= UNITS) continue;
      if constexpr (TRANS) {
        const int c = u % (kDepth / BK) * BK, r = u / (kDepth / BK) * V;
#pragma unroll
        for (int k = 0; k < BK; ++k)
          if (c + k < depth && r < rows && (labels == nullptr || (unsigned)labels[c + k] < (unsigned)classes))
            reg[q][k] = load16(base + (int64_t)(c + k) * ld + r, rows - r);
      } else {
        const int r = u / (kDepth / V), c = u % (kDepth / V) * V;
        if (r < rows && c < depth) reg[q][0] = load16(base + (int64_t)r * ld + c, depth - c);
      }
    }
  }
  __device__ __forceinline__ void store(unsigned char* tile) const {
#pragma unroll
    for (int q = 0; q < NPT; ++q) {
      const int u = q * kThreads + (int)threadIdx.x;
      if (UNITS % kThreads != 0 && u >= UNITS) continue;
      if constexpr (TRANS) {
        const int c = u % (kDepth / BK) * BK, r = u / (kDepth / BK) * V;
#pragma unroll
        for (int e = 0; e < V; ++e) {
          unsigned char* to = tile + (r + e) * LD + c * ES;
          if constexpr (ES == 4) {
            *reinterpret_cast<u32x4_t*>(to) = (u32x4_t){reg[q][0][e], reg[q][1][e], reg[q][2][e], reg[q][3][e]};
          } else {
            const uint32_t lo = reg[q][0][e / 2] >> (16 * (e & 1)) & 0xFFFFu, hi = reg[q][1][e / 2] >> (16 * (e & 1)) << 16;
            *reinterpret_cast<uint32_t*>(to) = lo | hi;
          }
        }
      } else {
        const int r = u / (kDepth / V), c = u % (kDepth / V) * V;
        *reinterpret_cast<u32x4_t*>(tile + r * LD + c * ES) = reg[q][0];
      }
    }
  }
  __device__ static __forceinline__ Frag<Tag<T>> frag(const unsigned char* tile, int block, int kk, int lane) {
    Frag<Tag<T>> f;
    const u32x4_t v = *reinterpret_cast<const u32x4_t*>(tile + (block * 32 + (lane & 31)) * LD + (2 * kk + (lane >> 5)) * 16);
    f.v = __builtin_bit_cast(decltype(f.v), v);
    return f;
  }
};

// ---- epilogues -----------------------------------------------------------------------------------

// (m, s) of the union of two sets of logits
__device__ __forceinline__ void join_stats(float& m, float& s, float m2, float s2) {
  const float top = fmaxf(m, m2);
  // a set without logits, or of logits of -infinity alone, has no sum
  s = (s == 0.0f ? 0.0f : s * expf(m - top)) + (s2 == 0.0f ? 0.0f : s2 * expf(m2 - top));
  m = top;
}

// Rows of the accumulators: element e of a 32 x 32 block lies at row acc_row(e, lane), column lane % 32.
__device__ __forceinline__ int acc_row(int e, int lane) { return 8 * (e / 4) + 4 * (lane >> 5) + (e & 3); }

template <typename T, int EPI, int TM, int TN, int WM, int WN>
__device__ __forceinline__ void product_epilogue(const ProductArgs& p, const f32x16_t (&acc)[TM][TN], int g, int m0, int n0, int ti, int wm, int wn, int lane,
                                                 unsigned char* smem) {
  if constexpr (EPI == PX_STATS) {
    // a lane has classes of one row per block column
    float2* shared = reinterpret_cast<float2*>(smem);        // [WM][WN * TN * 32]
#pragma unroll
    for (int j = 0; j < TN; ++j) {
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
            if (p.class0 + c == label) p.picked[g * p.rows + row] = acc[i][j][e];
          }
        }
      const float top = m == -INFINITY ? 0.0f : m;
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int c = m0 + (wm * TM + i) * 32 + acc_row(e, lane);
          if (c < p.M) s += expf(acc[i][j][e] - top);
        }
      if (odd) s = NAN;
      join_stats(m, s, __shfl_xor(m, 32), __shfl_xor(s, 32));
      if (lane < 32) shared[wm * (WN * TN * 32) + col] = make_float2(m, s);
    }
    __syncthreads();
    for (int col = threadIdx.x; col < WN * TN * 32; col += kThreads) {
      if (n0 + col >= p.N) continue;
      float2 v = shared[col];
#pragma unroll
      for (int w = 1; w < WM; ++w) {
        const float2 o = shared[w * (WN * TN * 32) + col];
        join_stats(v.x, v.y, o.x, o.y);
      }
      p.stats[(g * p.rows + n0 + col) * p.stat_tiles + ti] = v;
    }
  } else if constexpr (EPI == PX_DZ) {
#pragma unroll
    for (int j = 0; j < TN; ++j) {
      const int row = n0 + (wn * TN + j) * 32 + (lane & 31);
      if (row >= p.N) continue;
      const int64_t r = g * p.rows + row;
      const int label = p.labels[r];
      const bool real = (unsigned)label < (unsigned)p.classes;
      const float lse = p.lse[r], weight = p.dloss[r];
      T* out = reinterpret_cast<T*>(p.out) + g * p.out_gs + (int64_t)row * p.out_ld;
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int c = m0 + (wm * TM + i) * 32 + acc_row(4 * q, lane);
          if (c >= p.out_ld) continue;                     // a whole tile of classes is stored, zeros behind the last one
          float v[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float z = acc[i][j][4 * q + e];
            v[e] = real && c + e < p.M ? weight * (expf(z - lse) - (p.class0 + c + e == label ? 1.0f : 0.0f)) : 0.0f;
          }
          if constexpr (kIsBf16<T>) *reinterpret_cast<uint2*>(out + c) = make_uint2(f32x2_to_bf16x2_rne(v[0], v[1]), f32x2_to_bf16x2_rne(v[2], v[3]));
          else *reinterpret_cast<float4*>(out + c) = make_float4(v[0], v[1], v[2], v[3]);
        }
    }
  } else {
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int r = m0 + (wm * TM + i) * 32 + acc_row(e, lane);
        if (r >= p.M) continue;
        bool real = true;
        if constexpr (EPI == PX_DH) real = (unsigned)p.labels[g * p.rows + r] < (unsigned)p.classes;
#pragma unroll
        for (int j = 0; j < TN; ++j) {
          const int c = n0 + (wn * TN + j) * 32 + (lane & 31);
          if (c >= p.N) continue;
          float v = real ? acc[i][j][e] : 0.0f;
          if constexpr (EPI == PX_DH) {
            if (p.sums != nullptr) {
              float* at = p.sums + ((int64_t)g * p.M + r) * p.N + c;
              if (!p.first_piece) v += *at;
              if (!p.last_piece) {
                *at = v;
                continue;
              }
            }
          }
          T* out = reinterpret_cast<T*>(p.out) + g * p.out_gs + (int64_t)r * p.out_ld + c;
          if constexpr (kIsBf16<T>) *out = (uint16_t)f32x2_to_bf16x2_rne(v, 0.0f);
          else *out = v;
        }
      }
  }
}

// ---- the kernel ----------------------------------------------------------------------------------

constexpr int product_stage_bytes(int bm, int bn, int es) { return (bm + bn) * (kDepth * es + 16); }

template <typename T, int BM, int BN, bool TA, bool TB, int EPI> __global__ void __launch_bounds__(kThreads) product_kernel(ProductArgs p) {
  constexpr int WM = 2, WN = 2, TM = BM / WM / 32, TN = BN / WN / 32, KK = kDepth * (int)sizeof(T) / 32;
  using A = Stage<T, BM, TA>;
  using B = Stage<T, BN, TB>;
  constexpr int STAGE = product_stage_bytes(BM, BN, (int)sizeof(T));
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave / WN, wn = wave % WN;
  // consecutive workgroups go to the XCDs in turn; each gets a contiguous range of the tiles
  const int tiles = p.tiles_m * p.tiles_n, total = tiles * p.groups, xcd = blockIdx.x & 7;
  const int idx = xcd * (total >> 3) + min(xcd, total & 7) + (int)(blockIdx.x >> 3), g = idx / tiles, in = idx - g * tiles;
  const int ti = in / p.tiles_n, tj = in - ti * p.tiles_n, m0 = ti * BM, n0 = tj * BN;
  const T* a = reinterpret_cast<const T*>(p.a.p) + g * p.a.gs + (int64_t)m0 * (TA ? 1 : p.a.ld);
  const T* b = reinterpret_cast<const T*>(p.b.p) + g * p.b.gs + (int64_t)n0 * (TB ? 1 : p.b.ld);
  const int64_t step_a = (int64_t)kDepth * (TA ? p.a.ld : 1), step_b = (int64_t)kDepth * (TB ? p.b.ld : 1);
  const int32_t* labels = EPI == PX_DW ? p.labels + g * p.rows : nullptr;
  f32x16_t acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;
  A ra;
  B rb;
  const int n_k = (p.K + kDepth - 1) / kDepth;
  auto load = [&](int t) __attribute__((always_inline)) {
    const int32_t* of = EPI == PX_DW ? labels + t * kDepth : nullptr;
    ra.load(a + t * step_a, p.a.ld, p.M - m0, p.K - t * kDepth, of, p.classes);
    rb.load(b + t * step_b, p.b.ld, p.N - n0, p.K - t * kDepth, of, p.classes);
  };
  load(0);
  ra.store(smem);
  rb.store(smem + A::BYTES);
  __syncthreads();
  for (int t = 0; t < n_k; ++t) {
    const unsigned char* here = smem + (t & 1) * STAGE;
    if (t + 1 < n_k) load(t + 1);
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
      Frag<Tag<T>> fa[TM], fb[TN];
#pragma unroll
      for (int i = 0; i < TM; ++i) fa[i] = A::frag(here, wm * TM + i, kk, lane);
#pragma unroll
      for (int j = 0; j < TN; ++j) fb[j] = B::frag(here + A::BYTES, wn * TN + j, kk, lane);
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = mma(fa[i], fb[j], acc[i][j]);
    }
    if (t + 1 < n_k) {
      unsigned char* next = smem + ((t + 1) & 1) * STAGE;
      ra.store(next);
      rb.store(next + A::BYTES);
    }
    __syncthreads();
  }
  product_epilogue<T, EPI, TM, TN, WM, WN>(p, acc, g, m0, n0, ti, wm, wn, lane, smem);
}

template <typename T, int BM, int BN, bool TA, bool TB, int EPI> hipError_t launch_tile(ProductArgs p, hipStream_t s) {
  constexpr int kLds = 2 * product_stage_bytes(BM, BN, (int)sizeof(T));
  static_assert(kLds <= 160 * 1024 && kLds >= 2 * BN * (int)sizeof(float2), "LDS");
  auto kernel = product_kernel<T, BM, BN, TA, TB, EPI>;
  if constexpr (kLds > 64 * 1024) {
    static std::atomic<bool> configured{false};            // setting the limit twice is harmless
    if (!configured.load(std::memory_order_acquire)) {
      hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, kLds);
      if (e != hipSuccess) return e;
      configured.store(true, std::memory_order_release);
    }
  }
  p.tiles_m = (p.M + BM - 1) / BM;
  p.tiles_n = (p.N + BN - 1) / BN;
  if (p.tiles_m == 0 || p.tiles_n == 0) return hipSuccess;   // no rows: what remains is the zeros of dW
  hipLaunchKernelGGL(kernel, dim3((unsigned)p.tiles_m * (unsigned)p.tiles_n * (unsigned)p.groups), dim3(kThreads), kLds, s, p);
  return hipGetLastError();
}
template <typename T, bool TA, bool TB, int EPI> hipError_t launch_product(const ProductArgs& p, hipStream_t s) {
  return launch_tile<T, 128, 128, TA, TB, EPI>(p, s);
}

// Loss and lse of every row from its tiles' statistics: a wavefront a row.
__global__ void __launch_bounds__(kThreads) join_tiles_kernel(XentArgs p, const float2* stats, const float* picked, int tiles) {
  const int lane = threadIdx.x % kWave;
  const int64_t rows = p.rows * p.workers;
  for (int64_t r = (int64_t)blockIdx.x * (kThreads / kWave) + threadIdx.x / kWave; r < rows; r += (int64_t)gridDim.x * (kThreads / kWave)) {
    float m = -INFINITY, s = 0.0f;
    for (int t = lane; t < tiles; t += kWave) {
      const float2 v = stats[r * tiles + t];
      join_stats(m, s, v.x, v.y);
    }
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) join_stats(m, s, __shfl_xor(m, d), __shfl_xor(s, d));
    if (lane == 0) {
      const float lse = m + logf(s);
      const bool real = (unsigned)p.labels[r] < (unsigned)p.classes;
      p.lse[r] = lse;
      p.loss[r] = real ? lse - picked[r] : 0.0f;
    }
  }
}

constexpr int kClassTile = 128;
constexpr size_t kPieceBytes = (size_t)128 << 20;          // of dz

template <typename T> hipError_t forward(const XentArgs& x, const XentPlan& plan, char* ws, hipStream_t s) {
  ProductArgs p{};
  p.a = {x.w, x.w_gs, x.w_row};
  p.b = {x.h, x.rows * x.h_row, x.h_row};
  p.M = x.classes;
  p.N = (int)x.rows;
  p.K = x.width;
  p.groups = x.workers;
  p.labels = x.labels;
  p.rows = x.rows;
  p.classes = x.classes;
  p.stats = reinterpret_cast<float2*>(ws + plan.stats);
  p.stat_tiles = plan.tiles;
  p.picked = reinterpret_cast<float*>(ws + plan.picked);
  hipError_t e = x.classes_first ? launch_product<T, false, false, PX_STATS>(p, s) : launch_product<T, true, false, PX_STATS>(p, s);
  if (e != hipSuccess) return e;
  const unsigned grid = (unsigned)std::min<int64_t>((x.rows * x.workers + 3) / 4, 256 * 64);
  hipLaunchKernelGGL(join_tiles_kernel, dim3(grid), dim3(kThreads), 0, s, x, (const float2*)p.stats, (const float*)p.picked, plan.tiles);
  return hipGetLastError();
}

template <typename T> hipError_t backward(const XentArgs& x, const XentPlan& plan, char* ws, hipStream_t s) {
  const T* w = reinterpret_cast<const T*>(x.w);
  T* dw = reinterpret_cast<T*>(x.dw);
  for (int k = 0; k < plan.pieces; ++k) {
    const int first = k * plan.piece, n = std::min(plan.piece, x.classes - first);
    const int64_t w_at = x.classes_first ? first * x.w_row : first, dw_at = x.classes_first ? first * x.dw_row : first;
    const Operand rows{x.h, x.rows * x.h_row, x.h_row}, matrix{w + w_at, x.w_gs, x.w_row};
    ProductArgs p{};
    p.groups = x.workers;
    p.labels = x.labels;
    p.lse = x.lse_in;
    p.dloss = x.dloss;
    p.rows = x.rows;
    p.class0 = first;
    p.classes = x.classes;
    p.a = matrix;
    p.b = rows;
    p.M = n;
    p.N = (int)x.rows;
    p.K = x.width;
    p.out = ws + plan.dz;
    p.out_ld = plan.piece;
    p.out_gs = x.rows * plan.piece;
    const Operand dz{p.out, p.out_gs, p.out_ld};
    hipError_t e = x.classes_first ? launch_product<T, false, false, PX_DZ>(p, s) : launch_product<T, true, false, PX_DZ>(p, s);
    if (e != hipSuccess) return e;
    p.a = dz;
    p.b = matrix;
    p.M = (int)x.rows;
    p.N = x.width;
    p.K = n;
    p.out = x.dh;
    p.out_ld = x.dh_row;
    p.out_gs = x.rows * x.dh_row;
    p.sums = plan.pieces > 1 ? reinterpret_cast<float*>(ws + plan.sums) : nullptr;
    p.first_piece = k == 0;
    p.last_piece = k + 1 == plan.pieces;
    e = x.classes_first ? launch_product<T, false, true, PX_DH>(p, s) : launch_product<T, false, false, PX_DH>(p, s);
    if (e != hipSuccess) return e;
    p.a = x.classes_first ? dz : rows;
    p.b = x.classes_first ? rows : dz;
    p.M = x.classes_first ? n : x.width;
    p.N = x.classes_first ? x.width : n;
    p.K = (int)x.rows;
    p.out = dw + dw_at;
    p.out_ld = x.dw_row;
    p.out_gs = x.dw_gs;
    if ((e = launch_product<T, true, true, PX_DW>(p, s)) != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace

XentPlan xent_plan(int workers, int64_t rows, int width, int classes, bool bf16, bool backward) {
  XentPlan e{};
  const size_t n = (size_t)workers * (size_t)rows;
  size_t at = 0;
  auto take = [&](size_t bytes) { const size_t v = at; at += (bytes + 255) / 256 * 256; return v; };
  if (!backward) {
    e.tiles = (classes + kClassTile - 1) / kClassTile;
    e.stats = take(n * e.tiles * sizeof(float2));
    e.picked = take(n * sizeof(float));
  } else {
    const int whole = (classes + 255) / 256;               // in 256 classes
    const int64_t fit = (int64_t)(kPieceBytes / (std::max<size_t>(n, 1) * 256 * (bf16 ? 2 : 4)));
    const int pieces = (int)std::min<int64_t>(whole, (whole + std::max<int64_t>(fit, 1) - 1) / std::max<int64_t>(fit, 1));
    e.piece = (whole + pieces - 1) / pieces * 256;
    e.pieces = (classes + e.piece - 1) / e.piece;
    e.dz = take(n * e.piece * (bf16 ? 2 : 4));
    e.sums = e.pieces > 1 ? take(n * width * sizeof(float)) : 0;
  }
  e.total = at;
  return e;
}

hipError_t launch_xent(const XentArgs& p, const XentPlan& plan, char* ws, bool bf16, hipStream_t s) {
  return bf16 ? forward<uint16_t>(p, plan, ws, s) : forward<float>(p, plan, ws, s);
}
hipError_t launch_xent_backward(const XentArgs& p, const XentPlan& plan, char* ws, bool bf16, hipStream_t s) {
  return bf16 ? backward<uint16_t>(p, plan, ws, s) : backward<float>(p, plan, ws, s);
}

}  // namespace prsgd
