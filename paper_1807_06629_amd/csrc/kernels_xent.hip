// Softmax cross entropy of the workers' rows through their last matrices, in pieces of the classes; the logits are never stored whole.
//   z = W^T h,  lse = log sum exp z,  loss = lse - z[label]
//   dz = dloss (exp(z - lse) - onehot(label)),  dh = W dz,  dW = h dz^T
// Forward: a tile of logits is reduced to the maximum, the sum of exponentials and the label's logit of each of its rows; a second launch joins the tiles'.
// Backward, piece by piece: a tile of logits becomes dz (in the rows' type, which is what the products take: for bf16 8 bits, an error that the
// sums over rows or classes average to about that of the result's own rounding), two products follow.  Rows without a label have dz = 0, take no part in dW, also where they are
// no numbers, and get zeros.
// Bound by the matrix cores from about a hundred rows a worker on, by W's passage through HBM below (one row over 4096 x 65536 bf16: 108 us, 5.0 TB/s), by launches where both are
// small: the gradients are three products, of 4 to 8 us each at least.
#include <algorithm>

#include "row_pieces.h"
#include "xent_products.h"

namespace prsgd {

namespace {

// Parts that a contraction is cut into where its product has few tiles: 512 tiles of 64 x 64 in all, a part at least eight steps of 64.  The parts' addition takes
// 4 us, and half of a contraction of 2048 not much more.
int splits_of(int64_t m, int64_t n, int64_t k, int groups) {
  const int64_t tiles = (m + 63) / 64 * ((n + 63) / 64) * groups;
  return tiles == 0 || k < 2048 ? 1 : (int)std::max<int64_t>(std::min<int64_t>(512 / tiles, k / 512), 1);
}
// Of the logits' gradients: 256 tiles of 128 x 128 in all (smaller ones wait for L2), a part at least 512 deep.  A bf16 step takes a third of an fp32 one's time, so that the parts'
// addition is worth it from longer contractions on only, and longer yet where whole tiles nearly fill the card.  Gradients in parts and whole: 3 workers' 31 rows x 2704 x 938 fp32 48 and
// 63 us, 33 x 12 x 3010 x 20 31 and 51 us, 8 x 128 x 1024 x 1000 91 and 92 us; bf16 of the first 32 and 37 us, 4 x 64 x 2048 x 512 21.1 and 22.3 us, of 1024 15.2 and 14.5 us,
// 8 x 128 x 1000 classes by widths of 1024, 2048, 4096 and 8192 30.1, 42.2, 60.1, 102 and 24.2, 36.2, 57.5, 108 us (4096 with inputs out of the caches 72 and 74), 12 x 128 x 4096 x 1000 82 and 89 us.
int splits_of_logits(int64_t m, int64_t n, int64_t k, int groups, bool bf16) {
  const int64_t tiles = (m + 127) / 128 * ((n + 127) / 128) * groups, least = !bf16 ? 1024 : tiles < 64 ? 2048 : 4096;
  return tiles == 0 || k < least ? 1 : (int)std::max<int64_t>(std::min<int64_t>(256 / tiles, k / 512), 1);
}
size_t parts_bytes(int64_t m, int64_t n, int splits, int groups) {
  return splits > 1 ? (size_t)splits * groups * std::max(m * parts_row(n), n * parts_row(m)) * sizeof(float) : 0;
}

// dz, dh or dW of the parts: a lane eight columns.
template <typename T, int EPI> __global__ void __launch_bounds__(kThreads) join_parts_kernel(ProductArgs p) {
  const int64_t per_row = (p.N + 7) / 8, part = parts_row(p.N) * p.M * p.groups, total = per_row * p.M * p.groups;
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < total; i += (int64_t)gridDim.x * kThreads) {
    const int64_t row = i / per_row, g = row / p.M;
    const int r = (int)(row - g * p.M), c = (int)(i - row * per_row) * 8, n = p.N - c;
    const float* from = p.parts + row * parts_row(p.N) + c;
    float v[8];
    load8(from, 8, v);
#pragma unroll 4
    for (int q = 1; q < p.splits; ++q) {
      float more[8];
      load8(from + q * part, 8, more);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += more[e];
    }
    finish<T, EPI>(p, (int)g, r, c, n, v);
  }
}

// A product by the kernel that takes its operands.
hipError_t launch_product(const ProductArgs& p, int epi, bool a_transposed, bool b_transposed, bool bf16, Cut* cut, hipStream_t s) {
  *cut = {0, 1};
  if (p.M == 0 || p.N == 0) return hipSuccess;               // no rows: what remains is the zeros of dW
  if (bf16 && product_aligned(p, a_transposed, b_transposed)) return launch_product_bf16(p, epi, a_transposed, b_transposed, cut, s);
  return launch_product_any(p, epi, a_transposed, b_transposed, bf16, cut, s);
}
template <int EPI> hipError_t launch_gradient(ProductArgs p, bool a_transposed, bool b_transposed, bool bf16, hipStream_t s) {
  Cut cut;
  const hipError_t e = launch_product(p, EPI, a_transposed, b_transposed, bf16, &cut, s);
  if (e != hipSuccess || cut.splits == 1) return e;
  p.splits = cut.splits;
  const unsigned grid = (unsigned)std::min<int64_t>(((int64_t)(p.N + 7) / 8 * p.M * p.groups + kThreads - 1) / kThreads, 256 * 16);
  if (bf16) hipLaunchKernelGGL((join_parts_kernel<uint16_t, EPI>), dim3(grid), dim3(kThreads), 0, s, p);
  else hipLaunchKernelGGL((join_parts_kernel<float, EPI>), dim3(grid), dim3(kThreads), 0, s, p);
  return hipGetLastError();
}

// Statistics of the classes' pieces, `stride` apart: [rows of all workers][tiles], in the last one [..][last_tiles].
struct XentPieces { int pieces, tiles, last_tiles; int64_t stride; };

// Loss and lse of every row from its tiles' statistics, by as many lanes as it has tiles, at most a wavefront.
__global__ void __launch_bounds__(kThreads) join_tiles_kernel(XentArgs p, const float2* stats, const float* picked, XentPieces pieces, int lanes_log2) {
  const int lanes = 1 << lanes_log2, lane = threadIdx.x & (lanes - 1), slots = kThreads >> lanes_log2;
  const int64_t rows = p.rows * p.workers;
  for (int64_t r = (int64_t)blockIdx.x * slots + (threadIdx.x >> lanes_log2); r < rows; r += (int64_t)gridDim.x * slots) {
    float m = -INFINITY, s = 0.0f;
    for (int k = 0; k < pieces.pieces; ++k) {
      const int tiles = k + 1 == pieces.pieces ? pieces.last_tiles : pieces.tiles;
      constexpr int U = 4;
      for (int t = lane; t < tiles; t += lanes * U) {
        float2 v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) v[u] = t + u * lanes < tiles ? stats[k * pieces.stride + r * tiles + t + u * lanes] : make_float2(-INFINITY, 0.0f);
#pragma unroll
        for (int u = 0; u < U; ++u) join_stats(m, s, v[u].x, v[u].y);
      }
    }
    for (int d = 1; d < lanes; d <<= 1) join_stats(m, s, __shfl_xor(m, d), __shfl_xor(s, d));
    if (lane == 0) {
      const bool real = (unsigned)p.labels[r] < (unsigned)p.classes;
      write_loss(p.loss, p.lse, r, m, s, real, real ? picked[r] : 0.0f);
    }
  }
}

constexpr size_t kPieceBytes = (size_t)256 << 20;          // of dz, and of a copy of W

// Rows of bf16 whose length is no multiple of eight are copied to such a multiple, with zeros, where the products gain more by it than the copies take: aligned operands
// go to LDS by themselves.  An element of h is worth a copy from that many classes on, one of W from that many rows: gradients of 8 workers' rows x 1024 x 8001 classes, as
// they lie and by copies of W: 128 rows 174 and 175 us, 256 rows 289 and 222 us, 512 rows 491 and 296 us; of 16 workers' 256 rows x 129 x 333 24 and 24 us.
constexpr double kWorthACopy = 160, kWorthACopyForward = 256;
constexpr int64_t kLeastAligned = (int64_t)1 << 28;        // products of two elements
constexpr int64_t eights(int64_t n) { return (n + 7) / 8 * 8; }

__global__ void __launch_bounds__(kThreads) align_kernel(Operand from, Operand to, int rows, int width, int64_t total, int lanes_log2) {
  const int lanes = 1 << lanes_log2, slots = kThreads >> lanes_log2;
  for (int64_t i = (int64_t)blockIdx.x * slots + (threadIdx.x >> lanes_log2); i < total; i += (int64_t)gridDim.x * slots) {
    const int64_t g = (uint32_t)i / (uint32_t)rows, r = i - g * rows;
    const uint16_t* in = reinterpret_cast<const uint16_t*>(from.p) + g * from.gs + r * from.ld;
    uint16_t* out = reinterpret_cast<uint16_t*>(const_cast<void*>(to.p)) + g * to.gs + r * to.ld;
    for (int c = (threadIdx.x & (lanes - 1)) * 8; c < width; c += lanes * 8) {
      const int n = width - c;
      u32x4_t v = load_piece<2>(in + c, n, width < 8);
      if (n < 8) v = place_piece<2>(v, n);
      *reinterpret_cast<u32x4_t*>(out + c) = v;
    }
  }
}
hipError_t launch_align(const Operand& from, const Operand& to, int rows, int width, int workers, hipStream_t s) {
  const int lanes_log2 = lanes_for_row(width), slots = kThreads >> lanes_log2;
  const int64_t total = (int64_t)rows * workers;
  const unsigned grid = (unsigned)std::min<int64_t>((total + slots - 1) / slots, 256 * 64);
  hipLaunchKernelGGL(align_kernel, dim3(grid), dim3(kThreads), 0, s, from, to, rows, width, total, lanes_log2);
  return hipGetLastError();
}

// What a piece of the classes, `first` .. `first` + n, works on: rows and matrices, as they lie or as copies in whole eights.
hipError_t operands_of_piece(const XentArgs& x, const XentPlan& plan, char* ws, bool bf16, int first, int n, Operand* rows, Operand* matrix, hipStream_t s) {
  const int64_t at = x.classes_first ? first * x.w_row : first;
  *rows = {x.h, x.rows * x.h_row, x.h_row, false};
  *matrix = {(const char*)x.w + at * (bf16 ? 2 : 4), x.w_gs, x.w_row, false};
  if (plan.align_h) {
    const Operand copy{ws + plan.h, x.rows * eights(x.width), eights(x.width), true};
    if (first == 0)
      if (const hipError_t e = launch_align(*rows, copy, (int)x.rows, x.width, x.workers, s); e != hipSuccess) return e;
    *rows = copy;
  }
  if (plan.align_w) {
    const int r = x.classes_first ? n : x.width, c = x.classes_first ? x.width : n;
    const Operand copy{ws + plan.w, r * eights(c), eights(c), true};
    if (const hipError_t e = launch_align(*matrix, copy, r, c, x.workers, s); e != hipSuccess) return e;
    *matrix = copy;
  }
  return hipSuccess;
}

}  // namespace

hipError_t launch_xent(const XentArgs& x, const XentPlan& plan, char* ws, bool bf16, hipStream_t s) {
  Cut cut{};
  int64_t stats = 0;                     // of the pieces so far, one behind another
  XentPieces pieces{};
  for (int k = 0; k < plan.pieces; ++k) {
    const int first = k * plan.piece, n = std::min(plan.piece, x.classes - first);
    ProductArgs p{};
    if (const hipError_t e = operands_of_piece(x, plan, ws, bf16, first, n, &p.b, &p.a, s); e != hipSuccess) return e;
    p.M = n;
    p.N = (int)x.rows;
    p.K = x.width;
    p.groups = x.workers;
    p.splits = 1;
    p.labels = x.labels;
    p.rows = x.rows;
    p.class0 = first;
    p.classes = x.classes;
    p.stats = reinterpret_cast<float2*>(ws + plan.stats) + stats;
    p.picked = reinterpret_cast<float*>(ws + plan.picked);
    p.most_tiles = plan.tiles;
    p.loss_out = plan.pieces == 1 ? x.loss : nullptr;
    p.lse_out = x.lse;
    if (const hipError_t e = launch_product(p, PX_STATS, !x.classes_first, false, bf16, &cut, s); e != hipSuccess) return e;
    if (k == 0) pieces.tiles = cut.tiles_m;
    pieces.last_tiles = cut.tiles_m;
    stats += x.rows * x.workers * plan.tiles;
  }
  if (plan.pieces == 1 && cut.tiles_m == 1) return hipSuccess;             // done
  pieces.pieces = plan.pieces;
  pieces.stride = x.rows * x.workers * plan.tiles;
  const int tiles = (pieces.pieces - 1) * pieces.tiles + pieces.last_tiles;
  int lanes_log2 = 0;
  while (lanes_log2 < 6 && (1 << lanes_log2) < tiles) ++lanes_log2;
  const int slots = kThreads >> lanes_log2;
  const unsigned grid = (unsigned)std::min<int64_t>((x.rows * x.workers + slots - 1) / slots, 256 * 64);
  hipLaunchKernelGGL(join_tiles_kernel, dim3(grid), dim3(kThreads), 0, s, x, reinterpret_cast<const float2*>(ws + plan.stats),
                     reinterpret_cast<const float*>(ws + plan.picked), pieces, lanes_log2);
  return hipGetLastError();
}

hipError_t launch_xent_backward(const XentArgs& x, const XentPlan& plan, char* ws, bool bf16, hipStream_t s) {
  const int es = bf16 ? 2 : 4;
  for (int k = 0; k < plan.pieces; ++k) {
    const int first = k * plan.piece, n = std::min(plan.piece, x.classes - first);
    const int64_t dw_at = x.classes_first ? first * x.dw_row : first;
    const Operand dz{ws + plan.dz, x.rows * plan.piece, plan.piece, true};
    Operand rows, matrix;
    hipError_t e = operands_of_piece(x, plan, ws, bf16, first, n, &rows, &matrix, s);
    if (e != hipSuccess) return e;
    ProductArgs p{};
    p.groups = x.workers;
    p.labels = x.labels;
    p.lse = x.lse_in;
    p.dloss = x.dloss;
    p.rows = x.rows;
    p.class0 = first;
    p.classes = x.classes;
    p.real = reinterpret_cast<uint32_t*>(ws + plan.real);
    p.first_piece = k == 0;
    p.last_piece = k + 1 == plan.pieces;
    p.a = rows;
    p.b = matrix;
    p.M = (int)x.rows;
    p.N = n;
    p.K = x.width;
    p.out = ws + plan.dz;
    p.out_ld = dz.ld;
    p.out_gs = dz.gs;
    p.splits = 1;
    p.parts = reinterpret_cast<float*>(ws + plan.parts);
    const bool small = plan.pieces == 1 && small_gradients(x.rows, x.width, x.classes, bf16);
    const ProductArgs dz_of = p;
    if (!small) {
      p.splits = splits_of_logits(p.M, p.N, p.K, p.groups, bf16);
      if ((e = launch_gradient<PX_DZ>(p, false, !x.classes_first, bf16, s)) != hipSuccess) return e;
      p.splits = 1;
    }
    p.a = dz;
    p.N = x.width;
    p.K = n;
    p.out = x.dh;
    p.out_ld = x.dh_row;
    p.out_gs = x.rows * x.dh_row;
    p.sums = plan.pieces > 1 ? reinterpret_cast<float*>(ws + plan.sums) : nullptr;
    ProductArgs dh = p;
    p.a = x.classes_first ? dz : rows;
    p.b = x.classes_first ? rows : dz;
    p.M = x.classes_first ? n : x.width;
    p.N = x.classes_first ? x.width : n;
    p.K = (int)x.rows;
    p.out = (char*)x.dw + dw_at * es;
    p.out_ld = x.dw_row;
    p.out_gs = x.dw_gs;
    if (small) return launch_small_gradients(dz_of, dh, p, x.classes_first, bf16, s);
    dh.splits = splits_of(dh.M, dh.N, dh.K, dh.groups);
    p.splits = splits_of(p.M, p.N, p.K, p.groups);
    if (pair_gradients(dh, p, n, x.width, bf16)) {
      const bool aligned = bf16 && product_aligned(dh, false, x.classes_first) && product_aligned(p, true, true);
      if ((e = aligned ? launch_pair_bf16(dh, p, x.classes_first, s) : launch_pair_any(dh, p, x.classes_first, bf16, s)) != hipSuccess) return e;
      continue;
    }
    if ((e = launch_gradient<PX_DH>(dh, false, x.classes_first, bf16, s)) != hipSuccess) return e;
    if ((e = launch_gradient<PX_DW>(p, true, true, bf16, s)) != hipSuccess) return e;
  }
  return hipSuccess;
}

XentPlan xent_plan(int workers, int64_t rows, int width, int classes, bool classes_first, bool bf16, bool backward) {
  XentPlan e{};
  const size_t n = (size_t)workers * (size_t)rows, es = bf16 ? 2 : 4;
  size_t at = 0;
  auto take = [&](size_t bytes) { const size_t v = at; at += (bytes + 255) / 256 * 256; return v; };
  const bool odd_h = width % 8 != 0, odd_w = (classes_first ? width : classes) % 8 != 0;
  if (bf16 && rows > 0 && (double)n * width * classes >= (double)kLeastAligned) {
    const double copies = (odd_h ? 1.0 / classes : 0.0) + (odd_w ? 1.0 / (double)rows : 0.0);
    const bool worth = copies < 1.0 / (backward ? kWorthACopy : kWorthACopyForward);
    e.align_h = odd_h && worth;
    e.align_w = odd_w && worth;
  }
  const int whole = (classes + 255) / 256;                 // in 256 classes
  // of a class: what a piece holds of it
  const size_t held = std::max(backward ? n : 0, e.align_w ? (size_t)workers * eights(width) : 0) * es;
  const int64_t fit = held == 0 ? whole : std::max<int64_t>((int64_t)(kPieceBytes / (held * 256)), 1);
  const int pieces = (int)std::min<int64_t>(whole, (whole + fit - 1) / fit);
  e.piece = (whole + pieces - 1) / pieces * 256;
  e.pieces = (classes + e.piece - 1) / e.piece;
  if (!backward) {
    if (e.pieces == 1) e.piece = classes;
    // as many tiles as a piece gets, by whichever kernels take its operands
    auto tiles_of_piece = [&](int classes_of) {
      ProductArgs p{};
      p.a.padded = e.align_w;
      p.b.padded = e.align_h;
      p.M = classes_of;
      p.N = (int)rows;
      p.K = width;
      p.groups = workers;
      p.splits = 1;
      const int any = stats_rows_any(p, !classes_first, bf16), tile = bf16 ? std::min(any, stats_rows_bf16(p)) : any;
      return (classes_of + tile - 1) / tile;
    };
    e.tiles = tiles_of_piece(e.piece);
    if (e.pieces > 1) e.tiles = std::max(e.tiles, tiles_of_piece(classes - (e.pieces - 1) * e.piece));
    e.stats = take(n * e.pieces * e.tiles * sizeof(float2));
    e.picked = take(n * sizeof(float));
  } else {
    // rows of dz start at 16 bytes, at whole lines where they are longer than those
    if (e.pieces == 1) e.piece = classes < 64 ? (int)eights(classes) : (classes + 63) / 64 * 64;
    e.dz = take(n * e.piece * es);
    e.sums = e.pieces > 1 ? take(n * width * sizeof(float)) : 0;
    size_t parts = 0;
    for (const int n_of : {std::min(e.piece, classes), classes - (e.pieces - 1) * e.piece}) {          // the last piece has fewer tiles, and so perhaps more parts
      parts = std::max({parts, parts_bytes(rows, n_of, splits_of_logits(rows, n_of, width, workers, bf16), workers),
                        parts_bytes(rows, width, splits_of(rows, width, n_of, workers), workers), parts_bytes(width, n_of, splits_of(width, n_of, rows, workers), workers)});
    }
    e.parts = take(parts);
    e.real = take((size_t)workers * real_words(rows) * sizeof(uint32_t));
  }
  e.h = e.align_h ? take(n * eights(width) * es) : 0;
  e.w = e.align_w ? take((size_t)workers * eights(width) * eights(std::min(e.piece, classes)) * es) : 0;
  e.total = at;
  return e;
}

}  // namespace prsgd
