// Newton-Schulz orthogonalisation around its products: the sums of squares (and the momentum step, which is where the update is first
// read), the normalised update as halves, and whole calls whose shorter side is at most kShortSide.
// The elementwise launches are bound by HBM: 8 x 4096 x 4096 bf16 squares 58 us (4.6 TB/s), halves 153 us (5.2 TB/s); with momentum, 8 x 4096 x
// 1000 squares 58 us (6.3 TB/s), halves of the transpose 73 us (4.5 TB/s).
#include <atomic>

#include "orth_rows.h"

namespace prsgd {

namespace {

// the scale that normalises; a zero matrix stays zero
__device__ __forceinline__ double norm_scale(double squares, float eps) {
  const double d = sqrt(squares) + (double)eps;
  return d == 0.0 ? 0.0 : 1.0 / d;
}

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int d = 1; d < kWave; d <<= 1) v += __shfl_xor(v, d);
  return v;
}

// Sums of squares in 64 bits (an fp32 sum overflows from elements of 1e19 on), a share of the matrix per workgroup.
template <typename T> __global__ void __launch_bounds__(kThreads) orth_squares_kernel(OrthMatrices p, double* parts) {
  const int g = blockIdx.y;
  const uint32_t per_row = (uint32_t)(p.cols + 7) / 8, total = (uint32_t)p.rows * per_row;
  double s = 0.0;
#pragma unroll 2
  for (uint32_t i = blockIdx.x * kThreads + threadIdx.x; i < total; i += gridDim.x * kThreads) {
    const uint32_t row = i / per_row;
    const int c = (int)(i - row * per_row) * 8;
    float u[8];
    update8<T>(p, g, (int)row, c, p.cols - c, false, u);
#pragma unroll
    for (int e = 0; e < 8; ++e) s = fma((double)u[e], (double)u[e], s);
  }
  s = wave_sum(s);
  __shared__ double sums[kThreads / kWave];
  if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) parts[g * gridDim.x + blockIdx.x] = ((sums[0] + sums[1]) + sums[2]) + sums[3];
}

// X_0 = U / (|U| + eps) times kHalfScale and 2^room as halves, a tile of 64 x 64 elements per workgroup.  TURNED: X is the transpose of U, by way of LDS.
template <typename T, bool TURNED>
__global__ void __launch_bounds__(kThreads) orth_load_kernel(OrthMatrices p, const double* parts, int n_parts, OrthHalves h) {
  constexpr bool SPLIT = sizeof(T) == 4;
  __shared__ float tile[64][65];
  const int g = blockIdx.z, r0 = blockIdx.y * 64, c0 = blockIdx.x * 64;
  double squares = 0.0;
  for (int i = threadIdx.x & 63; i < n_parts; i += kWave) squares += parts[g * n_parts + i];
  squares = wave_sum(squares);
  const double normal = norm_scale(squares, p.eps), size = sqrt(squares) * normal;        // |X_0|, below 2^e
  int e = 0;
  if (size > 0.0) (void)frexp(size, &e);
  const int room = min(max(-e, 0), kMostRoom);
  const double scale = ldexp(normal * (double)kHalfScale, room);
  if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) h.room[g] = room;
  const int lane_row = threadIdx.x >> 3, lane_col = (threadIdx.x & 7) * 8;
  const int rows = TURNED ? p.cols : p.rows, cols = TURNED ? p.rows : p.cols;           // of X
  auto write = [&](int row, int col, const float (&v)[8]) __attribute__((always_inline)) {
    const int hc = SPLIT ? (col >> 4) * 32 + (col & 15) : col;
    if (row >= half_rows(rows) || hc >= h.ld_x) return;
    u32x4_t hi, lo;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const _Float16 a = (_Float16)v[2 * e], b = (_Float16)v[2 * e + 1];
      const _Float16 ra = (_Float16)(v[2 * e] - (float)a), rb = (_Float16)(v[2 * e + 1] - (float)b);
      hi[e] = (uint32_t)__builtin_bit_cast(uint16_t, a) | (uint32_t)__builtin_bit_cast(uint16_t, b) << 16;
      lo[e] = (uint32_t)__builtin_bit_cast(uint16_t, ra) | (uint32_t)__builtin_bit_cast(uint16_t, rb) << 16;
    }
    const int64_t at = g * h.x_gs + (int64_t)row * h.ld_x + hc;
    *reinterpret_cast<u32x4_t*>(h.x + at) = hi;
    if (SPLIT) *reinterpret_cast<u32x4_t*>(h.x + at + 16) = lo;
    else *reinterpret_cast<u32x4_t*>(h.x_lo + at) = lo;
    if (row >= rows) {
      const u32x4_t zero = {0, 0, 0, 0};
      *reinterpret_cast<u32x4_t*>(h.spare + at) = zero;
      if (SPLIT) *reinterpret_cast<u32x4_t*>(h.spare + at + 16) = zero;
    }
  };
#pragma unroll
  for (int i = 0; i < 64; i += 32) {
    const int r = r0 + i + lane_row, c = c0 + lane_col;
    float u[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
    if (r < p.rows && c < p.cols) update8<T>(p, g, r, c, p.cols - c, true, u);
#pragma unroll
    for (int e = 0; e < 8; ++e) u[e] = c + e < p.cols ? (float)((double)u[e] * scale) : 0.0f;
    if (r >= p.rows) {
#pragma unroll
      for (int e = 0; e < 8; ++e) u[e] = 0.0f;
    }
    if (TURNED) {
#pragma unroll
      for (int e = 0; e < 8; ++e) tile[i + lane_row][lane_col + e] = u[e];
    } else {
      write(r, c, u);
    }
  }
  if (!TURNED) return;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 64; i += 32) {
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = tile[lane_col + e][i + lane_row];
    write(c0 + i + lane_row, r0 + lane_col, v);
  }
}

// ---- short sides -------------------------------------------------------------------------------
// With r = min(rows, cols) <= kShortSide every iterate is P U with P an r x r polynomial of the Gram matrix K = U U^T (all of them
// symmetric, and they commute):
//   A_0 = K / (|U| + eps)^2,  Q = a + b A + c A A,  P <- Q P,  A <- Q A Q,   |U|^2 = trace K,
// so U is read for K and for P U, 3 r^2 L operations in all instead of 3 r^2 L per step, and a whole call is one launch or two.  The Gram
// matrix squares the condition: in 64 bits its smallest eigenvalues are as good as fp32 singular values are for as many steps as the
// host lets through here (10 at the default coefficients); rounded ones may be negative, and grow without bound in the end.  K and the polynomials run on v_mfma_f64_16x16x4, P U on v_mfma_f32_16x16x4.
// 64 x (128 x 10) 8.3 us in one launch of 64 workgroups, latency from end to end.  A call of this and of the products' path: 64 x (64 x
// 64) in fp32 53 and 68 us, 64 x (64 x 512) 72 and 95, 4 x (64 x 4096) 79 and 176; in bf16 8 x (64 x 1024) 66 and 73, 64 x (64 x 512) 72 and 80.
// A symmetric matrix of NB x NB blocks of 16 is kept as operands: element q of lane (g = lane / 16, i = lane % 16) of block (x, y) is
// M[16 x + i][16 y + 4 q + g].  That is what a product takes from either side, and the product's block (x, y) comes out as block (y, x).
typedef double f64x4_t __attribute__((ext_vector_type(4)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));

struct ShortShape { int r, longer; bool tall; };
template <int NB> struct Short {
  static constexpr int ROWS = 16 * NB, CHUNK = NB <= 2 ? 256 : 128;        // long-side positions in LDS at a time
  static constexpr int PITCH = CHUNK + 4;                                  // 16 rows x 4 positions on 64 banks
  static constexpr int MATRIX = NB * NB * 256;                             // doubles of a matrix
  static constexpr int U_BYTES = ROWS * PITCH * 4;
  // four matrices; U lies on the last two of them where the two would not fit beside each other
  static constexpr int U_AT = NB <= 2 ? 4 * MATRIX * 8 : 2 * MATRIX * 8;
  static constexpr int LDS = U_AT + U_BYTES > 4 * MATRIX * 8 ? U_AT + U_BYTES : 4 * MATRIX * 8;
  static_assert(LDS <= 160 * 1024, "LDS of a compute unit");
};

// U at long-side positions [l0, l0 + n), zeros up to a multiple of 16 positions; eight elements of a row of U at a time
template <typename T, int NB>
__device__ __forceinline__ void stage(const OrthMatrices& p, const ShortShape& s, int g, int l0, int n, bool stepped, float* u) {
  constexpr int P = Short<NB>::PITCH;
  const int m = (n + 15) & ~15, per_row = ((s.tall ? s.r : m) + 7) / 8, total = (s.tall ? m : s.r) * per_row;
#pragma unroll 2
  for (int i = threadIdx.x; i < total; i += kThreads) {
    const int row = i / per_row, c = (i - row * per_row) * 8;
    float v[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
    if (s.tall) {
      if (row < n) update8<T>(p, g, l0 + row, c, s.r - c, stepped, v);
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (c + e < s.r) u[(c + e) * P + row] = v[e];
    } else {
      if (c < n) update8<T>(p, g, row, l0 + c, n - c, stepped, v);
      f32x4_t* to = reinterpret_cast<f32x4_t*>(u + row * P + c);
      to[0] = (f32x4_t){v[0], v[1], v[2], v[3]};
      to[1] = (f32x4_t){v[4], v[5], v[6], v[7]};
    }
  }
}
// ... and the result from there to the caller's matrices
template <typename T, int NB>
__device__ __forceinline__ void unstage(const OrthMatrices& p, const ShortShape& s, int g, int l0, int n, const float* u) {
  constexpr int P = Short<NB>::PITCH;
  const int per_row = ((s.tall ? s.r : n) + 7) / 8, total = (s.tall ? n : s.r) * per_row;
#pragma unroll 2
  for (int i = threadIdx.x; i < total; i += kThreads) {
    const int row = i / per_row, c = (i - row * per_row) * 8;
    float v[8];
    if (s.tall) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = u[min(c + e, s.r - 1) * P + row];
      result8<T>(p, g * p.out_matrix + (int64_t)(l0 + row) * p.out_row + c, s.r - c, v);
    } else {
      const f32x4_t* from = reinterpret_cast<const f32x4_t*>(u + row * P + c);
      const f32x4_t lo = from[0], hi = from[1];
#pragma unroll
      for (int e = 0; e < 4; ++e) { v[e] = lo[e]; v[4 + e] = hi[e]; }
      result8<T>(p, g * p.out_matrix + (int64_t)row * p.out_row + l0 + c, n - c, v);
    }
  }
}

// Place of element e of a lane of one block in the transposed block
__device__ __forceinline__ int transposed_place(int e, int lane) { return (lane & 15) / 4 * 64 + (lane & 3) * 16 + 4 * e + (lane >> 4); }
// K over the long-side positions [l0, l1) into the first matrix of LDS; U's last chunk stays there if U has a place of its own.
template <typename T, int NB>
__device__ __forceinline__ void gram_of(const OrthMatrices& p, const ShortShape& s, int g, int l0, int l1, double* lds, float* u) {
  using S = Short<NB>;
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6, i = lane & 15, q4 = lane >> 4;
  for (int e = t + s.r * S::PITCH; e < S::ROWS * S::PITCH; e += kThreads) u[e] = 0.0f;       // rows past the side
  f64x4_t acc[NB * (NB + 1) / 2];
#pragma unroll
  for (int b = 0; b < NB * (NB + 1) / 2; ++b) acc[b] = (f64x4_t){0.0, 0.0, 0.0, 0.0};
  for (int l = l0; l < l1; l += S::CHUNK) {
    const int n = min(S::CHUNK, l1 - l);
    if (l > l0) __syncthreads();
    stage<T, NB>(p, s, g, l, n, false, u);
    __syncthreads();
    for (int x = wave; x < (n + 3) / 4; x += 4) {
      double v[NB];
#pragma unroll
      for (int b = 0; b < NB; ++b) v[b] = u[(16 * b + i) * S::PITCH + 4 * x + q4];
      int k = 0;
#pragma unroll
      for (int y = 0; y < NB; ++y)
#pragma unroll
        for (int x2 = 0; x2 <= y; ++x2, ++k) acc[k] = __builtin_amdgcn_mfma_f64_16x16x4f64(v[x2], v[y], acc[k], 0, 0, 0);
    }
  }
  if (S::U_AT < 4 * S::MATRIX * 8) __syncthreads();
  int k = 0;
#pragma unroll
  for (int y = 0; y < NB; ++y)
#pragma unroll
    for (int x = 0; x <= y; ++x, ++k)
#pragma unroll
      for (int e = 0; e < 4; ++e) lds[wave * S::MATRIX + (y * NB + x) * 256 + e * 64 + lane] = acc[k][e];
  __syncthreads();
  // the wavefronts' shares in ascending order; a block above the diagonal is the transpose of the one below
  const int mirrored = transposed_place(wave, lane);       // thread: element wave of lane
#pragma unroll
  for (int y = 0; y < NB; ++y)
#pragma unroll
    for (int x = 0; x <= y; ++x) {
      const int at = (y * NB + x) * 256 + t;
      const double v = ((lds[at] + lds[S::MATRIX + at]) + lds[2 * S::MATRIX + at]) + lds[3 * S::MATRIX + at];
      lds[at] = v;
      if (x != y) lds[(x * NB + y) * 256 + mirrored] = v;
    }
  __syncthreads();
}

// d <- f(y x^T), blocks come out transposed; every wavefront meets the others behind it.  Operands are symmetric but for rounding, and the
// order counts for that: A <- (Q A^T) Q^T turns an unsymmetric rounding of A's around and makes it q_i q_j times as large, as it does a
// symmetric one between two directions; Q (Q A^T) would make it 2 |b| + 1 times as large where A is the identity (1e-3 of the result after 14
// default steps at 2 x 7, NaN after 30 of (2, -1.5, 0.5)).  (Blocks on and below the diagonal alone, with the others written as their
// transposes, save a quarter of the products at NB = 4 and took as long: 55 against 52 us for a call on 64 x 64.)
template <int NB, typename F>
__device__ __forceinline__ void short_product(const double* x, const double* y, double* d, F&& f) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int b = wave; b < NB * NB; b += 4) {
    const int i = b / NB, j = b % NB;
    f64x4_t acc = {0.0, 0.0, 0.0, 0.0};
#pragma unroll
    for (int k = 0; k < NB; ++k)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        acc = __builtin_amdgcn_mfma_f64_16x16x4f64(x[(i * NB + k) * 256 + q * 64 + lane], y[(j * NB + k) * 256 + q * 64 + lane], acc, 0, 0, 0);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int at = (j * NB + i) * 256 + e * 64 + lane;
      d[at] = f(acc[e], at, i == j && 4 * e + (lane >> 4) == (lane & 15));
    }
  }
  __syncthreads();
}

// P of the scaled Gram matrix in the first matrix of LDS, as operands in fp32; a single block stays in registers, in every wavefront
template <int NB>
__device__ __forceinline__ void polynomial_of(const OrthMatrices& p, double* lds, float (&pf)[NB][NB][4]) {
  const int lane = threadIdx.x & 63;
  const double a = p.a, b = p.b, c = p.c;
  if constexpr (NB == 1) {
    auto product = [](f64x4_t x, f64x4_t y) __attribute__((always_inline)) {
      f64x4_t acc = {0.0, 0.0, 0.0, 0.0};
#pragma unroll
      for (int q = 0; q < 4; ++q) acc = __builtin_amdgcn_mfma_f64_16x16x4f64(x[q], y[q], acc, 0, 0, 0);
      return acc;
    };
    f64x4_t m, poly = {0.0, 0.0, 0.0, 0.0};
#pragma unroll
    for (int q = 0; q < 4; ++q) m[q] = lds[q * 64 + lane];
    for (int step = 0; step < p.steps; ++step) {
      const f64x4_t square = product(m, m);
      f64x4_t f;
#pragma unroll
      for (int q = 0; q < 4; ++q) f[q] = fma(c, square[q], fma(b, m[q], 4 * q + (lane >> 4) == (lane & 15) ? a : 0.0));
      poly = step == 0 ? f : product(f, poly);
      if (step + 1 < p.steps) m = product(f, product(m, f));
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) pf[0][0][q] = (float)poly[q];
  } else {
    constexpr int M = Short<NB>::MATRIX;
    double* m = lds;
    double* f = lds + M;
    double* poly = lds + 2 * M;
    double* spare = lds + 3 * M;
    auto plain = [](double v, int, bool) { return v; };
    for (int step = 0; step < p.steps; ++step) {
      short_product<NB>(m, m, f, [&](double v, int at, bool diagonal) { return fma(c, v, fma(b, m[at], diagonal ? a : 0.0)); });
      if (step == 0) {
        for (int e = threadIdx.x; e < M; e += kThreads) poly[e] = f[e];
      } else {
        short_product<NB>(f, poly, spare, plain);
        double* old = poly;
        poly = spare;
        spare = old;
      }
      if (step + 1 < p.steps) {
        short_product<NB>(m, f, spare, plain);
        short_product<NB>(f, spare, m, plain);
      }
    }
    __syncthreads();
#pragma unroll
    for (int x = 0; x < NB; ++x)
#pragma unroll
      for (int y = 0; y < NB; ++y)
#pragma unroll
        for (int q = 0; q < 4; ++q) pf[x][y][q] = (float)poly[(x * NB + y) * 256 + q * 64 + lane];
    if (Short<NB>::U_AT < 4 * M * 8) __syncthreads();
  }
}

template <int NB> __device__ __forceinline__ int slice_length(const ShortShape& s, int slices) {
  constexpr int C = Short<NB>::CHUNK;
  return ((s.longer + C - 1) / C + slices - 1) / slices * C;
}
template <typename T, int NB>
__global__ void __launch_bounds__(kThreads) orth_short_gram_kernel(OrthMatrices p, ShortShape s, double* grams, int slices) {
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  double* lds = reinterpret_cast<double*>(smem);
  const int g = blockIdx.y, per = slice_length<NB>(s, slices), l0 = min(s.longer, (int)blockIdx.x * per), l1 = min(s.longer, l0 + per);
  gram_of<T, NB>(p, s, g, l0, l1, lds, reinterpret_cast<float*>(smem + Short<NB>::U_AT));
  double* out = grams + ((int64_t)g * slices + blockIdx.x) * Short<NB>::MATRIX;
  for (int e = threadIdx.x; e < Short<NB>::MATRIX; e += kThreads) out[e] = lds[e];
}

// ALONE: a matrix has one workgroup, which computes K itself.
template <typename T, int NB, bool ALONE>
__global__ void __launch_bounds__(kThreads) orth_short_kernel(OrthMatrices p, ShortShape s, const double* grams, int slices) {
  using S = Short<NB>;
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  double* lds = reinterpret_cast<double*>(smem);
  float* u = reinterpret_cast<float*>(smem + S::U_AT);
  const int g = blockIdx.y, t = threadIdx.x, lane = t & 63, wave = t >> 6, i = lane & 15, q4 = lane >> 4;
  const int per = slice_length<NB>(s, slices), l0 = min(s.longer, (int)blockIdx.x * per), l1 = min(s.longer, l0 + per);
  if (ALONE) {
    gram_of<T, NB>(p, s, g, 0, s.longer, lds, u);
  } else {
    // slices in ascending order; a thread asks for all its elements of a slice at once (one by one this took 70 us of 6 x (2233 x 55))
    constexpr int N = S::MATRIX / kThreads;
    double v[N];
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = 0.0;
#pragma unroll 2
    for (int q = 0; q < slices; ++q) {
      const double* from = grams + ((int64_t)g * slices + q) * S::MATRIX + t;
#pragma unroll
      for (int k = 0; k < N; ++k) v[k] += from[k * kThreads];
    }
#pragma unroll
    for (int k = 0; k < N; ++k) lds[k * kThreads + t] = v[k];
    __syncthreads();
  }
  // the diagonal: element 4 q + g = i of block (x, x)
  double squares = 0.0;
  if (lane < S::ROWS) squares = lds[(lane / 16) * (NB + 1) * 256 + (lane % 16 / 4) * 64 + (lane % 4) * 16 + lane % 16];
  const double scale = norm_scale(wave_sum(squares), p.eps);
  __syncthreads();
  for (int e = t; e < S::MATRIX; e += kThreads) lds[e] *= scale * scale;
  __syncthreads();
  float pf[NB][NB][4];
  polynomial_of<NB>(p, lds, pf);

  const bool staged = ALONE && NB <= 2 && s.longer <= S::CHUNK;            // U still lies in LDS
  if (!staged)
    for (int e = t + s.r * S::PITCH; e < S::ROWS * S::PITCH; e += kThreads) u[e] = 0.0f;
  for (int l = l0; l < l1; l += S::CHUNK) {
    const int n = min(S::CHUNK, l1 - l);
    if (!staged) {
      stage<T, NB>(p, s, g, l, n, true, u);
      __syncthreads();
    }
    // P U, 16 positions at a time, in place
    for (int x = wave; x < (n + 15) / 16; x += 4) {
      f32x4_t o[NB];
#pragma unroll
      for (int a = 0; a < NB; ++a) o[a] = (f32x4_t){0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int k = 0; k < NB; ++k)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const float v = (float)((double)u[(16 * k + 4 * q + q4) * S::PITCH + 16 * x + i] * scale);
#pragma unroll
          for (int a = 0; a < NB; ++a) o[a] = __builtin_amdgcn_mfma_f32_16x16x4f32(pf[a][k][q], v, o[a], 0, 0, 0);
        }
#pragma unroll
      for (int a = 0; a < NB; ++a)
#pragma unroll
        for (int e = 0; e < 4; ++e) u[(16 * a + 4 * q4 + e) * S::PITCH + 16 * x + i] = o[a][e];
    }
    __syncthreads();
    unstage<T, NB>(p, s, g, l, n, u);
    __syncthreads();
  }
}

}  // namespace

hipError_t launch_orth_squares(const OrthMatrices& p, double* parts, hipStream_t s) {
  const dim3 grid((unsigned)norm_parts(p.rows, p.cols), (unsigned)p.count);
  if (p.bf16) hipLaunchKernelGGL(orth_squares_kernel<uint16_t>, grid, dim3(kThreads), 0, s, p, parts);
  else hipLaunchKernelGGL(orth_squares_kernel<float>, grid, dim3(kThreads), 0, s, p, parts);
  return hipGetLastError();
}

hipError_t launch_orth_load(const OrthMatrices& p, const double* parts, const OrthHalves& h, hipStream_t s) {
  const dim3 grid((unsigned)(p.cols + 63) / 64, (unsigned)(p.rows + 63) / 64, (unsigned)p.count);
  const int n = norm_parts(p.rows, p.cols);
  const bool turned = p.rows > p.cols;
  if (p.bf16) {
    if (turned) hipLaunchKernelGGL((orth_load_kernel<uint16_t, true>), grid, dim3(kThreads), 0, s, p, parts, n, h);
    else hipLaunchKernelGGL((orth_load_kernel<uint16_t, false>), grid, dim3(kThreads), 0, s, p, parts, n, h);
  } else {
    if (turned) hipLaunchKernelGGL((orth_load_kernel<float, true>), grid, dim3(kThreads), 0, s, p, parts, n, h);
    else hipLaunchKernelGGL((orth_load_kernel<float, false>), grid, dim3(kThreads), 0, s, p, parts, n, h);
  }
  return hipGetLastError();
}

namespace {
int short_blocks(int r) { return (r + 15) / 16; }
int short_chunk(int r) { return short_blocks(r) <= 2 ? Short<2>::CHUNK : Short<4>::CHUNK; }

template <typename T, int NB> hipError_t launch_short_as(const OrthMatrices& p, const ShortShape& shape, double* grams, int slices, hipStream_t s) {
  constexpr int kLds = Short<NB>::LDS;
  static std::atomic<bool> configured{false};              // past the 64 KB default; setting the limit twice is harmless
  if (!configured.load(std::memory_order_acquire)) {
    for (const void* k : {reinterpret_cast<const void*>(orth_short_gram_kernel<T, NB>), reinterpret_cast<const void*>(orth_short_kernel<T, NB, true>),
                          reinterpret_cast<const void*>(orth_short_kernel<T, NB, false>)}) {
      hipError_t e = hipFuncSetAttribute(k, hipFuncAttributeMaxDynamicSharedMemorySize, kLds);
      if (e != hipSuccess) return e;
    }
    configured.store(true, std::memory_order_release);
  }
  const dim3 grid((unsigned)slices, (unsigned)p.count);
  if (slices == 1) {
    hipLaunchKernelGGL((orth_short_kernel<T, NB, true>), grid, dim3(kThreads), kLds, s, p, shape, grams, slices);
    return hipGetLastError();
  }
  hipLaunchKernelGGL((orth_short_gram_kernel<T, NB>), grid, dim3(kThreads), kLds, s, p, shape, grams, slices);
  hipLaunchKernelGGL((orth_short_kernel<T, NB, false>), grid, dim3(kThreads), kLds, s, p, shape, grams, slices);
  return hipGetLastError();
}
template <typename T> hipError_t launch_short(const OrthMatrices& p, const ShortShape& shape, double* grams, int slices, hipStream_t s) {
  switch (short_blocks(shape.r)) {
    case 1: return launch_short_as<T, 1>(p, shape, grams, slices, s);
    case 2: return launch_short_as<T, 2>(p, shape, grams, slices, s);
    case 3: return launch_short_as<T, 3>(p, shape, grams, slices, s);
    default: return launch_short_as<T, 4>(p, shape, grams, slices, s);
  }
}
}  // namespace

size_t orth_short_doubles(int r) { return (size_t)short_blocks(r) * short_blocks(r) * 256; }
// Slices of the long side: two chunks stay in one launch, which saves the second; more are dealt to as many workgroups as the device holds (8 x
// (16 x 1024) in one launch 21 us, in four slices 12).
int orth_short_slices(int count, int r, int longer) {
  const int chunks = (longer + short_chunk(r) - 1) / short_chunk(r);
  int slices = (short_blocks(r) == 4 ? 256 : 512) / count;    // what the device holds at once
  if (slices > 16) slices = 16;
  if (slices > chunks) slices = chunks;
  return chunks <= 2 || slices < 2 ? 1 : slices;
}

hipError_t launch_orth_short(const OrthMatrices& p, double* grams, int slices, hipStream_t s) {
  const ShortShape shape{p.rows < p.cols ? p.rows : p.cols, p.rows < p.cols ? p.cols : p.rows, p.rows > p.cols};
  return p.bf16 ? launch_short<uint16_t>(p, shape, grams, slices, s) : launch_short<float>(p, shape, grams, slices, s);
}

}  // namespace prsgd
