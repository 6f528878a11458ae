// Newton-Schulz orthogonalisation around its products: the sums of squares (and the momentum step, which is where the update is first
// read), the normalised update as halves in both orientations, and whole calls whose shorter side is at most kShortSide.
#include "prsgd_internal.h"
#include "prsgd_ops_internal.h"

namespace prsgd {

namespace {

template <typename T> __device__ __forceinline__ float value(T v) {
  if constexpr (sizeof(T) == 4) return v; else return bf16_to_f32(v);
}
template <typename T> __device__ __forceinline__ void put(T* p, float f) {
  if constexpr (sizeof(T) == 4) *p = f; else *p = f32_to_bf16_rne(f);
}
// M <- mu M + G, and the element of U; `stepped`: an earlier launch has moved M on
template <typename T> __device__ __forceinline__ float update_at(const OrthMatrices& p, int g, int row, int col, bool stepped) {
  const float v = value(reinterpret_cast<const T*>(p.g)[g * p.g_matrix + row * p.g_row + col]);
  if (p.m == nullptr) return v;
  float* at = p.m + g * p.m_matrix + row * p.m_row + col;
  float m = *at;
  if (!stepped) {
    m = fmaf(p.mu, m, v);
    *at = m;
  }
  return fmaf(p.m_part, m, p.g_part * v);
}
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

// Eight elements of U at a row's column c, n of them inside it (the others are zero); M moves on unless an earlier launch did that.
typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));
template <int ES> struct __attribute__((packed, aligned(ES))) Packed16 { u32x4_t v; };
template <typename T> __device__ __forceinline__ void load8(const T* p, int n, float (&v)[8]) {
  if (n >= 8) {
    if constexpr (sizeof(T) == 4) {
      const u32x4_t lo = reinterpret_cast<const Packed16<4>*>(p)->v, hi = reinterpret_cast<const Packed16<4>*>(p + 4)->v;
#pragma unroll
      for (int e = 0; e < 4; ++e) { v[e] = __uint_as_float(lo[e]); v[4 + e] = __uint_as_float(hi[e]); }
    } else {
      const u32x4_t x = reinterpret_cast<const Packed16<2>*>(p)->v;
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = __uint_as_float((e & 1) != 0 ? x[e / 2] & 0xFFFF0000u : x[e / 2] << 16);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = e < n ? value(p[e]) : 0.0f;
  }
}
template <typename T> __device__ __forceinline__ void update8(const OrthMatrices& p, int g, int row, int c, int n, bool stepped, float (&u)[8]) {
  load8(reinterpret_cast<const T*>(p.g) + g * p.g_matrix + row * p.g_row + c, n, u);
  if (p.m == nullptr) return;
  float* at = p.m + g * p.m_matrix + row * p.m_row + c;
  float m[8];
  load8(at, n, m);
  if (!stepped) {
#pragma unroll
    for (int e = 0; e < 8; ++e) m[e] = fmaf(p.mu, m[e], u[e]);
    if (n >= 8) {
      reinterpret_cast<Packed16<4>*>(at)->v = (u32x4_t){__float_as_uint(m[0]), __float_as_uint(m[1]), __float_as_uint(m[2]), __float_as_uint(m[3])};
      reinterpret_cast<Packed16<4>*>(at + 4)->v = (u32x4_t){__float_as_uint(m[4]), __float_as_uint(m[5]), __float_as_uint(m[6]), __float_as_uint(m[7])};
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e < n) at[e] = m[e];
    }
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) u[e] = fmaf(p.m_part, m[e], p.g_part * u[e]);
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

// X_0 = U / (|U| + eps) times kHalfScale as halves, a tile of 64 x 64 elements per workgroup.  TURNED: X is the transpose of U, by way of LDS.
template <typename T, bool TURNED>
__global__ void __launch_bounds__(kThreads) orth_load_kernel(OrthMatrices p, const double* parts, int n_parts, OrthHalves h) {
  constexpr bool SPLIT = sizeof(T) == 4;
  __shared__ float tile[64][65];
  const int g = blockIdx.z, r0 = blockIdx.y * 64, c0 = blockIdx.x * 64;
  double squares = 0.0;
  for (int i = threadIdx.x & 63; i < n_parts; i += kWave) squares += parts[g * n_parts + i];
  const double scale = norm_scale(wave_sum(squares), p.eps) * (double)kHalfScale;
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
// With r = min(rows, cols) <= 32 every iterate is P U with P an r x r polynomial of the Gram matrix K = U U^T (all of them commute):
//   A_0 = K / (|U| + eps)^2,  Q = a + b A + c A A,  P <- Q P,  A <- Q A Q,   |U|^2 = trace K,
// so U is read once for K and once for P U, 3 r^2 L operations in all instead of 3 r^2 L per step.  The Gram matrix squares the
// condition; in 64 bits its smallest eigenvalues are as good as fp32 singular values are, in fp32 they may come out negative and grow.
constexpr int kChunk = 128;              // long-side positions in LDS at a time
constexpr int kPitch = kShortSide + 1;

struct ShortShape { int r, longer; bool tall; };

template <typename T>
__device__ __forceinline__ void stage(const OrthMatrices& p, const ShortShape& s, int g, int l0, int n, bool stepped,
                                      double scale, float (&u)[kShortSide][kChunk + 1]) {
  for (int i = threadIdx.x; i < s.r * n; i += kThreads) {
    int a, l;
    if (s.tall) { l = i / s.r; a = i - l * s.r; } else { a = i / n; l = i - a * n; }
    u[a][l] = (float)((double)(s.tall ? update_at<T>(p, g, l0 + l, a, stepped) : update_at<T>(p, g, a, l0 + l, stepped)) * scale);
  }
}

// K over the long-side positions [l0, l1) into LDS.  A thread has a 2 x 2 block on or below the diagonal, and of the positions its share.
template <typename T>
__device__ __forceinline__ void gram_of(const OrthMatrices& p, const ShortShape& s, int g, int l0, int l1, bool stepped,
                                        float (&u)[kShortSide][kChunk + 1], double (&share)[4][kThreads], double (&k)[kShortSide][kPitch]) {
  const int rb = (s.r + 1) / 2, blocks = rb * (rb + 1) / 2, shares = kThreads / blocks;
  const int t = threadIdx.x, block = t % blocks, part = t / blocks;
  int bi = 0;
  while ((bi + 1) * (bi + 2) / 2 <= block) ++bi;
  const int bj = block - bi * (bi + 1) / 2;
  const int i0 = 2 * bi, i1 = min(2 * bi + 1, s.r - 1), j0 = 2 * bj, j1 = min(2 * bj + 1, s.r - 1);
  double a00 = 0.0, a01 = 0.0, a10 = 0.0, a11 = 0.0;
  for (int l = l0; l < l1; l += kChunk) {
    const int n = min(kChunk, l1 - l);
    __syncthreads();
    stage<T>(p, s, g, l, n, stepped, 1.0, u);
    __syncthreads();
    if (part < shares)
      for (int x = part; x < n; x += shares) {
        const double xi0 = u[i0][x], xi1 = u[i1][x], xj0 = u[j0][x], xj1 = u[j1][x];
        a00 = fma(xi0, xj0, a00);
        a01 = fma(xi0, xj1, a01);
        a10 = fma(xi1, xj0, a10);
        a11 = fma(xi1, xj1, a11);
      }
  }
  share[0][t] = a00;
  share[1][t] = a01;
  share[2][t] = a10;
  share[3][t] = a11;
  __syncthreads();
  for (int e = t; e < 4 * blocks; e += kThreads) {
    const int which = e / blocks, bk = e - which * blocks;
    double v = 0.0;
    for (int q = 0; q < shares; ++q) v += share[which][q * blocks + bk];
    int i = 0;
    while ((i + 1) * (i + 2) / 2 <= bk) ++i;
    const int j = bk - i * (i + 1) / 2, x = 2 * i + (which >> 1), y = 2 * j + (which & 1);
    if (x < s.r && y < s.r && (i != j || which != 1)) {
      k[x][y] = v;
      k[y][x] = v;
    }
  }
  __syncthreads();
}

// d <- x y for r x r matrices that commute and are symmetric (so y's columns are its rows), 2 x 2 elements a thread.  f: of the result.
template <typename F>
__device__ __forceinline__ void short_product(const double (&x)[kShortSide][kPitch], const double (&y)[kShortSide][kPitch],
                                              double (&d)[kShortSide][kPitch], int r, F&& f) {
  const int rb = (r + 1) / 2;
  for (int t = threadIdx.x; t < rb * rb; t += kThreads) {
    const int i0 = 2 * (t / rb), j0 = 2 * (t % rb), i1 = min(i0 + 1, r - 1), j1 = min(j0 + 1, r - 1);
    double a00 = 0.0, a01 = 0.0, a10 = 0.0, a11 = 0.0;
    for (int k = 0; k < r; ++k) {
      const double xi0 = x[i0][k], xi1 = x[i1][k], yj0 = y[k][j0], yj1 = y[k][j1];
      a00 = fma(xi0, yj0, a00);
      a01 = fma(xi0, yj1, a01);
      a10 = fma(xi1, yj0, a10);
      a11 = fma(xi1, yj1, a11);
    }
    d[i0][j0] = f(a00, i0, j0);
    if (j0 + 1 < r) d[i0][j1] = f(a01, i0, j1);
    if (i0 + 1 < r) d[i1][j0] = f(a10, i1, j0);
    if (i0 + 1 < r && j0 + 1 < r) d[i1][j1] = f(a11, i1, j1);
  }
  __syncthreads();
}

template <typename T> __global__ void __launch_bounds__(kThreads) orth_short_gram_kernel(OrthMatrices p, ShortShape s, double* grams, int slices) {
  __shared__ float u[kShortSide][kChunk + 1];
  __shared__ double share[4][kThreads], k[kShortSide][kPitch];
  const int g = blockIdx.y, per = ((s.longer + kChunk - 1) / kChunk + slices - 1) / slices * kChunk;
  const int l0 = blockIdx.x * per, l1 = min(s.longer, l0 + per);
  gram_of<T>(p, s, g, l0, l1, false, u, share, k);
  double* out = grams + ((int64_t)g * slices + blockIdx.x) * s.r * s.r;
  for (int e = threadIdx.x; e < s.r * s.r; e += kThreads) out[e] = k[e / s.r][e % s.r];
}

// ALONE: a matrix has one workgroup, which computes K itself.
template <typename T, bool ALONE>
__global__ void __launch_bounds__(kThreads) orth_short_kernel(OrthMatrices p, ShortShape s, const double* grams, int slices) {
  __shared__ float u[kShortSide][kChunk + 1];
  __shared__ double share[4][kThreads];
  __shared__ double m0[kShortSide][kPitch], m1[kShortSide][kPitch], m2[kShortSide][kPitch], m3[kShortSide][kPitch];
  __shared__ float pf[kShortSide][kShortSide + 1];
  const int g = blockIdx.y, r = s.r, per = ((s.longer + kChunk - 1) / kChunk + slices - 1) / slices * kChunk;
  const int l0 = blockIdx.x * per, l1 = min(s.longer, l0 + per);
  if (ALONE) {
    gram_of<T>(p, s, g, 0, s.longer, false, u, share, m0);
  } else {
    for (int e = threadIdx.x; e < r * r; e += kThreads) {
      double v = 0.0;
      for (int q = 0; q < slices; ++q) v += grams[((int64_t)g * slices + q) * r * r + e];
      m0[e / r][e % r] = v;
    }
    __syncthreads();
  }
  double squares = 0.0;
  for (int i = 0; i < r; ++i) squares += m0[i][i];
  const double scale = norm_scale(squares, p.eps);
  __syncthreads();
  for (int e = threadIdx.x; e < r * r; e += kThreads) m0[e / r][e % r] *= scale * scale;
  __syncthreads();

  const double a = p.a, b = p.b, c = p.c;
  auto plain = [](double v, int, int) { return v; };
  // A in m0; Q to m1; products over m2; P in m3 (after the first step)
  for (int step = 0; step < p.steps; ++step) {
    short_product(m0, m0, m1, r, [&](double v, int i, int j) { return fma(c, v, fma(b, m0[i][j], i == j ? a : 0.0)); });
    if (step > 0) {
      short_product(m1, m3, m2, r, plain);
      for (int e = threadIdx.x; e < r * r; e += kThreads) m3[e / r][e % r] = m2[e / r][e % r];
    } else {
      for (int e = threadIdx.x; e < r * r; e += kThreads) m3[e / r][e % r] = m1[e / r][e % r];
    }
    __syncthreads();
    if (step + 1 < p.steps) {
      short_product(m1, m0, m2, r, plain);
      short_product(m2, m1, m0, r, plain);
    }
  }
  for (int e = threadIdx.x; e < r * r; e += kThreads) pf[e / r][e % r] = (float)m3[e / r][e % r];
  __syncthreads();

  // P U, a column of 128 per pair of threads, half of the rows each
  constexpr int H = kShortSide / 2;
  T* out = reinterpret_cast<T*>(p.out) + g * p.out_matrix;
  for (int l = l0; l < l1; l += kChunk) {
    const int n = min(kChunk, l1 - l);
    stage<T>(p, s, g, l, n, true, scale, u);
    __syncthreads();
    const int x = threadIdx.x % kChunk, i0 = threadIdx.x / kChunk * H;
    float o[H];
#pragma unroll
    for (int i = 0; i < H; ++i) o[i] = 0.0f;
    if (x < n)
      for (int j = 0; j < r; ++j) {
        const float v = u[j][x];
#pragma unroll
        for (int i = 0; i < H; ++i) o[i] = fmaf(pf[min(i0 + i, r - 1)][j], v, o[i]);
      }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < H; ++i)
      if (i0 + i < r && x < n) u[i0 + i][x] = o[i];
    __syncthreads();
    for (int i = threadIdx.x; i < r * n; i += kThreads) {
      int q, at;
      if (s.tall) { at = i / r; q = i - at * r; } else { q = i / n; at = i - q * n; }
      T* to = out + (s.tall ? (l + at) * p.out_row + q : q * p.out_row + l + at);
      const float v = u[q][at];
      put(to, p.m == nullptr ? v : fmaf(-p.step, v, p.keep * value(*to)));
    }
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

int orth_short_slices(int count, int longer) {
  const int chunks = (longer + kChunk - 1) / kChunk;
  if (chunks <= 8) return 1;
  int slices = (512 + count - 1) / count;
  if (slices > 16) slices = 16;
  if (slices > chunks / 4) slices = chunks / 4;
  return slices < 1 ? 1 : slices;
}

hipError_t launch_orth_short(const OrthMatrices& p, double* grams, int slices, hipStream_t s) {
  const ShortShape shape{p.rows < p.cols ? p.rows : p.cols, p.rows < p.cols ? p.cols : p.rows, p.rows > p.cols};
  const dim3 grid((unsigned)slices, (unsigned)p.count);
  if (slices == 1) {
    if (p.bf16) hipLaunchKernelGGL((orth_short_kernel<uint16_t, true>), grid, dim3(kThreads), 0, s, p, shape, grams, slices);
    else hipLaunchKernelGGL((orth_short_kernel<float, true>), grid, dim3(kThreads), 0, s, p, shape, grams, slices);
    return hipGetLastError();
  }
  if (p.bf16) {
    hipLaunchKernelGGL(orth_short_gram_kernel<uint16_t>, grid, dim3(kThreads), 0, s, p, shape, grams, slices);
    hipLaunchKernelGGL((orth_short_kernel<uint16_t, false>), grid, dim3(kThreads), 0, s, p, shape, grams, slices);
  } else {
    hipLaunchKernelGGL(orth_short_gram_kernel<float>, grid, dim3(kThreads), 0, s, p, shape, grams, slices);
    hipLaunchKernelGGL((orth_short_kernel<float, false>), grid, dim3(kThreads), 0, s, p, shape, grams, slices);
  }
  return hipGetLastError();
}

}  // namespace prsgd
