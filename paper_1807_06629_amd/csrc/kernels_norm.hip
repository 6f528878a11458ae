// Root-mean-square norm of the workers' rows with the residual's addition, forward (result in the rows' type or in 8 bits with
// a scale per row) and backward.
//   s = x + res,  rstd = 1 / sqrt(mean(s^2) + eps),  y = s rstd w
//   dx = rstd (w dy - s rstd^2 mean(w dy s)) + dsum,  dw = sum over a worker's rows of dy s rstd
// A row is held in the registers of TPR threads, E elements each (fp32 once unpacked), so that every array crosses HBM once and
// the row's one reduction is all that stands between its loads and its stores.  The row maximum of the 8-bit form needs no second
// one: max |y| = rstd max |s w|.  Bound by HBM from a few thousand rows on, by the latency of a launch below:
//   forward, bf16, 65536 rows of 4096 (2.15 GB)   378 us, 5.7 TB/s (a large copy: 4.7);  one row 3.4 us, a call of it 5.9
//   8 bits, bf16, 800 rows of 1000                4.9 us, a call 6.0
//   backward, bf16, 32768 rows of 4096 (1.07 GB)  210 + 5 us, 5.0 TB/s;  fp32, 1024 rows of 1024  5.9 + 2.7 us
#include <algorithm>
#include <type_traits>

#include "prsgd_internal.h"
#include "prsgd_ops_internal.h"

namespace prsgd {

namespace {

typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));

// 16 bytes at any multiple of their elements' size: rows of odd widths start anywhere, and the hardware takes such addresses
typedef unsigned int u32x4_any2_t __attribute__((ext_vector_type(4), aligned(2)));
typedef unsigned int u32x4_any4_t __attribute__((ext_vector_type(4), aligned(4)));
template <typename T> using Piece = std::conditional_t<sizeof(T) == 2, u32x4_any2_t, u32x4_any4_t>;

template <typename T> struct Rows;
template <> struct Rows<float> {
  static constexpr int V = 4;
  __device__ static __forceinline__ float get(u32x4_t v, int e) { return __uint_as_float(v[e]); }
  __device__ static __forceinline__ u32x4_t pack(const float* f) {
    return (u32x4_t){__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])};
  }
};
template <> struct Rows<uint16_t> {
  static constexpr int V = 8;
  __device__ static __forceinline__ float get(u32x4_t v, int e) {
    return __uint_as_float((e & 1) != 0 ? v[e / 2] & 0xFFFF0000u : v[e / 2] << 16);
  }
  __device__ static __forceinline__ u32x4_t pack(const float* f) {
    return (u32x4_t){f32x2_to_bf16x2_rne(f[0], f[1]), f32x2_to_bf16x2_rne(f[2], f[3]), f32x2_to_bf16x2_rne(f[4], f[5]),
                     f32x2_to_bf16x2_rne(f[6], f[7])};
  }
};

// n elements (those at and past n are zero) of the vector at p; the last vector of an odd width takes them one by one
// NT: non-temporal, for rows that the caches cannot hold until somebody reads them again
template <bool NT, typename T> __device__ __forceinline__ u32x4_t load_row(const T* p, int n) {
  constexpr int V = Rows<T>::V;
  if (n >= V) {
    const Piece<T>* q = reinterpret_cast<const Piece<T>*>(p);
    return NT ? __builtin_nontemporal_load(q) : *q;
  }
  u32x4_t v = {0, 0, 0, 0};
#pragma unroll
  for (int e = 0; e < V; ++e)
    if (e < n) {
      if constexpr (sizeof(T) == 4) v[e] = __float_as_uint(p[e]);
      else v[e / 2] |= (uint32_t)p[e] << (16 * (e & 1));
    }
  return v;
}
template <bool NT, typename T> __device__ __forceinline__ void store_row(T* p, int n, u32x4_t v) {
  constexpr int V = Rows<T>::V;
  if (n >= V) {
    Piece<T>* q = reinterpret_cast<Piece<T>*>(p);
    if (NT) __builtin_nontemporal_store((Piece<T>)v, q);
    else *q = v;
    return;
  }
#pragma unroll
  for (int e = 0; e < V; ++e)
    if (e < n) {
      if constexpr (sizeof(T) == 4) p[e] = __uint_as_float(v[e]);
      else p[e] = (uint16_t)(v[e / 2] >> (16 * (e & 1)));
    }
}
template <int V> __device__ __forceinline__ void load_weights(const float* p, int n, float (&w)[V]) {
  if (n >= V) {
#pragma unroll
    for (int e = 0; e < V; e += 4) {
      const u32x4_t v = *reinterpret_cast<const Piece<float>*>(p + e);
#pragma unroll
      for (int i = 0; i < 4; ++i) w[e + i] = __uint_as_float(v[i]);
    }
  } else {
#pragma unroll
    for (int e = 0; e < V; ++e) w[e] = e < n ? p[e] : 0.0f;
  }
}
// four or eight bytes in e4m3 (v_cvt_pk_fp8_f32: two values, nearest even)
template <int V> __device__ __forceinline__ void store_fp8(uint8_t* p, int n, const float* f) {
  struct __attribute__((packed, aligned(1))) Word { uint32_t v; };
  uint32_t u[V / 4];
#pragma unroll
  for (int q = 0; q < V / 4; ++q) {
    int v = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * q], f[4 * q + 1], 0, false);
    v = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * q + 2], f[4 * q + 3], v, true);
    u[q] = (uint32_t)v;
  }
  if (n >= V) {
#pragma unroll
    for (int q = 0; q < V / 4; ++q) reinterpret_cast<Word*>(p + 4 * q)->v = u[q];
    return;
  }
#pragma unroll
  for (int e = 0; e < V; ++e)
    if (e < n) p[e] = (uint8_t)(u[e / 4] >> (8 * (e & 3)));
}

// Sum of a and maximum of m over the TPR threads of a row, in every one of them.  parity: of the call, so that one barrier is enough.
template <int TPR, bool MAX> __device__ __forceinline__ void row_reduce(float& a, float& m, int parity) {
#pragma unroll
  for (int d = 1; d < (TPR < kWave ? TPR : kWave); d <<= 1) {
    a += __shfl_xor(a, d);
    if (MAX) m = fmaxf(m, __shfl_xor(m, d));
  }
  if constexpr (TPR > kWave) {
    constexpr int NW = TPR / kWave;
    __shared__ float part[2][2][NW];
    if ((threadIdx.x & 63) == 0) {
      part[parity][0][threadIdx.x >> 6] = a;
      if (MAX) part[parity][1][threadIdx.x >> 6] = m;
    }
    __syncthreads();
    a = 0.0f;
    m = 0.0f;
#pragma unroll
    for (int i = 0; i < NW; ++i) {
      a += part[parity][0][i];
      if (MAX) m = fmaxf(m, part[parity][1][i]);
    }
  }
}

template <int TPR> constexpr int threads_of() { return TPR > kThreads ? TPR : kThreads; }
constexpr float kFp8Max = 448.0f;
constexpr float kFp8Least = 0x1p-100f;    // a row of zeros has a scale too
constexpr float kLeastSquares = 0x1p-90f;
constexpr float kLeastNormal = 0x1p-126f;

template <typename T, int TPR, int E, bool FP8, bool NT>
__global__ void __launch_bounds__(threads_of<TPR>()) rms_norm_kernel(NormArgs p) {
  constexpr int V = Rows<T>::V, NV = E / V, SLOTS = threads_of<TPR>() / TPR;
  const int slot = threadIdx.x / TPR, t = threadIdx.x % TPR;
  const float inv_width = 1.0f / (float)p.width;
  int parity = 0;
  for (uint64_t row0 = (uint64_t)blockIdx.x * SLOTS; row0 < p.rows; row0 += (uint64_t)gridDim.x * SLOTS, parity ^= 1) {
    const uint32_t row = (uint32_t)row0 + (uint32_t)slot;
    const bool live = row < p.rows;
    const uint32_t g = live ? row / p.rows_per_worker : 0;
    const T* x = reinterpret_cast<const T*>(p.x) + (int64_t)row * p.x_row;
    const T* res = reinterpret_cast<const T*>(p.res) + (int64_t)row * p.res_row;
    const float* w = p.w + (int64_t)g * p.w_row;
    u32x4_t xv[NV], rv[NV];
    float wv[NV][V], s[NV][V];
#pragma unroll
    for (int q = 0; q < NV; ++q) {
      const int c = (q * TPR + t) * V, n = live ? p.width - c : 0;
      xv[q] = rv[q] = (u32x4_t){0, 0, 0, 0};
      if (n > 0) {
        xv[q] = load_row<NT>(x + c, n);
        if (p.res != nullptr) rv[q] = load_row<NT>(res + c, n);
      }
    }
#pragma unroll
    for (int q = 0; q < NV; ++q) {
      const int c = (q * TPR + t) * V;
      load_weights<V>(w + c, live ? p.width - c : 0, wv[q]);
    }
    float a = 0.0f, m = 0.0f;
#pragma unroll
    for (int q = 0; q < NV; ++q)
#pragma unroll
      for (int e = 0; e < V; ++e) {
        s[q][e] = Rows<T>::get(xv[q], e);
        if (p.res != nullptr) s[q][e] += Rows<T>::get(rv[q], e);
        a = fmaf(s[q][e], s[q][e], a);
        if (FP8) m = fmaxf(m, fabsf(s[q][e] * wv[q][e]));
      }
    row_reduce<TPR, FP8>(a, m, parity);
    float rstd = 1.0f / sqrtf(a * inv_width + p.eps), top = m * rstd;
    // Squares past fp32 are summed again at 2^-80 of the row's size, ones that vanish beside an eps that small at 2^80; |y| is taken
    // from normed elements where their own products with w are past fp32 or below its normal numbers.  (All of them zero beside vanishing
    // squares is no matter: rstd is 2^45 at most then, and the least scale that of 2^-100.)
    const bool past = !(a < INFINITY), least = a < kLeastSquares && p.eps < kLeastSquares;
    if (past || least || (FP8 && (!(m < INFINITY) || (m < kLeastNormal && (m > 0.0f || a > 0.0f))))) {
      const float size = past ? 0x1p-80f : least ? 0x1p80f : 1.0f;
      if (past || least) {
        parity ^= 1;
        a = 0.0f;
#pragma unroll
        for (int q = 0; q < NV; ++q)
#pragma unroll
          for (int e = 0; e < V; ++e) a = fmaf(s[q][e] * size, s[q][e] * size, a);
        row_reduce<TPR, false>(a, m, parity);
        rstd = 1.0f / sqrtf(a * inv_width + p.eps * size * size);
      }
      if constexpr (FP8) {
        parity ^= 1;
        float none = top = 0.0f;
#pragma unroll
        for (int q = 0; q < NV; ++q)
#pragma unroll
          for (int e = 0; e < V; ++e) top = fmaxf(top, fabsf(s[q][e] * size * rstd * wv[q][e]));
        row_reduce<TPR, true>(none, top, parity);
        if (!(a < INFINITY)) top = NAN;                    // a row with a NaN or an infinity has no scale
      }
      rstd *= size;
    }
    float shrink = 1.0f;
    if constexpr (FP8) {
      const float scale = (top < kFp8Least ? kFp8Least : top) / kFp8Max;
      shrink = 1.0f / scale;
      if (t == 0 && live) p.stat[row] = scale;
    } else if (p.stat != nullptr && t == 0 && live) {
      p.stat[row] = rstd;
    }
#pragma unroll
    for (int q = 0; q < NV; ++q) {
      const int c = (q * TPR + t) * V, n = live ? p.width - c : 0;
      if (n <= 0) continue;
      if (p.sum != nullptr)
        store_row<NT>(reinterpret_cast<T*>(p.sum) + (int64_t)row * p.sum_row + c, n, Rows<T>::pack(s[q]));
      float y[V];
#pragma unroll
      for (int e = 0; e < V; ++e) y[e] = s[q][e] * rstd * wv[q][e];
      if constexpr (FP8) {                                 // last: rstd / scale may leave fp32 where y / scale does not
#pragma unroll
        for (int e = 0; e < V; ++e) y[e] *= shrink;
      }
      if constexpr (FP8) store_fp8<V>(reinterpret_cast<uint8_t*>(p.y) + (int64_t)row * p.y_row + c, n, y);
      else store_row<NT>(reinterpret_cast<T*>(p.y) + (int64_t)row * p.y_row + c, n, Rows<T>::pack(y));
    }
  }
}

// Backward: a workgroup has a run of one worker's rows and keeps its columns' shares of dw in registers over them.
template <typename T, int TPR, int E, bool NT>
__global__ void __launch_bounds__(threads_of<TPR>()) rms_norm_back_kernel(NormArgs p) {
  constexpr int V = Rows<T>::V, NV = E / V, SLOTS = threads_of<TPR>() / TPR;
  const int slot = threadIdx.x / TPR, t = threadIdx.x % TPR;
  const uint32_t g = blockIdx.x / (uint32_t)p.blocks, b = blockIdx.x % (uint32_t)p.blocks;
  // rows are dealt in whole passes of SLOTS rows
  const uint32_t passes = (p.rows_per_worker + SLOTS - 1) / SLOTS;
  const uint32_t first = (uint32_t)((uint64_t)passes * b / p.blocks) * SLOTS;
  const uint32_t last = min((uint32_t)((uint64_t)passes * (b + 1) / p.blocks) * SLOTS, p.rows_per_worker);
  const float inv_width = 1.0f / (float)p.width;
  float wv[NV][V], acc[NV][V];
#pragma unroll
  for (int q = 0; q < NV; ++q) {
    const int c = (q * TPR + t) * V;
    load_weights<V>(p.w + (int64_t)g * p.w_row + c, p.width - c, wv[q]);
#pragma unroll
    for (int e = 0; e < V; ++e) acc[q][e] = 0.0f;
  }
  int parity = 0;
  for (uint32_t r0 = first; r0 < last; r0 += SLOTS, parity ^= 1) {
    const bool live = r0 + slot < last;
    const int64_t row = (int64_t)g * p.rows_per_worker + r0 + slot;
    const T* dy = reinterpret_cast<const T*>(p.x) + row * p.x_row;
    const T* ds = reinterpret_cast<const T*>(p.res) + row * p.res_row;
    const T* s = reinterpret_cast<const T*>(p.sum) + row * p.sum_row;
    u32x4_t dyv[NV], sv[NV], dsv[NV];
#pragma unroll
    for (int q = 0; q < NV; ++q) {
      const int c = (q * TPR + t) * V, n = live ? p.width - c : 0;
      dyv[q] = sv[q] = dsv[q] = (u32x4_t){0, 0, 0, 0};
      if (n > 0) {
        dyv[q] = load_row<NT>(dy + c, n);
        sv[q] = load_row<NT>(s + c, n);
        if (p.res != nullptr) dsv[q] = load_row<NT>(ds + c, n);
      }
    }
    const float rstd = live ? p.stat[row] : 0.0f;
    float a = 0.0f, none = 0.0f;
#pragma unroll
    for (int q = 0; q < NV; ++q)
#pragma unroll
      for (int e = 0; e < V; ++e) a = fmaf(Rows<T>::get(dyv[q], e) * wv[q][e], Rows<T>::get(sv[q], e) * rstd, a);
    row_reduce<TPR, false>(a, none, parity);
    const float mean = a * inv_width;
#pragma unroll
    for (int q = 0; q < NV; ++q) {
      const int c = (q * TPR + t) * V, n = live ? p.width - c : 0;
      if (n <= 0) continue;
      float dx[V];
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float d = Rows<T>::get(dyv[q], e), sh = Rows<T>::get(sv[q], e) * rstd;
        acc[q][e] = fmaf(d, sh, acc[q][e]);
        dx[e] = rstd * (d * wv[q][e] - sh * mean);
        if (p.res != nullptr) dx[e] += Rows<T>::get(dsv[q], e);
      }
      store_row<NT>(reinterpret_cast<T*>(p.y) + row * p.y_row + c, n, Rows<T>::pack(dx));
    }
  }
  float* out = p.dw + (int64_t)blockIdx.x * p.dw_row;
  if constexpr (SLOTS > 1) {
    // slots are added in ascending order, a column at a time
    constexpr int W = TPR * E;
    __shared__ float part[SLOTS][W];
#pragma unroll
    for (int q = 0; q < NV; ++q)
#pragma unroll
      for (int e = 0; e < V; ++e) part[slot][(q * TPR + t) * V + e] = acc[q][e];
    __syncthreads();
    for (int c = threadIdx.x; c < p.width; c += threads_of<TPR>()) {
      float v = 0.0f;
#pragma unroll
      for (int i = 0; i < SLOTS; ++i) v += part[i][c];
      out[c] = v;
    }
  } else {
#pragma unroll
    for (int q = 0; q < NV; ++q) {
      const int c = (q * TPR + t) * V;
#pragma unroll
      for (int e = 0; e < V; ++e)
        if (c + e < p.width) out[c + e] = acc[q][e];
    }
  }
}

// dw of a worker from its workgroups' shares: a workgroup has 64 columns, its sixteen wavefronts a run of the shares each, added in order.
constexpr int kShareWaves = 16;
__global__ void __launch_bounds__(64 * kShareWaves) norm_dw_kernel(const float* shares, int64_t share_row, int blocks, float* dw,
                                                                   int64_t dw_row, int width) {
  const int lane = threadIdx.x & 63, part = threadIdx.x >> 6, c = blockIdx.x * 64 + lane;
  const float* from = shares + (int64_t)blockIdx.y * blocks * share_row + c;
  float v = 0.0f;
  if (c < width) {
#pragma unroll 8
    for (int b = blocks * part / kShareWaves; b < blocks * (part + 1) / kShareWaves; ++b) v += from[b * share_row];
  }
  __shared__ float sums[kShareWaves][64];
  sums[part][lane] = v;
  __syncthreads();
  if (part == 0 && c < width) {
#pragma unroll
    for (int i = 1; i < kShareWaves; ++i) v += sums[i][lane];
    dw[(int64_t)blockIdx.y * dw_row + c] = v;
  }
}

__global__ void __launch_bounds__(kThreads) norm_dw_zero_kernel(float* dw, int64_t dw_row, int width) {
  const int c = blockIdx.x * kThreads + threadIdx.x;
  if (c < width) dw[(int64_t)blockIdx.y * dw_row + c] = 0.0f;
}

// Threads and elements per thread of a row: 16 elements at most, so that a compute unit has rows enough in flight, and more threads
// with fewer elements where rows are few and one row's latency counts.  512 threads between 4096 and 8192 elements leave fewer of them without
// any than 1024 do (4120 rows of 6581 in fp32: 98 -> 86 us, 8 bits 90 -> 73; 4000 of 6000 in bf16 40 -> 30); fp32 rows from 17 to 64
// elements are read in whole lines by 16 threads (322543 rows of 52: four threads 56 us, sixteen 41).
struct RowShape { int tpr, e; };
RowShape row_shape(int64_t rows, int width, bool bf16) {
  const int least = bf16 ? 8 : 4;
  int tpr = 4;
  while (tpr < 1024 && width > (tpr == 4 && !bf16 ? 4 : 16) * tpr) tpr *= 4;
  while (tpr < 1024 && rows * tpr < 256 * 256 && width > least * tpr) tpr *= 4;
  if (tpr == 1024 && width > 8 * 512 && width <= 16 * 512 && rows >= 256) tpr = 512;
  int e = least;
  while (e * tpr < width) e *= 2;
  return {tpr, e};
}

// shapes that row_shape gives
template <typename T, int TPR, int E> constexpr bool shape_exists() { return E >= Rows<T>::V && !(sizeof(T) == 4 && TPR == 4 && E > 4); }

template <typename T, int TPR, int E> hipError_t launch_forward(const NormArgs& p, bool fp8, hipStream_t s) {
  if constexpr (!shape_exists<T, TPR, E>()) return hipErrorInvalidValue;
  else {
  constexpr int THR = threads_of<TPR>(), SLOTS = THR / TPR;
  const uint64_t blocks = ((uint64_t)p.rows + SLOTS - 1) / SLOTS;
  const dim3 grid((unsigned)(blocks < (1u << 20) ? blocks : (1u << 20)));
  const bool nt = p.streamed;
  if (fp8 && nt) hipLaunchKernelGGL((rms_norm_kernel<T, TPR, E, true, true>), grid, dim3(THR), 0, s, p);
  else if (fp8) hipLaunchKernelGGL((rms_norm_kernel<T, TPR, E, true, false>), grid, dim3(THR), 0, s, p);
  else if (nt) hipLaunchKernelGGL((rms_norm_kernel<T, TPR, E, false, true>), grid, dim3(THR), 0, s, p);
  else hipLaunchKernelGGL((rms_norm_kernel<T, TPR, E, false, false>), grid, dim3(THR), 0, s, p);
  return hipGetLastError();
  }
}
template <typename T, int TPR, int E> hipError_t launch_backward(const NormArgs& p, int workers, hipStream_t s) {
  if constexpr (!shape_exists<T, TPR, E>()) return hipErrorInvalidValue;
  else {
  const dim3 grid((unsigned)workers * (unsigned)p.blocks);
  if (p.streamed) hipLaunchKernelGGL((rms_norm_back_kernel<T, TPR, E, true>), grid, dim3(threads_of<TPR>()), 0, s, p);
  else hipLaunchKernelGGL((rms_norm_back_kernel<T, TPR, E, false>), grid, dim3(threads_of<TPR>()), 0, s, p);
  return hipGetLastError();
  }
}

// f(TPR, E) for a row shape
template <int TPR, typename F> hipError_t with_elements(int e, F&& f) {
  using Tpr = std::integral_constant<int, TPR>;
  switch (e) {
    case 4: return f(Tpr{}, std::integral_constant<int, 4>{});
    case 8: return f(Tpr{}, std::integral_constant<int, 8>{});
    case 16: return f(Tpr{}, std::integral_constant<int, 16>{});
  }
  return hipErrorInvalidValue;
}
template <typename F> hipError_t with_shape(const RowShape& r, F&& f) {
  switch (r.tpr) {
    case 4: return with_elements<4>(r.e, f);
    case 16: return with_elements<16>(r.e, f);
    case 64: return with_elements<64>(r.e, f);
    case 256: return with_elements<256>(r.e, f);
    case 512: return r.e == 16 ? f(std::integral_constant<int, 512>{}, std::integral_constant<int, 16>{}) : hipErrorInvalidValue;
    case 1024: return with_elements<1024>(r.e, f);
  }
  return hipErrorInvalidValue;
}

}  // namespace

// Calls whose four arrays pass twice the last-level cache take them non-temporally: nothing of them is left for the next reader anyway.
// Forward and backward, 65536 rows of 4096 in bf16 386 and 441 us, 384 and 418 so; 16384 rows of 4096 in fp32 191 and 219, 181 and 202.
// What the cache holds is slower so: 8192 rows in bf16 (256 MB) 41 and 55 us, 47 and 63.
static bool streamed_rows(const NormArgs& p, bool bf16) { return (int64_t)p.rows * p.width * (bf16 ? 2 : 4) * 4 > (int64_t)512 << 20; }

hipError_t launch_rms_norm(NormArgs p, bool bf16, bool fp8, hipStream_t s) {
  p.streamed = streamed_rows(p, bf16);
  const RowShape r = row_shape(p.rows, p.width, bf16);
  if (bf16) return with_shape(r, [&](auto tpr, auto e) { return launch_forward<uint16_t, decltype(tpr)::value, decltype(e)::value>(p, fp8, s); });
  return with_shape(r, [&](auto tpr, auto e) { return launch_forward<float, decltype(tpr)::value, decltype(e)::value>(p, fp8, s); });
}

// Four workgroups per compute unit in all, where that leaves eight rows to each: a share of dw is written and read once, 8 bytes per
// column, against 8 (bf16) to 16 per column of a row.  (4000 rows of 8192 in bf16, one worker: 65 us at four rows, 47 at eight.)
// Fewer rows where the device would be left empty otherwise (16 x 64 rows of 1024 in fp32: 64 workgroups 10.8 us, 256 8.5), but not so
// few that the second launch is all that it adds (64 x 8 rows of 128: 5.9 us in one launch, 8.4 in two).
int norm_back_blocks(int workers, int64_t rows_per_worker, int width, bool bf16) {
  if (rows_per_worker <= 0) return 0;
  const RowShape r = row_shape((int64_t)workers * rows_per_worker, width, bf16);
  const int slots = r.tpr >= kThreads ? 1 : kThreads / r.tpr;
  const int64_t passes = (rows_per_worker + slots - 1) / slots;
  if (passes <= 4) return 1;
  const int64_t most = std::min<int64_t>(passes, std::max<int64_t>((rows_per_worker + 7) / 8, (256 + workers - 1) / workers));
  return (int)std::min<int64_t>(most, (1024 + workers - 1) / workers);
}

size_t norm_back_share_floats(int workers, int64_t rows_per_worker, int width, bool bf16) {
  const int blocks = norm_back_blocks(workers, rows_per_worker, width, bf16);
  return blocks <= 1 ? 0 : (size_t)workers * blocks * (((size_t)width + 63) / 64 * 64);
}

hipError_t launch_rms_norm_backward(NormArgs p, float* shares, int workers, bool bf16, hipStream_t s) {
  if (p.rows_per_worker == 0) {
    hipLaunchKernelGGL(norm_dw_zero_kernel, dim3((p.width + kThreads - 1) / kThreads, workers), dim3(kThreads), 0, s, p.dw, p.dw_row, p.width);
    return hipGetLastError();
  }
  p.streamed = streamed_rows(p, bf16);
  float* dw = p.dw;
  const int64_t dw_row = p.dw_row;
  p.blocks = norm_back_blocks(workers, p.rows_per_worker, p.width, bf16);
  if (p.blocks > 1) {
    p.dw = shares;
    p.dw_row = (p.width + 63) / 64 * 64;
  }
  const RowShape r = row_shape(p.rows, p.width, bf16);
  hipError_t e = bf16 ? with_shape(r, [&](auto tpr, auto el) { return launch_backward<uint16_t, decltype(tpr)::value, decltype(el)::value>(p, workers, s); })
                      : with_shape(r, [&](auto tpr, auto el) { return launch_backward<float, decltype(tpr)::value, decltype(el)::value>(p, workers, s); });
  if (e != hipSuccess || p.blocks <= 1) return e;
  hipLaunchKernelGGL(norm_dw_kernel, dim3((p.width + 63) / 64, workers), dim3(64 * kShareWaves), 0, s, shares, p.dw_row, p.blocks, dw, dw_row, p.width);
  return hipGetLastError();
}

}  // namespace prsgd
