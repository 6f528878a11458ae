// Eight elements of a row of the caller's matrices at a time, at any alignment of their own type, for the kernels of the orthogonalised updates.
#pragma once

#include "prsgd_internal.h"
#include "prsgd_ops_internal.h"

namespace prsgd {

typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));
template <int ES> struct __attribute__((packed, aligned(ES))) Packed16 { u32x4_t v; };

// n: elements from p on that exist (the others read as zeros and are not written); the end of an odd row is taken one by one
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
    for (int e = 0; e < 8; ++e) {
      if constexpr (sizeof(T) == 4) v[e] = e < n ? p[e] : 0.0f;
      else v[e] = e < n ? bf16_to_f32(p[e]) : 0.0f;
    }
  }
}
template <typename T> __device__ __forceinline__ void store8(T* p, int n, const float (&v)[8]) {
  if constexpr (sizeof(T) == 4) {
    if (n >= 8) {
      reinterpret_cast<Packed16<4>*>(p)->v = (u32x4_t){__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
      reinterpret_cast<Packed16<4>*>(p + 4)->v = (u32x4_t){__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7])};
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e < n) p[e] = v[e];
    }
  } else {
    const u32x4_t w = {f32x2_to_bf16x2_rne(v[0], v[1]), f32x2_to_bf16x2_rne(v[2], v[3]), f32x2_to_bf16x2_rne(v[4], v[5]), f32x2_to_bf16x2_rne(v[6], v[7])};
    if (n >= 8) {
      reinterpret_cast<Packed16<2>*>(p)->v = w;
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e < n) p[e] = (uint16_t)(w[e / 2] >> (16 * (e & 1)));
    }
  }
}

// U at row `row`, columns c.. of matrix g; M <- mu M + G unless an earlier launch (`stepped`) has moved it on.
template <typename T> __device__ __forceinline__ void update8(const OrthMatrices& p, int g, int row, int c, int n, bool stepped, float (&u)[8]) {
  load8(reinterpret_cast<const T*>(p.g) + g * p.g_matrix + row * p.g_row + c, n, u);
  if (p.m == nullptr) return;
  float* at = p.m + g * p.m_matrix + row * p.m_row + c;
  float m[8];
  load8(at, n, m);
  if (!stepped) {
#pragma unroll
    for (int e = 0; e < 8; ++e) m[e] = fmaf(p.mu, m[e], u[e]);
    store8(at, n, m);
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) u[e] = fmaf(p.m_part, m[e], p.g_part * u[e]);
}

// The result, or the parameters' update with it, at element `at` of the caller's matrices.
template <typename T> __device__ __forceinline__ void result8(const OrthMatrices& p, int64_t at, int n, const float (&v)[8]) {
  T* out = reinterpret_cast<T*>(p.out) + at;
  if (p.m == nullptr) {
    store8(out, n, v);
    return;
  }
  float x[8];
  load8(out, n, x);
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = fmaf(-p.step, v[e], p.keep * x[e]);
  store8(out, n, x);
}

}  // namespace prsgd
