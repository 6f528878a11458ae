// Rows whose length is a multiple of nothing, 16 bytes at a time.  The last bytes of a row come in one load that ends where the row does, and are moved into place when
// they are used: elements loaded one by one would each be waited for where they are put together, and a branch between both ways of loading waits for what is on its way.
#pragma once

#include "orth_rows.h"

namespace prsgd {

// Where a piece of V elements is read, n > 0 of which exist from its place on: that many before it ...
constexpr int missing_of(int n, int V) { return n < V ? V - n : 0; }
// ... or, of a row that is shorter than a piece, its element e there.
constexpr int narrow_element(int e, int missing) { return e < missing ? 0 : e - missing; }
// No element outside a row is read, of rows of any width at any place that is a multiple of V: what a piece reads depends on these modulo V, and on whether a whole one
// lies before it.
constexpr bool pieces_stay_in_rows(int V) {
  for (int width = 1; width <= 4 * V; ++width)
    for (int c = 0; c < width; c += V) {
      const int n = width - c, missing = missing_of(n, V);
      if (width >= V && (c - missing < 0 || c - missing + V > width)) return false;
      for (int e = 0; e < V && width < V; ++e)
        if (narrow_element(e, missing) < 0 || c + narrow_element(e, missing) >= width) return false;
    }
  return true;
}
static_assert(pieces_stay_in_rows(4) && pieces_stay_in_rows(8), "pieces of fp32 and bf16");

// 16 bytes of a row from p on, n > 0 elements of which exist; fewer than 16 / ES come to lie at the end, behind what lies before them.  narrow (of all lanes): the
// row as a whole is shorter than that, and is loaded one by one.
template <int ES> __device__ __forceinline__ u32x4_t load_piece(const void* p, int n, bool narrow) {
  constexpr int V = 16 / ES;
  const int missing = missing_of(n, V);
  if (!narrow) return reinterpret_cast<const Packed16<ES>*>(reinterpret_cast<const char*>(p) - missing * ES)->v;
  u32x4_t v = {0, 0, 0, 0};
#pragma unroll
  for (int e = 0; e < V; ++e) {
    const int from = narrow_element(e, missing);
    if constexpr (ES == 4) v[e] = reinterpret_cast<const uint32_t*>(p)[from];
    else v[e / 2] |= (uint32_t)reinterpret_cast<const uint16_t*>(p)[from] << (16 * (e & 1));
  }
  return v;
}
// What load_piece returned of n < 16 / ES elements, with these in front and zeros behind.
template <int ES> __device__ __forceinline__ u32x4_t place_piece(u32x4_t v, int n) {
  const int bytes = (16 / ES - n) * ES;
  if constexpr (ES == 2) {
    const u32x4_t half = {v[0] >> 16 | v[1] << 16, v[1] >> 16 | v[2] << 16, v[2] >> 16 | v[3] << 16, v[3] >> 16};
#pragma unroll
    for (int w = 0; w < 4; ++w) v[w] = (bytes & 2) != 0 ? half[w] : v[w];
  }
  const u32x4_t one = {v[1], v[2], v[3], 0};
#pragma unroll
  for (int w = 0; w < 4; ++w) v[w] = (bytes & 4) != 0 ? one[w] : v[w];
  const u32x4_t two = {v[2], v[3], 0, 0};
#pragma unroll
  for (int w = 0; w < 4; ++w) v[w] = (bytes & 8) != 0 ? two[w] : v[w];
  return v;
}

// Eight elements of a row as they lie in memory, n of which exist; until raw_place has moved them, the last ones of an odd row lie elsewhere.
template <typename T> struct Raw8 { u32x4_t q[sizeof(T) / 2]; };
template <typename T> __device__ __forceinline__ float raw_at(const Raw8<T>& v, int e) {
  if constexpr (sizeof(T) == 4) return __uint_as_float(v.q[e / 4][e % 4]);
  else return __uint_as_float((e & 1) != 0 ? v.q[0][e / 2] & 0xFFFF0000u : v.q[0][e / 2] << 16);
}
// n > 0
template <typename T> __host__ __device__ constexpr bool narrow_row(int width) { return width < 16 / (int)sizeof(T); }
template <typename T> __device__ __forceinline__ void raw_load(Raw8<T>& v, const T* p, int n, bool narrow) {
  constexpr int ES = (int)sizeof(T), V = 16 / ES;
#pragma unroll
  for (int i = 0; i < 8 / V; ++i) {
    if (i == 0) v.q[i] = load_piece<ES>(p, n, narrow);
    // of a second piece that does not exist the first one once more
    else v.q[i] = load_piece<ES>(n > i * V ? p + i * V : p, n > i * V ? n - i * V : n, narrow);
  }
}
template <typename T> __device__ __forceinline__ void raw_place(Raw8<T>& v, int n) {
  constexpr int ES = (int)sizeof(T), V = 16 / ES;
#pragma unroll
  for (int i = 0; i < 8 / V; ++i)
    if (n < (i + 1) * V) v.q[i] = n > i * V ? place_piece<ES>(v.q[i], n - i * V) : (u32x4_t){0, 0, 0, 0};
}

}  // namespace prsgd
