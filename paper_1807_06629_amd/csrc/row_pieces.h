// The ends of rows whose length is a multiple of nothing.  16 bytes that end where the row does take one load, and are moved into place when they
// are used: elements loaded one by one would each be waited for where they are put together.
#pragma once

#include "orth_rows.h"

namespace prsgd {

// Of the 16 bytes from p on, n elements exist, 0 < n < 16 / ES: they come to lie at the end.  first: start of the buffer; the elements of a row's first piece
// that has nothing in front of it are loaded one by one.
template <int ES> __device__ __forceinline__ u32x4_t load_end(const void* p, int n, const void* first) {
  constexpr int V = 16 / ES;
  const char* from = reinterpret_cast<const char*>(p) - (V - n) * ES;
  u32x4_t v = {0, 0, 0, 0};
  if (from >= reinterpret_cast<const char*>(first)) {
    v = reinterpret_cast<const Packed16<ES>*>(from)->v;
  } else {
    for (int e = 0; e < n; ++e) {
      const int at = V - n + e;
      uint32_t x;
      if constexpr (ES == 4) x = reinterpret_cast<const uint32_t*>(p)[e];
      else x = (uint32_t)reinterpret_cast<const uint16_t*>(p)[e] << (16 * (at & 1));
#pragma unroll
      for (int w = 0; w < 4; ++w) v[w] |= at * ES / 4 == w ? x : 0;
    }
  }
  return v;
}
// What load_end returned, with its n elements in front and zeros behind.
template <int ES> __device__ __forceinline__ u32x4_t place_end(u32x4_t v, int n) {
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

}  // namespace prsgd
