// Dropout with the residual's addition: y = res + keep x / (1 - p).  The mask is never stored: eight elements of a row share the four
// words that Philox4x32-10 makes of (block of the row set, step, layer) under the seed, 16 bits each, and an element is dropped if its
// 16 bits are below round(65536 p).  (32 bits an element would take twice the products: at 20 of 32 x 32 -> 64 bits per call of the
// generator that is more time than the rows take to pass through HBM; as it is, 65536 x 4096 bf16 with the residual take 297 us, 5.4 TB/s.)  A residual or a dropped
// element's place takes nothing of x, also where x is no number.
#include <algorithm>

#include "orth_rows.h"
#include "prsgd_token_internal.h"

namespace prsgd {

namespace {

// lanes_log2: lanes that share a row, eight elements of it each at a time
template <typename T> __global__ void __launch_bounds__(kThreads) dropout_kernel(DropoutArgs p, int lanes_log2) {
  const uint32_t per_row = (uint32_t)(p.width + 7) / 8, lanes = 1u << lanes_log2, slots = kThreads >> lanes_log2;
  const uint64_t step = p.step_at != nullptr ? (uint64_t)*p.step_at : p.step;
  const float scale = 65536.0f / (65536.0f - (float)p.dropped);
  for (int64_t row = (int64_t)blockIdx.x * slots + (threadIdx.x >> lanes_log2); row < p.rows; row += (int64_t)gridDim.x * slots)
    for (uint32_t q = threadIdx.x & (lanes - 1); q < per_row; q += lanes) {
      const uint64_t b = (uint64_t)row * per_row + q;
      const int c = (int)q * 8, n = p.width - c;
      float x[8], y[8];
      load8(reinterpret_cast<const T*>(p.x) + row * p.x_row + c, n, x);
      if (p.res != nullptr) load8(reinterpret_cast<const T*>(p.res) + row * p.res_row + c, n, y);
      uint32_t word[4];
      philox4x32_10((uint32_t)b, (uint32_t)step, (uint32_t)(step >> 32), (uint32_t)(b >> 32) + (0x80000000u | p.layer << 16),
                    (uint32_t)p.seed, (uint32_t)(p.seed >> 32), word);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const bool keep = (word[e / 2] >> (16 * (e & 1)) & 0xFFFFu) >= p.dropped;
        const float t = x[e] * scale;
        y[e] = p.res == nullptr ? (keep ? t : 0.0f) : keep ? y[e] + t : y[e];
      }
      store8(reinterpret_cast<T*>(p.y) + row * p.y_row + c, n, y);
    }
}

}  // namespace

hipError_t launch_dropout(const DropoutArgs& p, bool bf16, hipStream_t s) {
  const int lanes_log2 = lanes_for_row(p.width), slots = kThreads >> lanes_log2;
  const unsigned grid = (unsigned)std::min<int64_t>((p.rows + slots - 1) / slots, 256 * 64);
  if (bf16) hipLaunchKernelGGL(dropout_kernel<uint16_t>, dim3(grid), dim3(kThreads), 0, s, p, lanes_log2);
  else hipLaunchKernelGGL(dropout_kernel<float>, dim3(grid), dim3(kThreads), 0, s, p, lanes_log2);
  return hipGetLastError();
}

}  // namespace prsgd
