// Products of the cross entropy's gradients that share a launch, where it is launches that take the time: all three of a worker by one workgroup, or dh and dW, which
// need nothing of each other, by workgroups of either.
#include "xent_any_tile.h"

namespace prsgd {

namespace {

// All of a worker's products one after another.  (The arguments of all three do not fit the scalar registers: 14 to 34 of these are kept in lanes of vector registers, and 36 bytes a
// lane in scratch.)
template <typename T, bool CF> constexpr int small_lds_bytes() {
  constexpr int dz = lds_bytes<T, 32, 32, 1, 1, 4, 128, PX_DZ>(), wide = lds_bytes<T, 32, 128, 1, 4, 1, 32, PX_DH>(), high = lds_bytes<T, 128, 32, 4, 1, 1, 32, PX_DW>();
  return std::max(dz, std::max(wide, high));
}
template <typename T, bool CF> __global__ void __launch_bounds__(kThreads) small_gradients_kernel(ProductArgs dz, ProductArgs dh, ProductArgs dw) {
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  const int g = blockIdx.x;
  for (int i = 0; i < dz.tiles_m * dz.tiles_n; ++i) {
    product_tile<T, 32, 32, 1, 1, 4, 128, false, !CF, PX_DZ>(dz, {g, i / dz.tiles_n, i % dz.tiles_n, 0}, smem);
    __syncthreads();
  }
  for (int i = 0; i < dh.tiles_m * dh.tiles_n; ++i) {
    product_tile<T, 32, 128, 1, 4, 1, 32, false, CF, PX_DH>(dh, {g, i / dh.tiles_n, i % dh.tiles_n, 0}, smem);
    __syncthreads();
  }
  for (int i = 0; i < dw.tiles_m * dw.tiles_n; ++i) {
    product_tile<T, CF ? 32 : 128, CF ? 128 : 32, CF ? 1 : 4, CF ? 4 : 1, 1, 32, true, true, PX_DW>(dw, {g, i / dw.tiles_n, i % dw.tiles_n, 0}, smem);
    __syncthreads();
  }
}
template <typename T, bool CF> hipError_t launch_small(ProductArgs& dz, ProductArgs& dh, ProductArgs& dw, hipStream_t s) {
  constexpr int kLds = small_lds_bytes<T, CF>();
  constexpr auto kernel = small_gradients_kernel<T, CF>;
  if (const hipError_t e = allow_lds<kernel>(kLds); e != hipSuccess) return e;
  Cut cut;
  cut_product(dz, 32, 32, 128, &cut);
  cut_product(dh, 32, 128, 32, &cut);
  cut_product(dw, CF ? 32 : 128, CF ? 128 : 32, 32, &cut);
  hipLaunchKernelGGL(kernel, dim3((unsigned)dz.groups), dim3(kThreads), kLds, s, dz, dh, dw);
  return hipGetLastError();
}

// dh by the first workgroups, dW by the others; tiles of 64 x 64 or (H32, W32) of 32 x 32.
template <typename T, bool CF, bool H32, bool W32> constexpr int pair_lds_bytes() {
  constexpr int dh = H32 ? lds_bytes<T, 32, 32, 1, 1, 4, 128, PX_DH>() : lds_bytes<T, 64, 64, 2, 2, 1, 64, PX_DH>();
  constexpr int dw = W32 ? lds_bytes<T, 32, 32, 1, 1, 4, 128, PX_DW>() : lds_bytes<T, 64, 64, 2, 2, 1, 64, PX_DW>();
  return std::max(dh, dw);
}
template <typename T, bool CF, bool H32, bool W32> __global__ void __launch_bounds__(kThreads) pair_kernel(ProductArgs dh, ProductArgs dw, int first_dw) {
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  if ((int)blockIdx.x < first_dw) {
    const TilePosition at = tile_of_workgroup(dh, blockIdx.x);
    if constexpr (H32) product_tile<T, 32, 32, 1, 1, 4, 128, false, CF, PX_DH>(dh, at, smem);
    else product_tile<T, 64, 64, 2, 2, 1, 64, false, CF, PX_DH>(dh, at, smem);
  } else {
    const TilePosition at = tile_of_workgroup(dw, blockIdx.x - first_dw);
    if constexpr (W32) product_tile<T, 32, 32, 1, 1, 4, 128, true, true, PX_DW>(dw, at, smem);
    else product_tile<T, 64, 64, 2, 2, 1, 64, true, true, PX_DW>(dw, at, smem);
  }
}
template <typename T, bool CF, bool H32, bool W32> hipError_t launch_both(ProductArgs dh, ProductArgs dw, hipStream_t s) {
  constexpr int kLds = pair_lds_bytes<T, CF, H32, W32>();
  constexpr auto kernel = pair_kernel<T, CF, H32, W32>;
  if (const hipError_t e = allow_lds<kernel>(kLds); e != hipSuccess) return e;
  Cut cut;
  const unsigned n_dh = H32 ? cut_product(dh, 32, 32, 128, &cut) : cut_product(dh, 64, 64, 64, &cut);
  const unsigned n_dw = W32 ? cut_product(dw, 32, 32, 128, &cut) : cut_product(dw, 64, 64, 64, &cut);
  hipLaunchKernelGGL(kernel, dim3(n_dh + n_dw), dim3(kThreads), kLds, s, dh, dw, (int)n_dh);
  return hipGetLastError();
}
// tiles of 32 x 32 where there are fewer than one of 64 x 64 for every compute unit
template <typename T, bool CF> hipError_t launch_both_of(const ProductArgs& dh, const ProductArgs& dw, hipStream_t s) {
  const bool h32 = tiles_of(dh, 64) < 256, w32 = tiles_of(dw, 64) < 256;
  if (h32) return w32 ? launch_both<T, CF, true, true>(dh, dw, s) : launch_both<T, CF, true, false>(dh, dw, s);
  return w32 ? launch_both<T, CF, false, true>(dh, dw, s) : launch_both<T, CF, false, false>(dh, dw, s);
}

// A step takes a workgroup 1.3 us to 2 us, a launch 4 to 6 us: 64 workers' 8 rows x 128 x 10 fp32 (6 steps) 17.8 us as three launches, 12.7 us as one; 2 workers'
// 3 x 370 x 6 (16 steps) 20.0 and 24.1 us.
constexpr int64_t kSmallSteps = 8;

// Both products' tiles of 64 x 64 that are few enough to be worth a common launch: gradients of 4 workers' 1115 rows x 112 x 474 bf16 25.2 -> 18.9 us, of 32 x 2 x 40 x 157 fp32
// 20.1 -> 15.0 us.
constexpr int64_t kPairTiles = 1024;

}  // namespace

bool small_gradients(int64_t rows, int width, int classes, bool bf16) {
  auto t = [](int64_t n, int b) { return (n + b - 1) / b; };
  const int64_t r = t(rows, 32), c = t(classes, 32), w = t(width, 128);
  // steps of the contraction and a tile's beginning and end
  const int least = bf16 ? 8 : 4;          // rows of 16 bytes
  return rows > 0 && width >= least && classes >= least && r * c * (1 + w) + r * w * (1 + c) + w * c * (1 + r) <= kSmallSteps;
}
hipError_t launch_small_gradients(ProductArgs dz, ProductArgs dh, ProductArgs dw, bool classes_first, bool bf16, hipStream_t s) {
  if (bf16) return classes_first ? launch_small<uint16_t, true>(dz, dh, dw, s) : launch_small<uint16_t, false>(dz, dh, dw, s);
  return classes_first ? launch_small<float, true>(dz, dh, dw, s) : launch_small<float, false>(dz, dh, dw, s);
}
bool pair_gradients(const ProductArgs& dh, const ProductArgs& dw, int classes, int width, bool bf16) {
  const int least = bf16 ? 8 : 4;          // rows of 16 bytes
  return dh.M > 0 && dh.splits == 1 && dw.splits == 1 && width >= least && classes >= least && tiles_of(dh, 64) + tiles_of(dw, 64) <= kPairTiles;
}
hipError_t launch_pair_any(const ProductArgs& dh, const ProductArgs& dw, bool classes_first, bool bf16, hipStream_t s) {
  if (bf16) return classes_first ? launch_both_of<uint16_t, true>(dh, dw, s) : launch_both_of<uint16_t, false>(dh, dw, s);
  return classes_first ? launch_both_of<float, true>(dh, dw, s) : launch_both_of<float, false>(dh, dw, s);
}

}  // namespace prsgd
