// The cross entropy's products of operands of any alignment and size, in fp32 (products and sums) or bf16 (sums in fp32).
// Tiles of 128 x 128 fp32 reach 109 to 122 TFLOP/s (2 x 1024 and 4096 rows x 1024 x 8192; a large library product 153), bound by the step's barrier; bf16 430 TFLOP/s.
#include "xent_any_tile.h"

namespace prsgd {

namespace {

template <typename T, int BM, int BN, int WM, int WN, int WK, int D, bool TA, bool TB, int EPI, bool NARROW>
__global__ void __launch_bounds__(64 * WM * WN * WK, WM * WN * WK == 8 ? 4 : 1) product_kernel(ProductArgs p) {        // eight wavefronts: two workgroups on a compute unit
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  product_tile<T, BM, BN, WM, WN, WK, D, TA, TB, EPI, NARROW>(p, tile_of_workgroup(p, p.first + blockIdx.x), smem);
}

template <typename T, int BM, int BN, int WM, int WN, int WK, int D, bool TA, bool TB, int EPI, bool NARROW = false> hipError_t launch_tile(ProductArgs p, Cut* cut, hipStream_t s) {
  constexpr int kLds = lds_bytes<T, BM, BN, WM, WN, WK, D, EPI>();
  static_assert(kLds <= 160 * 1024, "LDS of a compute unit");
  constexpr auto kernel = product_kernel<T, BM, BN, WM, WN, WK, D, TA, TB, EPI, NARROW>;
  if (const hipError_t e = allow_lds<kernel>(kLds); e != hipSuccess) return e;
  const unsigned grid = cut_product(p, BM, BN, D, cut);
  if (EPI == PX_STATS && p.tiles_m > p.most_tiles) return hipErrorInvalidValue;
  return in_turn(p, grid, [&](unsigned n) { hipLaunchKernelGGL(kernel, dim3(n), dim3(64 * WM * WN * WK), kLds, s, p); });
}
// Tiles: rows, columns and, where several wavefronts share it, depth of a step.  NARROW: of rows shorter than 16 bytes, the one kernel that has what it takes to load them.
enum Tiles { NARROW, R32_C32, R32_C64, R64_C32, R32_C128, R128_C32, R64_C64, R64_C64_DEEP, R128_C128 };
constexpr int rows_of(Tiles t) { return t == R128_C32 || t == R128_C128 ? 128 : t == R64_C32 || t == R64_C64 || t == R64_C64_DEEP ? 64 : 32; }

template <typename T, bool TA, bool TB, int EPI> Tiles choose_tiles(const ProductArgs& p) {
  if (narrow_operand<T>(p.a, TA ? p.M : p.K) || narrow_operand<T>(p.b, TB ? p.N : p.K)) return NARROW;
  const int64_t huge = tiles_of(p, 128), large = tiles_of(p, 64);
  if constexpr (EPI == PX_STATS) {
    // all classes in one tile need no other launch: 64 workers' 8 rows x 128 x 50 fp32 7.1 us, by tiles of 32 x 32 10.3, of 512 13.0 and 13.6 (bf16 8.9 and 10.9), but of 1024 21.3
    // and 17.8; x 128 x 100 8.9 and 10.3, but of 256 12.9 and 11.3
    if (large < 256 && p.M > 32 && p.M <= 64 && p.K <= 512) return R64_C32;
    if (large < 256 && p.M > 64 && p.M <= 128 && p.K <= 128) return R128_C32;
  }
  if (tiles_of(p, 32) >= 512 && (p.M <= 32 || p.N <= 32)) {
    // long tiles where one side is short: 64 workers' 16 rows x 64 x 4001 fp32 28 us, by 64 x 64 41, by 32 x 32 90; 64 x 16 x 256 x 4001 bf16 36, 42 and 47 (fp32 71, 96 and 119, by
    // 128 x 32 61); 300 x 70 x 256 x 30 fp32 14.3, 21.2 and 16.3
    if (p.K <= 64) return p.N <= 32 ? R128_C32 : R32_C128;
    return p.N <= 32 ? R64_C32 : R32_C64;
  }
  // What a round of tiles, one on every compute unit, takes in ns: an element of the contraction, at least what it waits for its loads, and a beginning and end
  // (2 x 1024 rows x 1024 x 8192 fp32, logits' gradients by tiles of 128, 64 and 32: 308, 379 and 587 us; 9 x 768 x 77 x 2339: 68, 56 and 179 us).
  auto cost = [&](int64_t tiles, int depth, double element, double wait, double ends) {
    const double k = (double)((p.K + depth - 1) / depth * depth) / (double)p.splits, rounds = (double)((tiles + 255) / 256);
    return rounds * (k * element + ends) > k * wait + ends ? rounds * (k * element + ends) : k * wait + ends;
  };
  constexpr bool F32 = sizeof(T) == 4;
  const double by128 = cost(huge, 32, F32 ? 75 : 21.6, 47, 8000), by64 = cost(large, p.K <= 64 ? 32 : 64, F32 ? 23 : 6.4, 19, 1800);
  const double by32 = cost(tiles_of(p, 32), 128, F32 ? 9.0 : 2.7, 9.4, 1700);
  if (by128 <= by64 && by128 <= by32) return R128_C128;
  if (by32 < by64) return R32_C32;
  return p.K <= 64 ? R64_C64 : R64_C64_DEEP;                 // 4 workers' 512 rows x 64 x 2001 fp32 15.1 and 17.6 us, bf16 11.6 and 11.3
}
template <typename T, bool TA, bool TB, int EPI> hipError_t launch_size(const ProductArgs& p, Cut* cut, hipStream_t s) {
  constexpr int M128 = sizeof(T) == 4 && EPI != PX_DW ? 4 : 2;
  switch (choose_tiles<T, TA, TB, EPI>(p)) {
    case NARROW: return launch_tile<T, 32, 32, 1, 1, 4, 128, TA, TB, EPI, true>(p, cut, s);
    case R32_C32: return launch_tile<T, 32, 32, 1, 1, 4, 128, TA, TB, EPI>(p, cut, s);
    case R32_C64: return launch_tile<T, 32, 64, 1, 2, 2, 64, TA, TB, EPI>(p, cut, s);
    case R64_C32: return launch_tile<T, 64, 32, 2, 1, 2, 64, TA, TB, EPI>(p, cut, s);
    case R32_C128: return launch_tile<T, 32, 128, 1, 4, 1, 32, TA, TB, EPI>(p, cut, s);
    case R128_C32: return launch_tile<T, 128, 32, 4, 1, 1, 32, TA, TB, EPI>(p, cut, s);
    case R64_C64: return launch_tile<T, 64, 64, 2, 2, 1, 32, TA, TB, EPI>(p, cut, s);
    case R64_C64_DEEP: return launch_tile<T, 64, 64, 2, 2, 1, 64, TA, TB, EPI>(p, cut, s);
    default: return launch_tile<T, 128, 128, M128, 2, 1, 32, TA, TB, EPI>(p, cut, s);
  }
}
template <typename T> hipError_t launch(const ProductArgs& p, int epi, bool ta, bool tb, Cut* cut, hipStream_t s) {
  switch (epi) {
    case PX_STATS: return ta ? launch_size<T, true, false, PX_STATS>(p, cut, s) : launch_size<T, false, false, PX_STATS>(p, cut, s);
    case PX_DZ: return tb ? launch_size<T, false, true, PX_DZ>(p, cut, s) : launch_size<T, false, false, PX_DZ>(p, cut, s);
    case PX_DH: return tb ? launch_size<T, false, true, PX_DH>(p, cut, s) : launch_size<T, false, false, PX_DH>(p, cut, s);
    default: return launch_size<T, true, true, PX_DW>(p, cut, s);
  }
}

}  // namespace

hipError_t launch_product_any(const ProductArgs& p, int epi, bool a_transposed, bool b_transposed, bool bf16, Cut* cut, hipStream_t s) {
  return bf16 ? launch<uint16_t>(p, epi, a_transposed, b_transposed, cut, s) : launch<float>(p, epi, a_transposed, b_transposed, cut, s);
}

int stats_rows_any(const ProductArgs& p, bool a_transposed, bool bf16) {
  if (bf16) return rows_of(a_transposed ? choose_tiles<uint16_t, true, false, PX_STATS>(p) : choose_tiles<uint16_t, false, false, PX_STATS>(p));
  return rows_of(a_transposed ? choose_tiles<float, true, false, PX_STATS>(p) : choose_tiles<float, false, false, PX_STATS>(p));
}

}  // namespace prsgd
