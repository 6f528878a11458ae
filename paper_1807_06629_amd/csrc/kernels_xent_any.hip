// The cross entropy's products of operands of any alignment and size, in fp32 (products and sums) or bf16 (sums in fp32): tiles pass through registers into
// LDS, [row][contraction] whichever way they lie in memory and twice, the next one on its way while the matrix cores take the last.
// Tiles of 128 x 128 fp32 reach 90 to 105 TFLOP/s (a large library product 153), bound by the step's barrier; bf16 430 TFLOP/s.
#include "row_pieces.h"
#include "xent_products.h"

namespace prsgd {

namespace {

template <typename T> using Tag = std::conditional_t<kIsBf16<T>, TBF16, TF32>;

// An operand's tiles, D deep, rows padded by 16 bytes.
template <typename T_, int ROWS, bool TRANS_, int D, int THREADS_> struct Stage {
  using T = T_;
  static constexpr bool TRANS = TRANS_;
  static constexpr int THREADS = THREADS_;
  static constexpr int ES = (int)sizeof(T), V = 16 / ES, LD = D * ES + 16, BYTES = ROWS * LD;
  // transposed: a thread has a block of 16 bytes of rows by BK contraction elements (fp32 4 x 4, bf16 8 x 2)
  static constexpr int BK = TRANS ? (ES == 4 ? 4 : 2) : 1;
  static constexpr int UNITS = ROWS * D / V / BK, NPT = (UNITS + THREADS - 1) / THREADS;
  static __device__ __forceinline__ int row_of(int u) { return TRANS ? u % (ROWS / V) * V : u / (D / V); }
  static __device__ __forceinline__ int depth_of(int u) { return TRANS ? u / (ROWS / V) * BK : u % (D / V) * V; }
  u32x4_t reg[NPT][BK];
  uint32_t part[NPT];                    // of 32 elements of the contraction, this thread's among them, those that take part (MASKED)
  // rows, depth: what is left of the operand from the tile's first element on; NARROW: rows as they lie in memory may be shorter than 16 bytes; at: the tile's
  // first element of the contraction, in `words` of 32
  template <bool NARROW, bool MASKED, typename P>
  __device__ __forceinline__ void load(P& places, int64_t ld, int rows, int depth, bool narrow, const uint32_t* words, int at, int last_word) {
#pragma unroll
    for (int q = 0; q < NPT; ++q) {
      const int u = q * THREADS + (int)threadIdx.x, r = row_of(u), c = depth_of(u);
      // (written by this launch, where a workgroup makes all of a worker's products; past the last word any, as no element is loaded there)
      if constexpr (MASKED) part[q] = __hip_atomic_load(const_cast<uint32_t*>(words) + min((at + c) / 32, last_word), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
#pragma unroll
      for (int k = 0; k < BK; ++k) reg[q][k] = (u32x4_t){0, 0, 0, 0};
      if (UNITS % THREADS != 0 && u >= UNITS) continue;
      if constexpr (TRANS) {
#pragma unroll
        for (int k = 0; k < BK; ++k)
          if (c + k < depth && r < rows) reg[q][k] = load_piece<ES>(places.at[q] + k * ld, rows - r, NARROW && narrow);
      } else {
        if (r < rows && c < depth) reg[q][0] = load_piece<ES>(places.at[q], depth - c, NARROW && narrow);
      }
      places.at[q] += TRANS ? D * ld : D;
    }
  }
  // rows, depth: as they were loaded
  template <bool MASKED> __device__ __forceinline__ void store(unsigned char* tile, int rows, int depth) {
#pragma unroll
    for (int q = 0; q < NPT; ++q) {
      const int u = q * THREADS + (int)threadIdx.x, r = row_of(u), c = depth_of(u);
      if (UNITS % THREADS != 0 && u >= UNITS) continue;
      const int n = TRANS ? rows - r : depth - c;
      if (n > 0 && n < V) {
#pragma unroll
        for (int k = 0; k < BK; ++k) reg[q][k] = place_piece<ES>(reg[q][k], n);
      }
      if constexpr (TRANS) {
        u32x4_t v[BK];
        const uint32_t bits = MASKED ? part[q] >> c % 32 : ~0u;
#pragma unroll
        for (int k = 0; k < BK; ++k)
#pragma unroll
          for (int e = 0; e < 4; ++e) v[k][e] = (bits >> k & 1) != 0 ? reg[q][k][e] : 0;
#pragma unroll
        for (int e = 0; e < V; ++e) {
          unsigned char* to = tile + (r + e) * LD + c * ES;
          if constexpr (ES == 4) {
            *reinterpret_cast<u32x4_t*>(to) = (u32x4_t){v[0][e], v[1][e], v[2][e], v[3][e]};
          } else {
            const uint32_t lo = v[0][e / 2] >> (16 * (e & 1)) & 0xFFFFu, hi = v[1][e / 2] >> (16 * (e & 1)) << 16;
            *reinterpret_cast<uint32_t*>(to) = lo | hi;
          }
        }
      } else {
        *reinterpret_cast<u32x4_t*>(tile + r * LD + c * ES) = reg[q][0];
      }
    }
  }
  __device__ static __forceinline__ Frag<Tag<T>> frag(const unsigned char* tile, int block, int kk, int lane) {
    Frag<Tag<T>> f;
    const u32x4_t v = *reinterpret_cast<const u32x4_t*>(tile + (block * 32 + (lane & 31)) * LD + (2 * kk + (lane >> 5)) * 16);
    f.v = __builtin_bit_cast(decltype(f.v), v);
    return f;
  }
};

template <typename T> __host__ __device__ constexpr bool narrow_operand(const Operand& o, int contiguous) { return !o.padded && narrow_row<T>(contiguous); }

// Where a thread's pieces of the next tile lie.
template <typename S> struct Places {
  const typename S::T* at[S::NPT];
  __device__ __forceinline__ void set(const typename S::T* base, int64_t ld) {
#pragma unroll
    for (int q = 0; q < S::NPT; ++q) {
      const int u = q * S::THREADS + (int)threadIdx.x, r = S::row_of(u), c = S::depth_of(u);
      at[q] = base + (S::TRANS ? (int64_t)c * ld + r : (int64_t)r * ld + c);
    }
  }
};

// WM x WN wavefronts, WK of them at each place, which share out a tile's depth and join their sums at the end.
template <typename T, int BM, int BN, int WM, int WN, int WK, int D, int EPI> constexpr int lds_bytes() {
  constexpr int stages = 2 * (BM + BN) * (D * (int)sizeof(T) + 16), join = (WK - 1) * BM * BN * 4;
  constexpr int epilogue = epilogue_lds_bytes<BM, BN, WM, WN, EPI>(), most = stages > join ? stages : join;
  return most > epilogue ? most : epilogue;
}
template <typename T, int BM, int BN, int WM, int WN, int WK, int D, bool TA, bool TB, int EPI, bool NARROW = false>
__device__ __forceinline__ void product_tile(const ProductArgs& p, TilePosition at, unsigned char* smem) {
  constexpr int TM = BM / WM / 32, TN = BN / WN / 32, KK = D * (int)sizeof(T) / 32 / WK, THREADS = 64 * WM * WN * WK;
  static_assert(D * (int)sizeof(T) % (32 * WK) == 0, "a tile's depth splits evenly");
  constexpr int AHEAD = WK == 4 && !NARROW ? 2 : 1;                   // small tiles, which are few: nothing else covers what they wait for
  constexpr bool MASKED = EPI == PX_DW;
  static_assert(!MASKED || D % 32 == 0, "words of 32 rows");
  using A = Stage<T, BM, TA, D, THREADS>;
  using B = Stage<T, BN, TB, D, THREADS>;
  constexpr int STAGE = A::BYTES + B::BYTES;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wk = wave / (WM * WN), wm = wave / WN % WM, wn = wave % WN;
  const int g = at.g, m0 = at.ti * BM, n0 = at.tj * BN, k0 = at.split * p.split_steps * D, depth = min(p.K - k0, p.split_steps * D);
  const T* a = reinterpret_cast<const T*>(p.a.p) + g * p.a.gs + (int64_t)m0 * (TA ? 1 : p.a.ld) + (int64_t)k0 * (TA ? p.a.ld : 1);
  const T* b = reinterpret_cast<const T*>(p.b.p) + g * p.b.gs + (int64_t)n0 * (TB ? 1 : p.b.ld) + (int64_t)k0 * (TB ? p.b.ld : 1);
  const uint32_t* real = p.real + g * real_words(p.rows);
  f32x16_t acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;
  // AHEAD tiles on their way
  A ra[AHEAD];
  B rb[AHEAD];
  const int n_k = (depth + D - 1) / D;
  // what is left of the operands from the tile on; zeros behind the end of a padded one are loaded with the rest
  auto whole = [](const Operand& o, int n) { return o.padded ? (n + 7) / 8 * 8 : n; };
  const int a_rows = (TA ? whole(p.a, p.M) : p.M) - m0, b_rows = (TB ? whole(p.b, p.N) : p.N) - n0;
  const int a_depth = TA ? depth : whole(p.a, depth), b_depth = TB ? depth : whole(p.b, depth);
  Places<A> pa;
  Places<B> pb;
  pa.set(a, p.a.ld);
  pb.set(b, p.b.ld);
  auto load = [&](int t, auto set_) __attribute__((always_inline)) {         // 0, 1, 2 ..
    constexpr int set = decltype(set_)::value;
    if (t >= n_k) return;
    const int last_word = (int)real_words(p.rows) - 1;
    ra[set].template load<NARROW, MASKED>(pa, p.a.ld, a_rows, a_depth - t * D, narrow_operand<T>(p.a, TA ? p.M : p.K), real, k0 + t * D, last_word);
    rb[set].template load<NARROW, MASKED>(pb, p.b.ld, b_rows, b_depth - t * D, narrow_operand<T>(p.b, TB ? p.N : p.K), real, k0 + t * D, last_word);
  };
  auto store = [&](int t, auto set_) __attribute__((always_inline)) {
    constexpr int set = decltype(set_)::value;
    if (t >= n_k) return;
    unsigned char* stage = smem + (t & 1) * STAGE;
    ra[set].template store<MASKED>(stage, a_rows, a_depth - t * D);
    rb[set].template store<MASKED>(stage + A::BYTES, b_rows, b_depth - t * D);
  };
  using First = std::integral_constant<int, 0>;
  using Second = std::integral_constant<int, AHEAD - 1>;
  load(0, First{});
  if constexpr (AHEAD == 2) load(1, Second{});
  store(0, First{});
  if constexpr (AHEAD == 2) load(2, First{});
  __syncthreads();
  // tile t + 1 is in set (t + 1) mod AHEAD
  auto step = [&](int t, auto next_) __attribute__((always_inline)) {
    const unsigned char* here = smem + (t & 1) * STAGE;
    if constexpr (AHEAD == 1) load(t + 1, next_);
#pragma unroll
    for (int k = 0; k < KK; ++k) {
      const int kk = wk * KK + k;
      Frag<Tag<T>> fa[TM], fb[TN];
#pragma unroll
      for (int i = 0; i < TM; ++i) fa[i] = A::frag(here, wm * TM + i, kk, lane);
#pragma unroll
      for (int j = 0; j < TN; ++j) fb[j] = B::frag(here + A::BYTES, wn * TN + j, kk, lane);
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = mma(fa[i], fb[j], acc[i][j]);
    }
    store(t + 1, next_);
    if constexpr (AHEAD == 2) load(t + 3, next_);
    __syncthreads();
  };
  for (int t = 0; t < n_k; t += 2) {
    step(t, Second{});
    if (t + 1 < n_k) step(t + 1, First{});
  }
  if constexpr (WK > 1) {
    float* sums = reinterpret_cast<float*>(smem);            // [WK - 1][WM * WN][TM * TN][16][64]
    constexpr int BLOCK = 16 * kWave, PLACE = TM * TN * BLOCK;
    if (wk > 0) {
      float* to = sums + ((wk - 1) * WM * WN + wm * WN + wn) * PLACE + lane;
#pragma unroll
      for (int i = 0; i < TM * TN; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) to[i * BLOCK + e * kWave] = acc[i / TN][i % TN][e];
    }
    __syncthreads();
    if (wk == 0) {
#pragma unroll
      for (int w = 0; w < WK - 1; ++w)
#pragma unroll
        for (int i = 0; i < TM * TN; ++i)
#pragma unroll
          for (int e = 0; e < 16; ++e) acc[i / TN][i % TN][e] += sums[(w * WM * WN + wm * WN + wn) * PLACE + i * BLOCK + e * kWave + lane];
    }
    __syncthreads();
  }
  product_epilogue<T, EPI, BM, BN, WM, WN, WK>(p, acc, at, m0, n0, wm, wn, lane, wk == 0, smem);
}
template <typename T, int BM, int BN, int WM, int WN, int WK, int D, bool TA, bool TB, int EPI, bool NARROW>
__global__ void __launch_bounds__(64 * WM * WN * WK, WM * WN * WK == 8 ? 4 : 1) product_kernel(ProductArgs p) {        // eight wavefronts: two workgroups on a compute unit
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  product_tile<T, BM, BN, WM, WN, WK, D, TA, TB, EPI, NARROW>(p, tile_of_workgroup(p), smem);
}

// All of a worker's products one after another.
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

template <typename T, int BM, int BN, int WM, int WN, int WK, int D, bool TA, bool TB, int EPI, bool NARROW = false> hipError_t launch_tile(ProductArgs p, Cut* cut, hipStream_t s) {
  constexpr int kLds = lds_bytes<T, BM, BN, WM, WN, WK, D, EPI>();
  static_assert(kLds <= 160 * 1024, "LDS of a compute unit");
  constexpr auto kernel = product_kernel<T, BM, BN, WM, WN, WK, D, TA, TB, EPI, NARROW>;
  if (const hipError_t e = allow_lds<kernel>(kLds); e != hipSuccess) return e;
  const unsigned grid = cut_product(p, BM, BN, D, cut);
  hipLaunchKernelGGL(kernel, dim3(grid), dim3(64 * WM * WN * WK), kLds, s, p);
  return hipGetLastError();
}
template <typename T, bool TA, bool TB, int EPI> hipError_t launch_size(const ProductArgs& p, Cut* cut, hipStream_t s) {
  // rows shorter than 16 bytes: one kernel, which alone has what it takes to load them
  if (narrow_operand<T>(p.a, TA ? p.M : p.K) || narrow_operand<T>(p.b, TB ? p.N : p.K)) return launch_tile<T, 32, 32, 1, 1, 4, 128, TA, TB, EPI, true>(p, cut, s);
  constexpr int M128 = sizeof(T) == 4 && EPI != PX_DW ? 4 : 2;
  const int64_t huge = tiles_of(p, 128), large = tiles_of(p, 64);
  if constexpr (EPI == PX_STATS) {
    // all classes in one tile need no other launch
    if (large < 256 && p.M > 32 && p.M <= 64 && p.K <= 512) return launch_tile<T, 64, 32, 2, 1, 2, 64, TA, TB, EPI>(p, cut, s);
    if (large < 256 && p.M > 64 && p.M <= 128 && p.K <= 128) return launch_tile<T, 128, 32, 4, 1, 1, 32, TA, TB, EPI>(p, cut, s);
  }
  if (tiles_of(p, 32) >= 512 && (p.M <= 32 || p.N <= 32)) {
    if (p.K <= 64) return p.N <= 32 ? launch_tile<T, 128, 32, 4, 1, 1, 32, TA, TB, EPI>(p, cut, s) : launch_tile<T, 32, 128, 1, 4, 1, 32, TA, TB, EPI>(p, cut, s);
    return p.N <= 32 ? launch_tile<T, 64, 32, 2, 1, 2, 64, TA, TB, EPI>(p, cut, s) : launch_tile<T, 32, 64, 1, 2, 2, 64, TA, TB, EPI>(p, cut, s);
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
  if (by128 <= by64 && by128 <= by32) return launch_tile<T, 128, 128, M128, 2, 1, 32, TA, TB, EPI>(p, cut, s);
  if (by32 < by64) return launch_tile<T, 32, 32, 1, 1, 4, 128, TA, TB, EPI>(p, cut, s);
  if (p.K <= 64) return launch_tile<T, 64, 64, 2, 2, 1, 32, TA, TB, EPI>(p, cut, s);
  return launch_tile<T, 64, 64, 2, 2, 1, 64, TA, TB, EPI>(p, cut, s);
}
template <typename T> hipError_t launch(const ProductArgs& p, int epi, bool ta, bool tb, Cut* cut, hipStream_t s) {
  switch (epi) {
    case PX_STATS: return ta ? launch_size<T, true, false, PX_STATS>(p, cut, s) : launch_size<T, false, false, PX_STATS>(p, cut, s);
    case PX_DZ: return tb ? launch_size<T, false, true, PX_DZ>(p, cut, s) : launch_size<T, false, false, PX_DZ>(p, cut, s);
    case PX_DH: return tb ? launch_size<T, false, true, PX_DH>(p, cut, s) : launch_size<T, false, false, PX_DH>(p, cut, s);
    default: return launch_size<T, true, true, PX_DW>(p, cut, s);
  }
}

// A step takes a workgroup 1.3 us to 2 us, a launch 4 to 6 us: 64 workers' 8 rows x 128 x 10 fp32 (6 steps) 17.8 us as three launches, 12.7 us as one; 2 workers'
// 3 x 370 x 6 (16 steps) 20.0 and 24.1 us.
constexpr int64_t kSmallSteps = 8;

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
hipError_t launch_product_any(const ProductArgs& p, int epi, bool a_transposed, bool b_transposed, bool bf16, Cut* cut, hipStream_t s) {
  return bf16 ? launch<uint16_t>(p, epi, a_transposed, b_transposed, cut, s) : launch<float>(p, epi, a_transposed, b_transposed, cut, s);
}

}  // namespace prsgd
