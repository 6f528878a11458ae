// Tiles of the cross entropy's products for operands of any alignment and size: through registers into LDS, [row][contraction] whichever way they lie in memory and twice,
// the next one on its way while the matrix cores take the last.
#pragma once

#include "row_pieces.h"
#include "xent_products.h"

namespace prsgd {

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

}  // namespace prsgd
