// The cross entropy's products of operands of any alignment and size, in fp32 (products and sums) or bf16 (sums in fp32): tiles pass through registers into
// LDS, [row][contraction] whichever way they lie in memory, 32 deep and twice, the next one on its way while the matrix cores take the last.
#include "xent_products.h"

namespace prsgd {

namespace {

template <typename T> using Tag = std::conditional_t<kIsBf16<T>, TBF16, TF32>;

// n elements from p on (0 .. 16 bytes' worth)
template <typename T> __device__ __forceinline__ u32x4_t load16(const T* p, int n) {
  constexpr int V = 16 / (int)sizeof(T);
  u32x4_t v = {0, 0, 0, 0};
  if (n >= V) return reinterpret_cast<const Packed16<(int)sizeof(T)>*>(p)->v;
#pragma unroll
  for (int e = 0; e < V; ++e)
    if (e < n) {
      if constexpr (sizeof(T) == 4) v[e] = __float_as_uint(p[e]);
      else v[e / 2] |= (uint32_t)p[e] << (16 * (e & 1));
    }
  return v;
}

// ---- products of operands of any alignment and size --------------------------------------------
// Tiles pass through registers into LDS, [row][contraction] either way: 32 deep, rows padded by 16 bytes.  Fragments are those of the grouped products.
constexpr int kDepth = 32;
template <typename T, int ROWS, bool TRANS> struct Stage {
  static constexpr int ES = (int)sizeof(T), V = 16 / ES, LD = kDepth * ES + 16, BYTES = ROWS * LD;
  // transposed: a thread has a block of 4 / ES contraction elements ... of 16 bytes of rows
  static constexpr int BK = TRANS ? 4 / ES * (ES == 4 ? 4 : 1) : 1;            // fp32 4 x 4, bf16 2 x 8
  static constexpr int UNITS = TRANS ? kDepth / BK * (ROWS / V) : ROWS * kDepth / V;
  static constexpr int NPT = (UNITS + kThreads - 1) / kThreads;
  u32x4_t reg[NPT][BK];
  // rows, depth: what is left of the operand from the tile's first element on; labels: of the contraction index (PX_DW)
  __device__ __forceinline__ void load(const T* base, int64_t ld, int rows, int depth, const int32_t* labels, int classes) {
#pragma unroll
    for (int q = 0; q < NPT; ++q) {
      const int u = q * kThreads + (int)threadIdx.x;
#pragma unroll
      for (int k = 0; k < BK; ++k) reg[q][k] = (u32x4_t){0, 0, 0, 0};
      if (UNITS % kThreads != 0 && u >= UNITS) continue;
      if constexpr (TRANS) {
        const int c = u % (kDepth / BK) * BK, r = u / (kDepth / BK) * V;
#pragma unroll
        for (int k = 0; k < BK; ++k)
          if (c + k < depth && r < rows && (labels == nullptr || (unsigned)labels[c + k] < (unsigned)classes))
            reg[q][k] = load16(base + (int64_t)(c + k) * ld + r, rows - r);
      } else {
        const int r = u / (kDepth / V), c = u % (kDepth / V) * V;
        if (r < rows && c < depth) reg[q][0] = load16(base + (int64_t)r * ld + c, depth - c);
      }
    }
  }
  __device__ __forceinline__ void store(unsigned char* tile) const {
#pragma unroll
    for (int q = 0; q < NPT; ++q) {
      const int u = q * kThreads + (int)threadIdx.x;
      if (UNITS % kThreads != 0 && u >= UNITS) continue;
      if constexpr (TRANS) {
        const int c = u % (kDepth / BK) * BK, r = u / (kDepth / BK) * V;
#pragma unroll
        for (int e = 0; e < V; ++e) {
          unsigned char* to = tile + (r + e) * LD + c * ES;
          if constexpr (ES == 4) {
            *reinterpret_cast<u32x4_t*>(to) = (u32x4_t){reg[q][0][e], reg[q][1][e], reg[q][2][e], reg[q][3][e]};
          } else {
            const uint32_t lo = reg[q][0][e / 2] >> (16 * (e & 1)) & 0xFFFFu, hi = reg[q][1][e / 2] >> (16 * (e & 1)) << 16;
            *reinterpret_cast<uint32_t*>(to) = lo | hi;
          }
        }
      } else {
        const int r = u / (kDepth / V), c = u % (kDepth / V) * V;
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

constexpr int product_stage_bytes(int bm, int bn, int es) { return (bm + bn) * (kDepth * es + 16); }

template <typename T, int BM, int BN, bool TA, bool TB, int EPI> __global__ void __launch_bounds__(kThreads) product_kernel(ProductArgs p) {
  constexpr int WM = 2, WN = 2, TM = BM / WM / 32, TN = BN / WN / 32, KK = kDepth * (int)sizeof(T) / 32;
  using A = Stage<T, BM, TA>;
  using B = Stage<T, BN, TB>;
  constexpr int STAGE = product_stage_bytes(BM, BN, (int)sizeof(T));
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave / WN, wn = wave % WN;
  const TilePosition at = tile_of_workgroup(p);
  const int g = at.g, m0 = at.ti * BM, n0 = at.tj * BN;
  const T* a = reinterpret_cast<const T*>(p.a.p) + g * p.a.gs + (int64_t)m0 * (TA ? 1 : p.a.ld);
  const T* b = reinterpret_cast<const T*>(p.b.p) + g * p.b.gs + (int64_t)n0 * (TB ? 1 : p.b.ld);
  const int64_t step_a = (int64_t)kDepth * (TA ? p.a.ld : 1), step_b = (int64_t)kDepth * (TB ? p.b.ld : 1);
  const int32_t* labels = EPI == PX_DW ? p.labels + g * p.rows : nullptr;
  f32x16_t acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;
  A ra;
  B rb;
  const int n_k = (p.K + kDepth - 1) / kDepth;
  auto load = [&](int t) __attribute__((always_inline)) {
    const int32_t* of = EPI == PX_DW ? labels + t * kDepth : nullptr;
    ra.load(a + t * step_a, p.a.ld, p.M - m0, p.K - t * kDepth, of, p.classes);
    rb.load(b + t * step_b, p.b.ld, p.N - n0, p.K - t * kDepth, of, p.classes);
  };
  load(0);
  ra.store(smem);
  rb.store(smem + A::BYTES);
  __syncthreads();
  for (int t = 0; t < n_k; ++t) {
    const unsigned char* here = smem + (t & 1) * STAGE;
    if (t + 1 < n_k) load(t + 1);
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
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
    if (t + 1 < n_k) {
      unsigned char* next = smem + ((t + 1) & 1) * STAGE;
      ra.store(next);
      rb.store(next + A::BYTES);
    }
    __syncthreads();
  }
  product_epilogue<T, EPI, BM, BN, WM, WN>(p, acc, g, m0, n0, at.ti, wm, wn, lane, smem);
}

template <typename T, int BM, int BN, bool TA, bool TB, int EPI> hipError_t launch_tile(ProductArgs p, int* tiles_m, hipStream_t s) {
  constexpr int kStages = 2 * product_stage_bytes(BM, BN, (int)sizeof(T)), kEpilogue = epilogue_lds_bytes<BM, BN, 2, 2, EPI>();
  constexpr int kLds = kStages > kEpilogue ? kStages : kEpilogue;
  static_assert(kLds <= 160 * 1024, "LDS of a compute unit");
  constexpr auto kernel = product_kernel<T, BM, BN, TA, TB, EPI>;
  if (const hipError_t e = allow_lds<kernel>(kLds); e != hipSuccess) return e;
  *tiles_m = p.tiles_m = (p.M + BM - 1) / BM;
  p.tiles_n = (p.N + BN - 1) / BN;
  hipLaunchKernelGGL(kernel, dim3((unsigned)p.tiles_m * (unsigned)p.tiles_n * (unsigned)p.groups), dim3(kThreads), kLds, s, p);
  return hipGetLastError();
}
template <typename T> hipError_t launch(const ProductArgs& p, int epi, bool ta, bool tb, int* tiles_m, hipStream_t s) {
  constexpr int B = 128;
  switch (epi) {
    case PX_STATS: return ta ? launch_tile<T, B, B, true, false, PX_STATS>(p, tiles_m, s) : launch_tile<T, B, B, false, false, PX_STATS>(p, tiles_m, s);
    case PX_DZ: return tb ? launch_tile<T, B, B, false, true, PX_DZ>(p, tiles_m, s) : launch_tile<T, B, B, false, false, PX_DZ>(p, tiles_m, s);
    case PX_DH: return tb ? launch_tile<T, B, B, false, true, PX_DH>(p, tiles_m, s) : launch_tile<T, B, B, false, false, PX_DH>(p, tiles_m, s);
    default: return launch_tile<T, B, B, true, true, PX_DW>(p, tiles_m, s);
  }
}

}  // namespace

hipError_t launch_product_any(const ProductArgs& p, int epi, bool a_transposed, bool b_transposed, bool bf16, int* tiles_m, hipStream_t s) {
  return bf16 ? launch<uint16_t>(p, epi, a_transposed, b_transposed, tiles_m, s) : launch<float>(p, epi, a_transposed, b_transposed, tiles_m, s);
}

}  // namespace prsgd
