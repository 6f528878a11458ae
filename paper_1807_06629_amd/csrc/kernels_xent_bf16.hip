// The cross entropy's products of aligned bf16 operands: tiles go straight from memory to LDS, 64 deep, and an operand whose contraction index is not the
// contiguous one is read out of LDS as its transpose (ds_read_b64_tr_b16).  What lies past an operand is requested as copies of what lies in it: past its
// rows it is never stored; past the contraction, and in rows without a label, a tile is cleared before it is read.
// Tiles of 256 x 256 reach 1.13 to 1.16 PFLOP/s (2 x 4096 rows x 2048 x 32768, all three products; a large library product 1.22).  Products of some hundred tiles of 64 x 64 wait for
// L2: 12 TB/s out of it for the logits of 8 x 128 rows x 4096 x 1000 in 21 us (in four parts of 128 x 128 tiles 18).
#include "xent_products.h"

namespace prsgd {

namespace {

constexpr int kDepth = 64, kRowBytes = 2 * kDepth;

// A tile of an operand, requested by NW wavefronts.  LDS has 64 banks, and the 256 bytes that 16 lanes read at a time have to lie on different ones: a tile
// cannot be padded on its way, so pieces of a row are exchanged.
//   contraction contiguous: [ROWS][64], 16-byte chunk q of row r at q ^ ((r / 2) mod 8)
//   transposed: [64][ROWS], 32-byte unit u of contraction row c at u ^ unit_xor(c), for reads that transpose
template <int ROWS> __device__ __forceinline__ int unit_xor(int c) { return ROWS == 64 ? c & 2 : (c & 3) << 1; }
template <int ROWS, int NW, bool TRANS> struct Requests {
  static constexpr int NPT = ROWS * kRowBytes / 1024 / NW;
  static_assert(ROWS * kRowBytes % (1024 * NW) == 0, "a tile splits evenly over the wavefronts");
  uint32_t off[NPT];
  // rows, depth: of the operand from the tile's first element on; in the contiguous direction it has that many rounded up to eight
  __device__ __forceinline__ void set(int ld, int rows, int depth, int wave, int lane) {
#pragma unroll
    for (int q = 0; q < NPT; ++q) {
      const int chunk = (q * NW + wave) * 64 + lane;
      if constexpr (TRANS) {
        constexpr int CH = ROWS / 8;
        const int c = chunk / CH, pos = chunk % CH, from = ((((pos >> 1) ^ unit_xor<ROWS>(c)) << 1) | (pos & 1)) * 8;
        off[q] = ((uint32_t)min(c, depth - 1) * (uint32_t)ld + (uint32_t)min(from, (rows + 7) / 8 * 8 - 8)) * 2u;
      } else {
        const int r = chunk / 8, from = ((chunk % 8) ^ ((r >> 1) & 7)) * 8;
        off[q] = ((uint32_t)min(r, rows - 1) * (uint32_t)ld + (uint32_t)min(from, (depth + 7) / 8 * 8 - 8)) * 2u;
      }
    }
  }
  // Zeros in the contraction elements of the tile that take no part (bits of the 64): whole LDS rows of a transposed one, of the other whole pieces of
  // every row, from the contraction's end on.
  __device__ static __forceinline__ void clear(unsigned char* tile, uint64_t bits, int tid) {
#pragma unroll
    for (int i = 0; i < NPT; ++i) {
      const int chunk = i * NW * 64 + tid;
      bool part;
      if constexpr (TRANS) part = (bits >> (chunk / (ROWS / 8)) & 1) != 0;
      else part = (bits >> (((chunk % 8) ^ ((chunk / 8 >> 1) & 7)) * 8) & 1) != 0;
      if (!part) *reinterpret_cast<u32x4_t*>(tile + chunk * 16) = (u32x4_t){0, 0, 0, 0};
    }
  }
};

template <int N> __device__ __forceinline__ void wait_requests() {
  static_assert(N <= 63, "vmcnt");
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" :: "n"(N) : "memory");
}

// Operands of 32-row blocks: lane (r = lane % 32, kb = lane / 32) holds contraction elements 8 kb .. 8 kb + 7 of row r.  Where a lane reads depends on the
// slice (or, transposed, on the block's lowest bits) through an exchange, on the rest through a constant.
template <int ROWS, bool TRANS> struct Fragments {
  int at[4];
  __device__ __forceinline__ void set(int first_block, int lane) {
    if constexpr (TRANS) {
      // of every 16 lanes, lane r gives the address of four elements M[r], and lane i gets M[4 j + i / 4][i % 4], j = 0..3
      const int g = lane >> 4, r = lane & 15, c = 8 * (g >> 1) + (r >> 2);
#pragma unroll
      for (int x = 0; x < 4; ++x) at[x] = c * ROWS * 2 + ((2 * (first_block + x) + (g & 1)) ^ unit_xor<ROWS>(r >> 2)) * 32 + 8 * (r & 3);
    } else {
#pragma unroll
      for (int x = 0; x < 4; ++x) at[x] = (first_block * 32 + (lane & 31)) * kRowBytes + (((2 * x + (lane >> 5)) ^ ((lane >> 1) & 7)) << 4);
    }
  }
  __device__ __forceinline__ bf16x8_t read(const unsigned char* tile, int block, int kk) const {
    if constexpr (TRANS) {
      typedef __attribute__((__vector_size__(4 * sizeof(__bf16)))) __bf16 bf16x4_t;
      typedef __attribute__((address_space(3))) bf16x4_t* lds_bf16x4_ptr;
      const unsigned char* p = tile + at[block % 4] + block / 4 * 256 + kk * 16 * ROWS * 2;
      const bf16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4_ptr)(p));
      const bf16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4_ptr)(p + 4 * ROWS * 2));
      return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    } else {
      return __builtin_bit_cast(bf16x8_t, *reinterpret_cast<const u32x4_t*>(tile + at[kk] + block * 32 * kRowBytes));
    }
  }
};
template <int BM, int BN, int WM, int WN, int S, int EPI> constexpr int lds_bytes() {
  constexpr int stages = S * (BM + BN) * kRowBytes, epilogue = epilogue_lds_bytes<BM, BN, WM, WN, EPI>();
  return stages > epilogue ? stages : epilogue;
}

// WM x WN wavefronts, S tiles in LDS.
template <int BM, int BN, int WM, int WN, int S, bool TA, bool TB, int EPI>
__device__ __forceinline__ void product_bf16_tile(const ProductArgs& p, const TilePosition place_of, unsigned char* smem) {
  constexpr int NW = WM * WN, TM = BM / WM / 32, TN = BN / WN / 32, KK = 4, STAGE = (BM + BN) * kRowBytes, READS = TM + TN;
  using ReqA = Requests<BM, NW, TA>;
  using ReqB = Requests<BN, NW, TB>;
  constexpr int PER = ReqA::NPT + ReqB::NPT;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave / WN, wn = wave % WN;
  const int g = place_of.g, m0 = place_of.ti * BM, n0 = place_of.tj * BN, step0 = place_of.split * p.split_steps;
  const int depth = min(p.K - step0 * kDepth, p.split_steps * kDepth);

  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)smem;
  const int64_t a_step = (int64_t)kDepth * (TA ? p.a.ld : 1), b_step = (int64_t)kDepth * (TB ? p.b.ld : 1);
  const uint16_t* a = reinterpret_cast<const uint16_t*>(p.a.p) + g * p.a.gs + (int64_t)m0 * (TA ? 1 : p.a.ld) + step0 * a_step;
  const uint16_t* b = reinterpret_cast<const uint16_t*>(p.b.p) + g * p.b.gs + (int64_t)n0 * (TB ? 1 : p.b.ld) + step0 * b_step;
  const int lda = (int)p.a.ld, ldb = (int)p.b.ld, n_k = (depth + kDepth - 1) / kDepth, tail = depth - (n_k - 1) * kDepth;
  ReqA ra;
  ReqB rb;
  ra.set(lda, p.M - m0, n_k == 1 ? tail : kDepth, wave, lane);
  rb.set(ldb, p.N - n0, n_k == 1 ? tail : kDepth, wave, lane);
  auto request = [&](int t, int place, int first, int last) __attribute__((always_inline)) {       // place: t mod S
    const uint32_t stage = lds0 + (uint32_t)place * STAGE;
    if (first == 0 && t == n_k - 1 && tail != kDepth) {
      ra.set(lda, p.M - m0, tail, wave, lane);
      rb.set(ldb, p.N - n0, tail, wave, lane);
    }
#pragma unroll
    for (int q = first; q < last; ++q) {
      if (q < ReqA::NPT) load_to_lds(a + t * a_step, ra.off[q < ReqA::NPT ? q : 0], stage + (uint32_t)(q * NW + wave) * 1024u);
      else load_to_lds(b + t * b_step, rb.off[q < ReqA::NPT ? 0 : q - ReqA::NPT], stage + BM * kRowBytes + (uint32_t)((q - ReqA::NPT) * NW + wave) * 1024u);
    }
  };
  // contraction elements of tile t that take part
  const uint64_t* real = reinterpret_cast<const uint64_t*>(p.real + g * real_words(p.rows)) + step0;
  auto bits_of = [&](int t) __attribute__((always_inline)) -> uint64_t {
    if constexpr (EPI == PX_DW) return ((const __attribute__((address_space(4))) uint64_t*)real)[t];
    return t == n_k - 1 && tail != kDepth ? (1ull << tail) - 1 : ~0ull;
  };
  auto clear_rest = [&](unsigned char* tile, uint64_t bits) __attribute__((always_inline)) {
    if (bits == ~0ull) return;
    ReqA::clear(tile, bits, tid);
    ReqB::clear(tile + BM * kRowBytes, bits, tid);
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
  };
  bf16x8_t fa[2][TM], fb[2][TN];
  Fragments<BM, TA> rows;
  Fragments<BN, TB> cols;
  rows.set(wm * TM, lane);
  cols.set(wn * TN, lane);
  // fragment q of slice kk
  auto load = [&](const unsigned char* tile, int kk, int set, int q) __attribute__((always_inline)) {
    if (q < TM) fa[set][q < TM ? q : 0] = rows.read(tile, q, kk);
    else fb[set][q < TM ? 0 : q - TM] = cols.read(tile + BM * kRowBytes, q - TM, kk);
  };
  f32x16_t acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;

  // Tile t + 1 is met before the last slice of tile t is multiplied; from there on every fragment of tile t has been read, and its stage takes tile t + S.
  // Each row of a slice's products is followed by its share of the next slice's fragments and of the requests.
#pragma unroll
  for (int t = 0; t < S; ++t)
    if (t < n_k) request(t, t, 0, PER);
  if (n_k >= S) wait_requests<(S - 1) * PER>(); else wait_requests<0>();
  asm volatile("s_barrier" ::: "memory");
  clear_rest(smem, bits_of(0));
#pragma unroll
  for (int q = 0; q < READS; ++q) load(smem, 0, 0, q);
  int place = 0;
  auto step = [&](int t, auto whole_) __attribute__((always_inline)) {
    constexpr bool WHOLE = decltype(whole_)::value;        // tile t + S exists
    const int behind = place + 1 == S ? 0 : place + 1;
    const unsigned char* here = smem + place * STAGE;
    unsigned char* next = smem + behind * STAGE;
    const uint64_t bits = (EPI == PX_DW || !WHOLE) && t + 1 < n_k ? bits_of(t + 1) : ~0ull;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
      const int set = kk & 1;
      const bool last = kk == KK - 1;
      if (last) {
        if (WHOLE || t + S - 1 < n_k) wait_requests<(S - 2) * PER>(); else wait_requests<0>();
        asm volatile("s_barrier" ::: "memory");
        clear_rest(next, bits);
      }
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        if (!last || WHOLE || t + 1 < n_k) {
#pragma unroll
          for (int q = i * READS / TM; q < (i + 1) * READS / TM; ++q) load(last ? next : here, last ? 0 : kk + 1, set ^ 1, q);
        }
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa[set][i], fb[set][j], acc[i][j], 0, 0, 0);
        if (last && (WHOLE || t + S < n_k)) request(t + S, place, i * PER / TM, (i + 1) * PER / TM);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    place = behind;
  };
  int t = 0;
  for (; t + S < n_k; ++t) step(t, std::true_type{});
  for (; t < n_k; ++t) step(t, std::false_type{});
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
  product_epilogue<uint16_t, EPI, BM, BN, WM, WN, 1>(p, acc, place_of, m0, n0, wm, wn, lane, true, smem);
}

template <int BM, int BN, int WM, int WN, int S, bool TA, bool TB, int EPI>
__global__ void __launch_bounds__(64 * WM * WN, 2) product_bf16_kernel(const ProductArgs p) {
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  product_bf16_tile<BM, BN, WM, WN, S, TA, TB, EPI>(p, tile_of_workgroup(p, p.first + blockIdx.x), smem);
}
// dh by the first workgroups, dW by the others
template <bool CF> __global__ void __launch_bounds__(256, 2) pair_bf16_kernel(const ProductArgs dh, const ProductArgs dw, int first_dw) {
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  if ((int)blockIdx.x < first_dw) product_bf16_tile<64, 64, 2, 2, 3, false, CF, PX_DH>(dh, tile_of_workgroup(dh, blockIdx.x), smem);
  else product_bf16_tile<64, 64, 2, 2, 3, true, true, PX_DW>(dw, tile_of_workgroup(dw, blockIdx.x - first_dw), smem);
}
template <bool CF> hipError_t launch_pair(ProductArgs dh, ProductArgs dw, hipStream_t s) {
  constexpr int kLds = lds_bytes<64, 64, 2, 2, 3, PX_DH>();
  constexpr auto kernel = pair_bf16_kernel<CF>;
  if (const hipError_t e = allow_lds<kernel>(kLds); e != hipSuccess) return e;
  Cut cut;
  const unsigned n_dh = cut_product(dh, 64, 64, kDepth, &cut), n_dw = cut_product(dw, 64, 64, kDepth, &cut);
  hipLaunchKernelGGL(kernel, dim3(n_dh + n_dw), dim3(256), kLds, s, dh, dw, (int)n_dh);
  return hipGetLastError();
}

template <int BM, int BN, int WM, int WN, int S, bool TA, bool TB, int EPI> hipError_t launch_tile(ProductArgs p, Cut* cut, hipStream_t s) {
  static_assert(S >= 2, "a step's tile and the next one");
  constexpr int kLds = lds_bytes<BM, BN, WM, WN, S, EPI>();
  static_assert(kLds <= 160 * 1024, "LDS of a compute unit");
  constexpr auto kernel = product_bf16_kernel<BM, BN, WM, WN, S, TA, TB, EPI>;
  if (const hipError_t e = allow_lds<kernel>(kLds); e != hipSuccess) return e;
  const unsigned grid = cut_product(p, BM, BN, kDepth, cut);
  if (EPI == PX_STATS && p.tiles_m > p.most_tiles) return hipErrorInvalidValue;
  return in_turn(p, grid, [&](unsigned n) { hipLaunchKernelGGL(kernel, dim3(n), dim3(64 * WM * WN), kLds, s, p); });
}

// 256 square, 128 by eight or four wavefronts, 64.
enum Tiles { BY_256, BY_128_EIGHT, BY_128_FOUR, BY_64 };
Tiles choose_tiles(const ProductArgs& p) {
  // Time of a launch in units of a 64 x 64 tile's products: tiles per compute unit times their size over their efficiency.  Of tiles that a compute unit has
  // several of in hand, parts of a round count as such; of 256 x 256 tiles whole rounds.  The efficiencies are fitted: logits by 256, 128 (eight wavefronts), 128 (four) and 64, the
  // rule's first, of 2 x 4096 rows x 2048 x 32768 977, 1304, 1123 and 1594 us, 8 x 512 x 64 x 4096 19, 28, 21 and 28; by 128 (eight), 256, 128 (four) and 64 of 8 x 256 x 2048 x 2048
  // 25, 52, 34 and 34; by 128 (four), 256, 128 (eight) and 64 of 16 x 512 x 1024 x 1024 26, 36, 29 and 34; by 64, 256, 128 (eight) and 128 (four) of 8 x 128 x 4096 x 1000 24, 84, 34 and 48,
  // 4 x 256 x 512 x 2048 12, 26, 14 and 15.  Of 14 such sizes the rule took the best one or one within 1 %.
  auto cost = [](int64_t n, int b, double efficiency) { return (n < 256 ? 1.0 : (double)n / 256.0) * (b / 64) * (b / 64) / efficiency; };
  const int64_t n_middle = tiles_of(p, 128), n_huge = (tiles_of(p, 256) + 255) / 256 * 256;
  const double middle = cost(n_middle, 128, n_middle > 256 ? 0.9 : 1.34), small = cost(tiles_of(p, 64), 64, 0.68), huge = cost(n_huge, 256, 1.2);
  if (huge <= middle && huge <= small) return BY_256;
  if (middle > small) return BY_64;
  return n_middle <= 256 ? BY_128_EIGHT : BY_128_FOUR;
}
template <bool TA, bool TB, int EPI> hipError_t launch(const ProductArgs& p, Cut* cut, hipStream_t s) {
  switch (choose_tiles(p)) {
    case BY_256: return launch_tile<256, 256, 4, 2, 2, TA, TB, EPI>(p, cut, s);
    case BY_128_EIGHT: return launch_tile<128, 128, 4, 2, 3, TA, TB, EPI>(p, cut, s);
    case BY_128_FOUR: return launch_tile<128, 128, 2, 2, 2, TA, TB, EPI>(p, cut, s);
    default: return launch_tile<64, 64, 2, 2, 3, TA, TB, EPI>(p, cut, s);
  }
}

bool operand_aligned(const Operand& o, int64_t contiguous, int64_t other, int groups) {
  return (uintptr_t)o.p % 16 == 0 && o.ld % 8 == 0 && (groups == 1 || o.gs % 8 == 0) && contiguous % 8 == 0 && contiguous > 0 && o.ld < (1 << 21) && other > 0;
}

}  // namespace

bool product_aligned(const ProductArgs& p, bool a_transposed, bool b_transposed) {
  auto whole = [](const Operand& o, int n) { return o.padded ? (n + 7) / 8 * 8 : n; };
  return operand_aligned(p.a, whole(p.a, a_transposed ? p.M : p.K), a_transposed ? p.K : p.M, p.groups) &&
         operand_aligned(p.b, whole(p.b, b_transposed ? p.N : p.K), b_transposed ? p.K : p.N, p.groups);
}

int stats_rows_bf16(const ProductArgs& p) {
  const Tiles t = choose_tiles(p);
  return t == BY_256 ? 256 : t == BY_64 ? 64 : 128;
}
hipError_t launch_pair_bf16(const ProductArgs& dh, const ProductArgs& dw, bool classes_first, hipStream_t s) {
  return classes_first ? launch_pair<true>(dh, dw, s) : launch_pair<false>(dh, dw, s);
}
hipError_t launch_product_bf16(const ProductArgs& p, int epi, bool a_transposed, bool b_transposed, Cut* cut, hipStream_t s) {
  switch (epi) {
    case PX_STATS: return a_transposed ? launch<true, false, PX_STATS>(p, cut, s) : launch<false, false, PX_STATS>(p, cut, s);
    case PX_DZ: return b_transposed ? launch<false, true, PX_DZ>(p, cut, s) : launch<false, false, PX_DZ>(p, cut, s);
    case PX_DH: return b_transposed ? launch<false, true, PX_DH>(p, cut, s) : launch<false, false, PX_DH>(p, cut, s);
    default: return launch<true, true, PX_DW>(p, cut, s);
  }
}

}  // namespace prsgd
