// Products between the matrices of the Newton-Schulz steps, in half precision on the matrix cores with fp32 sums: X X^T and A A, whose
// operands' rows are contiguous along the contraction, and B X, whose second operand is read out of LDS as its transpose.  Symmetric results
// compute the tiles on and below the diagonal and write the others as transposes.  Split operands hold a second half per entry (22 bits); a tile then takes three products,
// lead x lead and the two crossed ones, of the same fragments.
// What is multiplied is held to 11 bits (22 if split), what is added (a X) to 22 either way: a rounding of the linear term is carried on
// and grows as the smallest singular values do, 3.4445 per step, one in a factor of B X only turns singular vectors.  (Updates of rank
// 32 at 512 x 512: error of the result 9e-4 so, 3e-2 with X in 11 bits throughout, 0.2 in bfloat16.)  B's diagonal, which holds most of
// B where the spectrum is flat, is held to 22 bits as well and meets both halves of X, in the sums of B X's epilogue: 2.1e-3 -> 1.1e-3 at
// 70 x 80, 1.5e-3 -> 8e-4 at 512 x 512 (where three quarters of the singular values are 0, 1e-3 -> 1.4e-3), for at most 1 % of a call's time.
// Large matrices: 8 x 4096 x 4096 in half precision, B X 1122 us (980 TFLOP/s; on another card 1084, 1014 TFLOP/s).  The matrix cores are busy
// 55 % of the cycles, at 1.7 GHz, and wavefronts wait 40 % of theirs: one workgroup to a compute unit, which meets at a barrier per 64 of depth and
// has nothing beside its first requests and its epilogue.  A library's batched product of that size runs at 1100 TFLOP/s, 1000 us.  X X^T 596 us for
// 136 of 256 tiles (5 rounds of 256 where 4.25 would do).  16 x 1024 x 1024 split, B X 110 us: 934 TFLOP/s of the three products.
// Bound by latency where they are small: no launch is under 5 us (4 x 4 tiles
// of 64 x 64 with a contraction of 256: 5.3), most of it the way from one kernel's last store to the next one's first operands.
#include <algorithm>
#include <atomic>
#include <type_traits>

#include "orth_rows.h"

namespace prsgd {

namespace {

typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));

__device__ __forceinline__ float half_value(uint16_t h) { return (float)__builtin_bit_cast(_Float16, h); }
__device__ __forceinline__ uint16_t half_bits(float f) { return __builtin_bit_cast(uint16_t, (_Float16)f); }
// leading halves and remainders of eight values
__device__ __forceinline__ void split8(const float* v, u32x4_t* hi, u32x4_t* lo) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const uint16_t h0 = half_bits(v[2 * e]), h1 = half_bits(v[2 * e + 1]);
    (*hi)[e] = (uint32_t)h0 | (uint32_t)h1 << 16;
    (*lo)[e] = (uint32_t)half_bits(v[2 * e] - half_value(h0)) | (uint32_t)half_bits(v[2 * e + 1] - half_value(h1)) << 16;
  }
}
__device__ __forceinline__ float half_at(u32x4_t v, int e) { return half_value((uint16_t)(v[e / 2] >> (16 * (e & 1)))); }

// halves of column c of a row; remainders of split columns stand kGroup halves behind
constexpr int kGroup = 16;
template <bool SPLIT> __device__ __forceinline__ int half_col(int c) { return SPLIT ? (c >> 4) * 32 + (c & 15) : c; }
// A tile of an operand: ROWS rows (or columns) of the product by RB bytes' depth each, requested by NW wavefronts.  LDS has 64 banks, and
// the 256 bytes that 16 lanes read at a time have to lie on different ones: a tile cannot be padded on its way, so pieces of a row are exchanged.
//   rows contiguous along the contraction: [ROWS][RB], 16-byte chunk q of row r at chunk_place(r, q)
//   TRANS: [depth][ROWS halves, or pairs of them], 32-byte unit u of contraction row c at u ^ unit_xor(c), for reads that transpose
template <int RB> __device__ __forceinline__ int chunk_place(int r, int q) { return RB == 128 ? q ^ ((r >> 1) & 7) : q ^ ((r >> 2) & 3); }
template <int ROW, bool SPLIT> __device__ __forceinline__ int unit_xor(int c) {      // ROW: bytes of a contraction row
  static_assert(ROW % 256 == 0 || (ROW == 128 && !SPLIT), "rows of whole bank sets, or two to a set");
  return SPLIT ? (c & 1) | (c & 2) << 1 : ROW == 128 ? c & 2 : (c & 3) << 1;
}
template <int ROWS, int RB, int NW, bool SPLIT, bool TRANS> struct TileRequests {
  static constexpr int NPT = ROWS * RB / 1024 / NW;
  static_assert(ROWS * RB % (1024 * NW) == 0, "a tile splits evenly over the wavefronts");
  uint32_t off[NPT];
  // n: rows (TRANS: halves of a row) of the operand from the tile's first on; what lies past them is a copy of the last, never stored
  __device__ __forceinline__ void set(int ld, int n, int wave, int lane) {
#pragma unroll
    for (int q = 0; q < NPT; ++q) {
      const int chunk = (q * NW + wave) * 64 + lane;
      if constexpr (TRANS) {
        constexpr int ROW = ROWS * (SPLIT ? 4 : 2), CH = ROW / 16;
        const int c = chunk / CH, pos = chunk % CH, from = ((((pos >> 1) ^ unit_xor<ROW, SPLIT>(c)) << 1) | (pos & 1)) * 8;
        off[q] = ((uint32_t)c * (uint32_t)ld + (uint32_t)min(from, n - 8)) * 2u;
      } else {
        constexpr int CH = RB / 16;
        const int r = chunk / CH;
        off[q] = (uint32_t)min(r, n - 1) * (uint32_t)ld * 2u + (uint32_t)chunk_place<RB>(r, chunk % CH) * 16u;
      }
    }
  }
  __device__ __forceinline__ void request(const uint16_t* base, uint32_t lds_tile, int q, int wave) const {
    load_to_lds(base, off[q], lds_tile + (uint32_t)(q * NW + wave) * 1024u);
  }
};

template <int N> __device__ __forceinline__ void wait_requests() {
  static_assert(N <= 63, "vmcnt");
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" :: "n"(N) : "memory");
}

// MFMA operands of 32-row blocks: lane (r = lane % 32, kb = lane / 32) holds contraction elements 8 kb .. 8 kb + 7 of row r.  Where a lane
// reads depends on the slice and the half through an exchange, on the block through a constant: COUNT places are kept per lane.
template <int RB, bool SPLIT> struct RowFragments {
  static constexpr int PARTS = SPLIT ? 2 : 1, KK = RB / 32 / PARTS, COUNT = KK * PARTS;
  int at[COUNT];
  __device__ __forceinline__ void set(int first_block, int lane) {
#pragma unroll
    for (int x = 0; x < COUNT; ++x) at[x] = (first_block * 32 + (lane & 31)) * RB + (chunk_place<RB>(lane & 31, 2 * x + (lane >> 5)) << 4);
  }
  __device__ __forceinline__ f16x8_t read(const unsigned char* tile, int block, int kk, int h) const {
    return __builtin_bit_cast(f16x8_t, *reinterpret_cast<const u32x4_t*>(tile + at[kk * PARTS + h] + block * 32 * RB));
  }
};
// The same out of a TRANS tile, by two ds_read_b64_tr_b16: of every 16 lanes, lane r gives the address of four halves M[r], and lane i gets
// M[4 j + i / 4][i % 4], j = 0..3.  The exchange takes in the lowest bits of the block.
template <int ROWS, bool SPLIT> struct ColumnFragments {
  static constexpr int ROW = ROWS * (SPLIT ? 4 : 2), COUNT = 4;
  int at[COUNT];
  __device__ __forceinline__ void set(int first_block, int lane) {
    const int g = lane >> 4, r = lane & 15, c = 8 * (g >> 1) + (r >> 2);
#pragma unroll
    for (int x = 0; x < COUNT; ++x) {      // split: block x / 2, half x % 2; otherwise block x
      const int unit = SPLIT ? 4 * (first_block + x / 2) + 2 * (g & 1) + x % 2 : 2 * (first_block + x) + (g & 1);
      at[x] = c * ROW + (unit ^ unit_xor<ROW, SPLIT>(r >> 2)) * 32 + 8 * (r & 3);
    }
  }
  __device__ __forceinline__ f16x8_t read(const unsigned char* tile, int block, int kk, int h) const {
    typedef __attribute__((__vector_size__(4 * sizeof(__fp16)))) __fp16 f16x4_t;
    typedef __attribute__((address_space(3))) f16x4_t* lds_f16x4_ptr;
    const unsigned char* p = tile + (SPLIT ? at[block % 2 * 2 + h] + block / 2 * 256 : at[block % 4] + block / 4 * 256) + kk * 16 * ROW;
    const f16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4f16((lds_f16x4_ptr)(p));
    const f16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4f16((lds_f16x4_ptr)(p + 4 * ROW));
    return __builtin_bit_cast(f16x8_t, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  }
};

// Order of a matrix's tiles: strips kStrip tiles high, column by column, so that the tiles that an XCD works on at a time share more of
// their operands in its L2 (of 32 tiles 4 rows and 8 columns, against 2 and 16 row by row).
constexpr int kStrip = 4;
__device__ __forceinline__ void strip_tile(int in, int tiles_m, int tiles_n, int* ti, int* tj) {
  const int strip = in / (kStrip * tiles_n), first = strip * kStrip, high = min(kStrip, tiles_m - first), rest = in - first * tiles_n;
  *tj = rest / high;
  *ti = first + rest - *tj * high;
}
// The same over the tiles on and below the diagonal.
__device__ __forceinline__ void triangle_tile(int in, int tiles, int* ti, int* tj) {
  int rest = in, first = 0, high = min(kStrip, tiles);
  while (rest >= high * first + high * (high + 1) / 2) {   // tiles of the strip's rows
    rest -= high * first + high * (high + 1) / 2;
    first += kStrip;
    high = min(kStrip, tiles - first);
  }
  int row, col = rest / high;
  if (col < first) {
    row = first + rest - col * high;
  } else {                                                 // the triangle at the strip's end
    rest -= first * high;
    col = first;
    for (int left = high; rest >= left; --left, ++col) rest -= left;
    row = col + rest;
  }
  *ti = row;
  *tj = col;
}

constexpr int strip_pitch(int columns) { return columns + 8; }     // the four rows between a register's two halves lie 32 banks apart
template <int BM, int BN, int S, int RB> constexpr int square_lds_bytes(int wm, int wn) {
  const int stages = S * (BM + BN) * RB, strips = wm * wn * 32 * strip_pitch(BN / wn) * 4;
  return stages > strips ? stages : strips;
}

// WM x WN wavefronts, S tiles of RB bytes' depth in LDS.
template <int BM, int BN, int WM, int WN, int S, int RB, bool SPLIT, int EPI>
__global__ void __launch_bounds__(64 * WM * WN, 2) square_kernel(const SquareArgs p) {
  constexpr int NW = WM * WN, TM = BM / WM / 32, TN = BN / WN / 32, PARTS = SPLIT ? 2 : 1, KK = RB / 32 / PARTS;
  constexpr bool SYMMETRIC = EPI == SQ_GRAM || EPI == SQ_POLY, TRANS = !SYMMETRIC;
  constexpr int STAGE = (BM + BN) * RB;
  using User = std::conditional_t<SPLIT, float, uint16_t>;
  using ReqA = TileRequests<BM, RB, NW, SPLIT, false>;
  using ReqB = TileRequests<BN, RB, NW, SPLIT, TRANS>;
  constexpr int PER = ReqA::NPT + ReqB::NPT;
  static_assert(!SYMMETRIC || BN == BM, "tiles of a symmetric result");
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  fetch_kernel_args<sizeof(SquareArgs)>();
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / WN, wn = wave % WN;

  // Consecutive workgroups go to the XCDs in turn; each XCD gets a contiguous range of the tiles, so that a matrix stays in few L2s.
  const int total = p.tiles * p.count, xcd = blockIdx.x & 7;
  const int idx = xcd * (total >> 3) + min(xcd, total & 7) + (blockIdx.x >> 3);
  const int g = idx / p.tiles, in = idx - g * p.tiles;
  int ti, tj;
  if (SYMMETRIC) triangle_tile(in, p.tiles_n, &ti, &tj);
  else strip_tile(in, (p.M + BM - 1) / BM, p.tiles_n, &ti, &tj);
  const int m0 = ti * BM, n0 = tj * BN;
  // what of the matrix's room the operand X holds, and the result will (asking for it costs a call 0.5 to 0.8 %, here or further down)
  int shift = 0;
  if constexpr (EPI != SQ_POLY) {
    const int room = ((const __attribute__((address_space(4))) int*)p.room)[g], held = max(room - (int)p.grown, 0);
    shift = EPI == SQ_GRAM ? -2 * held : EPI == SQ_NEXT ? max(room - (int)p.grown_next, 0) - held : -held;
  }

  // Strips of the epilogue: columns, pitch, 8-value vectors of a row, rows per pass
  constexpr int W = BN / WN, P = strip_pitch(W), VPR = W / 8, RPP = 64 / VPR, PASSES = 32 / RPP;
  const int c0 = n0 + wn * W;
  // what the epilogue adds to the product at pass q of strip i
  struct Linear { u32x4_t hi, lo; f32x2_t diag; };
  auto linear = [&](int i, int q) __attribute__((always_inline)) {
    Linear v = {{0, 0, 0, 0}, {0, 0, 0, 0}, {0.0f, 0.0f}};
    const int r = m0 + (wm * TM + i) * 32 + q * RPP + lane / VPR, c = c0 + lane % VPR * 8;
    if (EPI != SQ_GRAM && r < p.M && c < p.N) {
      const int64_t o = g * p.lin_gs + (int64_t)r * p.ld_lin + half_col<SPLIT>(c);
      v.hi = *reinterpret_cast<const u32x4_t*>(p.lin + o);
      if (SPLIT) v.lo = *reinterpret_cast<const u32x4_t*>(p.lin + o + kGroup);
      else if (EPI != SQ_POLY) v.lo = *reinterpret_cast<const u32x4_t*>(p.lin_lo + o);
      if (!SPLIT && TRANS) v.diag = *reinterpret_cast<const f32x2_t*>(p.diag + 2 * ((int64_t)g * p.M + r));
    }
    return v;
  };
  // A workgroup with a single strip per wavefront asks for all of that first: behind the products it would wait for it once more.
  constexpr bool AHEAD = TM == 1 && PASSES <= 2;
  Linear ahead[AHEAD ? PASSES : 1];
  if constexpr (AHEAD) {
#pragma unroll
    for (int q = 0; q < PASSES; ++q) ahead[q] = linear(0, q);
  }

  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)smem;
  const uint16_t* a = p.a + g * p.a_gs + (int64_t)m0 * p.lda;
  const uint16_t* b = p.b + g * p.b_gs + (TRANS ? (int64_t)half_col<SPLIT>(n0) : (int64_t)n0 * p.ldb);
  const int64_t b_step = TRANS ? (int64_t)(RB / 2 / PARTS) * p.ldb : RB / 2;
  ReqA ra;
  ReqB rb;
  ra.set(p.lda, p.M - m0, wave, lane);
  rb.set(p.ldb, TRANS ? p.ldb - half_col<SPLIT>(n0) : p.N - n0, wave, lane);
  const int n_k = p.lda * 2 / RB;
  auto request = [&](int t, int place, int first, int last) __attribute__((always_inline)) {       // place: t mod S
    const uint32_t stage = lds0 + (uint32_t)place * STAGE;
#pragma unroll
    for (int q = first; q < last; ++q) {
      if (q < ReqA::NPT) ra.request(a + t * (RB / 2), stage, q, wave);
      else rb.request(b + t * b_step, stage + BM * RB, q - ReqA::NPT, wave);
    }
  };
  f16x8_t fa[2][PARTS][TM], fb[2][PARTS][TN];
  constexpr int READS = PARTS * (TM + TN);
  RowFragments<RB, SPLIT> rows;
  std::conditional_t<TRANS, ColumnFragments<BN, SPLIT>, RowFragments<RB, SPLIT>> cols;
  rows.set(wm * TM, lane);
  cols.set(wn * TN, lane);
  // fragment q of slice kk
  auto load = [&](const unsigned char* tile, int kk, int set, int q) __attribute__((always_inline)) {
    const int h = q / (TM + TN), x = q % (TM + TN);
    if (x < TM) fa[set][h][x] = rows.read(tile, x, kk, h);
    else fb[set][h][x - TM] = cols.read(tile + BM * RB, x - TM, kk, h);
  };
  f32x16_t acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;

  // Tile t + 1 is met before the last slice of tile t is multiplied; from there on every fragment of tile t has been read, and its stage
  // takes tile t + S.  Each row of a slice's products is followed by its share of
  // the next slice's fragments and of the requests, so that neither waits in a burst of its own (a request takes 16 cycles of the compute
  // unit's one path to its cache).
#pragma unroll
  for (int t = 0; t < S; ++t)
    if (t < n_k) request(t, t, 0, PER);
  if (n_k >= S) wait_requests<(S - 1) * PER>(); else wait_requests<0>();
  asm volatile("s_barrier" ::: "memory");
#pragma unroll
  for (int q = 0; q < READS; ++q) load(smem, 0, 0, q);
  // set0: the fragments' set of the tile's first slice
  int place = 0;
  auto step = [&](int t, auto set0_, auto whole_) __attribute__((always_inline)) {
    constexpr bool WHOLE = decltype(whole_)::value;        // every tile that the step asks for exists
    const int behind = place + 1 == S ? 0 : place + 1;
    const unsigned char* here = smem + place * STAGE;
    const unsigned char* next = smem + behind * STAGE;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
      const int set = (decltype(set0_)::value + kk) & 1;
      const bool last = kk == KK - 1;
      if (last) {
        if (WHOLE || t + S - 1 < n_k) wait_requests<(S - 2) * PER>(); else wait_requests<0>();
        asm volatile("s_barrier" ::: "memory");
      }
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        if (!last || WHOLE || t + 1 < n_k) {
#pragma unroll
          for (int q = i * READS / TM; q < (i + 1) * READS / TM; ++q) load(last ? next : here, last ? 0 : kk + 1, set ^ 1, q);
        }
#pragma unroll
        for (int j = 0; j < TN; ++j) {
          acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(fa[set][0][i], fb[set][0][j], acc[i][j], 0, 0, 0);
          if constexpr (SPLIT) {
            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(fa[set][0][i], fb[set][1][j], acc[i][j], 0, 0, 0);
            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(fa[set][1][i], fb[set][0][j], acc[i][j], 0, 0, 0);
          }
        }
        if (last && (WHOLE || t + S < n_k)) request(t + S, place, i * PER / TM, (i + 1) * PER / TM);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    place = behind;
  };
  using Set0 = std::integral_constant<int, 0>;
  using Set1 = std::integral_constant<int, KK & 1>;        // of odd tiles
  int t = 0;
  for (; t + S + 1 < n_k; t += 2) {
    step(t, Set0{}, std::true_type{});
    step(t + 1, Set1{}, std::true_type{});
  }
  for (; t < n_k; t += 2) {
    step(t, Set0{}, std::false_type{});
    if (t + 1 < n_k) step(t + 1, Set1{}, std::false_type{});
  }
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");

  const float alpha = ldexpf(p.alpha, shift), beta = ldexpf(p.beta, shift), diag_scale = ldexpf(p.diag_scale, shift);
  // Epilogue: a wavefront passes strips of 32 rows through LDS, first along the rows and then, as transposes, along the columns.
  float* strip = reinterpret_cast<float*>(smem) + wave * 32 * P;
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    const int r0 = m0 + (wm * TM + i) * 32;
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) strip[(8 * (e / 4) + 4 * (lane >> 5) + (e % 4)) * P + j * 32 + (lane & 31)] = acc[i][j][e];
    __builtin_amdgcn_wave_barrier();
#pragma unroll(EPI == SQ_LAST && !AHEAD ? 1 : PASSES)
    for (int q = 0; q < PASSES; ++q) {
      const int lr = q * RPP + lane / VPR, lc = lane % VPR * 8, r = r0 + lr, c = c0 + lc;
      float* at = strip + lr * P + lc;
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; e += 2) {
        const f32x2_t x = *reinterpret_cast<const f32x2_t*>(at + e);
        v[e] = x[0];
        v[e + 1] = x[1];
      }
      const bool inside = r < p.M && c < p.N;
      const int hc = half_col<SPLIT>(c);
      if constexpr (EPI != SQ_GRAM) {
        Linear x;
        if constexpr (AHEAD) x = ahead[q];
        else x = linear(i, q);
        if constexpr (!SPLIT && TRANS) {
          // (a + what the half of B_ii leaves out) X + B X with X's remainder at B_ii
          const float whole = fmaf(diag_scale, x.diag[1], alpha), half = diag_scale * x.diag[0];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float rest = half_at(x.lo, e);
            v[e] = fmaf(whole, half_at(x.hi, e) + rest, fmaf(half, rest, beta * v[e]));
          }
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] = fmaf(alpha, half_at(x.hi, e) + half_at(x.lo, e), beta * v[e]);
        }
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] *= beta;
      }
      // padding columns of the halves hold zeros, and so do padding rows of transposes
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = r < p.M && c + e < p.N ? v[e] : 0.0f;
      if constexpr (!SPLIT && EPI == SQ_POLY) {
        if ((unsigned)(r - c) < 8u && r < p.M) {           // the vector holds the diagonal entry of its row
          float d = v[0];
#pragma unroll
          for (int e = 1; e < 8; ++e) d = r == c + e ? v[e] : d;
          const float half = half_value(half_bits(d));
          *reinterpret_cast<f32x2_t*>(p.diag + 2 * ((int64_t)g * p.M + r)) = (f32x2_t){half, d - half} * (1.0f / kHalfScale);
        }
      }
      if constexpr (EPI == SQ_LAST) {
        if (!p.transposed && inside) {
          const int64_t o = g * p.user.out_matrix + r * p.user.out_row + c;
          result8<User>(p.user, o, p.N - c, v);
        }
      } else if (r < p.M && hc < p.ldo) {
        u32x4_t hi, lo;
        split8(v, &hi, &lo);
        const int64_t o = g * p.out_gs + (int64_t)r * p.ldo + hc;
        *reinterpret_cast<u32x4_t*>(p.out + o) = hi;
        if (SPLIT) *reinterpret_cast<u32x4_t*>(p.out + o + kGroup) = lo;
        else if (EPI == SQ_NEXT) *reinterpret_cast<u32x4_t*>(p.out_lo + o) = lo;
      }
#pragma unroll
      for (int e = 0; e < 8; e += 2) *reinterpret_cast<f32x2_t*>(at + e) = (f32x2_t){v[e], v[e + 1]};
    }
    __builtin_amdgcn_wave_barrier();
    if (SYMMETRIC ? ti != tj : EPI == SQ_LAST && p.transposed) {
#pragma unroll(EPI == SQ_LAST ? 1 : W / 16)
      for (int q = 0; q < W / 16; ++q) {
        const int lc = q * 16 + lane % 16, lr = lane / 16 * 8, c = c0 + lc, r = r0 + lr;
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = strip[(lr + e) * P + lc];
        if (c >= p.N) continue;
        if constexpr (EPI == SQ_LAST) {
          if (r < p.M) {
            const int64_t o = g * p.user.out_matrix + c * p.user.out_row + r;
            result8<User>(p.user, o, p.M - r, v);
          }
        } else {
          const int hr = half_col<SPLIT>(r);
          if (hr < p.ldt) {
            u32x4_t hi, lo;
            split8(v, &hi, &lo);
            const int64_t o = g * p.t_gs + (int64_t)c * p.ldt + hr;
            *reinterpret_cast<u32x4_t*>(p.out_t + o) = hi;
            if (SPLIT) *reinterpret_cast<u32x4_t*>(p.out_t + o + kGroup) = lo;
          }
        }
      }
      __builtin_amdgcn_wave_barrier();
    }
  }
}

template <int BM, int BN, int WM, int WN, int S, int RB, bool SPLIT, int EPI> hipError_t launch_as(SquareArgs p, hipStream_t s) {
  constexpr int kLds = square_lds_bytes<BM, BN, S, RB>(WM, WN);
  static_assert(kLds <= 160 * 1024, "LDS of a compute unit");
  auto kernel = square_kernel<BM, BN, WM, WN, S, RB, SPLIT, EPI>;
  // the tiles can exceed the 64 KB default; setting the limit twice is harmless
  static std::atomic<bool> configured{false};
  if (!configured.load(std::memory_order_acquire)) {
    hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, kLds);
    if (e != hipSuccess) return e;
    configured.store(true, std::memory_order_release);
  }
  const int tiles_m = (p.M + BM - 1) / BM;
  p.tiles_n = (p.N + BN - 1) / BN;
  p.tiles = EPI == SQ_GRAM || EPI == SQ_POLY ? p.tiles_n * (p.tiles_n + 1) / 2 : tiles_m * p.tiles_n;
  hipLaunchKernelGGL(kernel, dim3((unsigned)p.tiles * (unsigned)p.count), dim3(64 * WM * WN), kLds, s, p);
  return hipGetLastError();
}
template <int BM, int BN, int WM, int WN, int S, int RB, bool SPLIT> hipError_t launch_tile(const SquareArgs& p, int epi, hipStream_t s) {
  switch (epi) {
    case SQ_GRAM: return launch_as<BM, BN, WM, WN, S, RB, SPLIT, SQ_GRAM>(p, s);
    case SQ_POLY: return launch_as<BM, BN, WM, WN, S, RB, SPLIT, SQ_POLY>(p, s);
    case SQ_NEXT: return launch_as<BM, BN, WM, WN, S, RB, SPLIT, SQ_NEXT>(p, s);
    default: return launch_as<BM, BN, WM, WN, S, RB, SPLIT, SQ_LAST>(p, s);
  }
}

}  // namespace

hipError_t launch_square(SquareArgs p, int epi, bool split, hipStream_t s) {
  const bool symmetric = epi == SQ_GRAM || epi == SQ_POLY;
  // Time of a launch in units of a 64 x 64 tile's products: tiles per compute unit times their size over their efficiency.  Of tiles that a
  // compute unit has several of in hand, parts of a round count as such; of 256 x 256 tiles whole rounds.
  // Measured over 28 shapes from 64 x (128 x 256) to 8 x (2048 x 2048), every tile size for each of the three products: this takes the
  // fastest or one within 4 % of a call.  Where it matters most: B X of 16 x (320 x 800) in bf16, call of 133 us in 64 x 64 tiles, 171 in
  // 256 x 256; X X^T of 8 x (1000 x 4096), 895 us in 128 x 128, 1018 in 256 x 256; B X of 8 x (2048 x 2048) 2244 us in 64 x 64, 1942 in
  // 128 x 128, 1766 in 256 x 256.  (128 x 256 tiles were nowhere better by more than 1 %.)  Split products keep to 128 x 128: larger tiles do not
  // leave two workgroups per compute unit the registers.
  // 128 x 128 tiles: three workgroups of four wavefronts to a compute unit where there are that many; where there are two or one to each,
  // workgroups of eight wavefronts that hold more of the contraction in LDS.  Calls in bf16: X X^T of 1 x (2048 x 2048), 136 tiles, 398 us
  // in four wavefronts and 370 in eight, of 1 x (2900 x 2900), 276 tiles, 986 and 925, B X of 12 x (512 x 1000), 384 tiles, 196 and
  // 187; from 513 tiles on the other way around (B X of 16 x (768 x 768) 372 and 383).  In fp32 1 to 2 %.  More rounds of tiles than one over
  // a long contraction run in two workgroups of four, half as many barriers (bf16 2 x (4096 x 4096) 3280 and 3010 us, fp32 7950 and
  // 7340); over a short one in three (bf16 30 x (700 x 700) 528 and 560).
  auto tiles = [&](int b) {
    const int64_t tm = (p.M + b - 1) / b, tn = (p.N + b - 1) / b;
    return (symmetric ? tn * (tn + 1) / 2 : tm * tn) * p.count;
  };
  auto cost = [](int64_t n, int b, double efficiency) { return (n < 256 ? 1.0 : (double)n / 256.0) * (b / 64) * (b / 64) / efficiency; };
  const int64_t n_middle = tiles(128), n_huge = (tiles(256) + 255) / 256 * 256;
  const double middle = cost(n_middle, 128, n_middle > 256 ? 0.9 : split ? 1.4 : 1.34), small = cost(tiles(64), 64, split ? 0.77 : 0.68);
  if (!split && cost(n_huge, 256, 1.2) <= std::min(middle, small)) return launch_tile<256, 256, 4, 2, 2, 128, false>(p, epi, s);
  auto launch = [&](auto split_) {
    constexpr bool SPLIT = decltype(split_)::value;
    if (middle > small) return launch_tile<64, 64, 2, 2, 4, 128, SPLIT>(p, epi, s);
    if (n_middle <= 256) return launch_tile<128, 128, 4, 2, 3, 128, SPLIT>(p, epi, s);
    if (n_middle <= 512) return launch_tile<128, 128, 4, 2, 2, 128, SPLIT>(p, epi, s);
    if (n_middle > 768 && p.lda >= 2048) return launch_tile<128, 128, 2, 2, 2, 128, SPLIT>(p, epi, s);
    return launch_tile<128, 128, 2, 2, 3, 64, SPLIT>(p, epi, s);
  };
  return split ? launch(std::true_type{}) : launch(std::false_type{});
}

}  // namespace prsgd
