// Gated linear recurrence over packed sequences, forward and backward.
//   f = sigmoid(gate),  h_t = f_t h_{t-1} + (1 - f_t) v_t
//   c_t = f_t (dh_t + c_{t+1}) (c behind the last row is dlast),  g_t = dh_t + c_{t+1},
//   dv_t = (1 - f_t) g_t,  dgate_t = f_t (1 - f_t) (h_{t-1} - v_t) g_t,  dinitial = c of the first row
// Both are x -> a x + b along a sequence, the second one from its end.  A workgroup has 64 channels of one sequence and walks along it: every lane
// holds R rows of eight channels, composes them, and lanes, then wavefronts, compose theirs, so that a pass over NW * 8 * R rows reads
// each of them once and needs no workgroup to wait for another.  States and compositions are fp32.  Bound by HBM where sequences are many (64 packed ones, 65536 x 2048
// bf16: 187 to 213 us by where they are cut, 3.8 to 4.3 TB/s; gradients 368 us, 4.4 TB/s), by the 2 us of a pass where they are few.
#include <algorithm>
#include <cmath>

#include "orth_rows.h"
#include "prsgd_token_internal.h"
#include "row_pieces.h"

namespace prsgd {

namespace {

// sigmoid(x) and sigmoid(-x), neither as a difference from 1.  The hardware's base-2 exponential is good to a rounding of its own, but its argument's rounding
// would leave 0.7 |x| 2^-23 of the result, which a product over a long sequence adds up: it is made good, and so is the reciprocal's.  (Rows in bf16 too: their
// gates are exact numbers, and the states' gradient is fp32.  With neither, that of 4 x 16384 x 2048 was off by four times as much, in no less time.)
__device__ __forceinline__ void gates(float x, float& f, float& rest) {
  const float t = fabsf(x) > 128.0f ? 128.0f : fabsf(x);         // NaN stays; from 104 on e is 0 anyway
  const float hi = t * -1.44269502f, lo = fmaf(t, -1.92596299e-8f, fmaf(t, -1.44269502f, -hi)), power = __builtin_amdgcn_exp2f(hi);
  const float e = fmaf(power * 0.693147181f, lo, power), d = 1.0f + e, close = __builtin_amdgcn_rcpf(d);
  const float r = fmaf(fmaf(-d, close, 1.0f), close, close), s = e * r;
  f = x >= 0.0f ? r : s;
  rest = x >= 0.0f ? s : r;
}

constexpr int kTile = 64, kWaves = 8;    // channels and wavefronts of a workgroup
constexpr int kPass = kWaves * (kWave / (kTile / 8)) * 2;      // rows that it takes at a time

struct Span { int first, end; };
__device__ __forceinline__ Span span_of(const ScanArgs& p, int s) {
  if (p.starts == nullptr) {
    const int length = (int)(p.rows / p.sequences);
    return {s * length, (s + 1) * length};
  }
  // what no caller should write, but a device can hold: never past the rows
  const int first = min(max(p.starts[s], 0), (int)p.rows);
  return {first, min(max(p.starts[s + 1], first), (int)p.rows)};
}

// Zeros in the rows that no sequence has, and (where rows are cut into parts) the states that pass sequences without rows, by workgroups behind the others.
enum ScanMode { WHOLE = 0, COMPOSE = 1, APPLY = 2 };
constexpr int kClearers = 64;
template <typename T, bool BACK, int MODE> __device__ __forceinline__ void clear_rest(const ScanArgs& p, int block) {
  if constexpr (MODE == APPLY) {
    const float* from = BACK ? p.dlast : p.initial;
    const int64_t from_row = BACK ? p.dlast_row : p.initial_row;
    for (int s = block; s < p.sequences && p.last != nullptr; s += kClearers) {
      const Span q = span_of(p, s);
      if (q.end > q.first) continue;
      for (int c = threadIdx.x; c < p.width; c += blockDim.x) p.last[s * p.last_row + c] = from != nullptr ? from[s * from_row + c] : 0.0f;
    }
  }
  const int first = min(max(p.starts[0], 0), (int)p.rows), end = min(max(p.starts[p.sequences], first), (int)p.rows);
  const float none[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  for (int i = block; i < first + ((int)p.rows - end) && p.clear != 0; i += kClearers) {
    const int64_t row = i < first ? i : end + (i - first);
    for (int c = threadIdx.x * 8; c < p.width; c += blockDim.x * 8) {
      if ((p.clear & 1) != 0) store8(reinterpret_cast<T*>(p.h) + row * p.h_row + c, p.width - c, none);
      if ((p.clear & 2) != 0) store8(reinterpret_cast<T*>(p.dgate) + row * p.dgate_row + c, p.width - c, none);
    }
  }
}

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
// Eight channels of a row.  VEC: rows are whole eights, so that no lane has a part of one.  Otherwise such a part comes with what lies before it (its rows begin at
// `first`), and is moved into place when it is used.  (The branch between both costs a wait, but what load_piece needs would not stay in registers here.)
template <bool VEC, typename T> __device__ __forceinline__ void load_channels(Raw8<T>& v, const T* p, int n, const void* first) {
  constexpr int ES = (int)sizeof(T), V = 16 / ES;
#pragma unroll
  for (int i = 0; i < 8 / V; ++i) {
    if (VEC || n >= (i + 1) * V) v.q[i] = reinterpret_cast<const Packed16<ES>*>(p + i * V)->v;
    else if (n > i * V) v.q[i] = load_end<ES>(p + i * V, n - i * V, first);
    else v.q[i] = (u32x4_t){0, 0, 0, 0};
  }
}
template <typename T> __device__ __forceinline__ void place_channels(Raw8<T>& v, int n) {
  constexpr int ES = (int)sizeof(T), V = 16 / ES;
#pragma unroll
  for (int i = 0; i < 8 / V; ++i)
    if (n > i * V && n < (i + 1) * V) v.q[i] = place_piece<ES>(v.q[i], n - i * V);
}

// Workgroups take packed sequences longest first, where these are few enough to be compared by each of them, so that the longest is not the last to start.
constexpr int kRanked = 256;
template <int THREADS> __device__ __forceinline__ int nth_longest(const ScanArgs& p, int nth) {
  __shared__ int length[kRanked], found;
  for (int i = threadIdx.x; i < p.sequences; i += THREADS) {
    const Span s = span_of(p, i);
    length[i] = s.end - s.first;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < p.sequences; i += THREADS) {
    const int mine = length[i];
    int rank = 0;
    for (int j = 0; j < p.sequences; ++j) rank += length[j] > mine || (length[j] == mine && j < i) ? 1 : 0;
    if (rank == nth) found = i;
  }
  __syncthreads();
  return found;
}

// Where the longest sequence would be walked for longer than all others take, the rows of all sequences are cut into equal parts (p.parts), wherever
// sequences end: a first launch composes each part's rows, a second composes the parts before its own, which gives the state that comes to it, and scans.
// A sequence's first row replaces what comes to it by the sequence's state, which a composition x -> a x + b notes as a < 0, so that a NaN before it goes nowhere.
constexpr int kTableRows = 4 * kPass;    // rows of which a workgroup knows at a time which are the first and the last of a sequence
__device__ __forceinline__ Span part_of(Span s, int part, int parts) {
  const int each = ((s.end - s.first + parts - 1) / parts + kPass - 1) / kPass * kPass, from = (int)min(s.first + (int64_t)part * each, (int64_t)s.end);
  return {from, (int)min(from + (int64_t)each, (int64_t)s.end)};
}
template <bool RESETS> __device__ __forceinline__ void compose(float& a, float& b, float2 next) {
  if constexpr (RESETS) {
    b = next.x < 0.0f ? next.y : fmaf(next.x, b, next.y);
    a = a < 0.0f || next.x < 0.0f ? -1.0f : a * next.x;
  } else {
    b = fmaf(next.x, b, next.y);
    a *= next.x;
  }
}

// NW wavefronts; CL lanes share a row, R rows a lane.  The next pass's rows are on their way while this one's are composed.
template <typename T, bool BACK, int NW, int R, int CL, bool VEC, int OCC, int MODE> __global__ void __launch_bounds__(NW * kWave, OCC) scan_kernel(ScanArgs p, int tiles) {
  constexpr int CH = 8 * CL, PARTS = kWave / CL, PASS = NW * PARTS * R;
  constexpr bool CUT = MODE != WHOLE;
  // compositions of the lanes' rows, then the states in front of them; of a wavefront, which alone reads them
  __shared__ __attribute__((aligned(16))) float composed[NW][PARTS][CH][2];
  __shared__ float total[2][NW][CH][2];
  __shared__ int head[CUT ? kTableRows : 1], tail[CUT ? kTableRows : 1];
  const int workgroups = tiles * (CUT ? p.parts : p.sequences);
  if (blockIdx.x >= (unsigned)workgroups) {
    clear_rest<T, BACK, MODE>(p, (int)(blockIdx.x - workgroups));
    return;
  }
  // Workgroups go to the XCDs in turn.  Those of half a line of bf16 that lie side by side go to one, so that they meet in its L2.
  int block = blockIdx.x;
  if constexpr (CL < 8) block = (block & 7) * (workgroups >> 3) + min(block & 7, workgroups & 7) + (block >> 3);
  const int slot = block / tiles, c_wg = (block - slot * tiles) * CH;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid / kWave), lane = tid % kWave, part = lane / CL, cl = lane % CL * 8;
  const int c = c_wg + cl, n = p.width - c;
  int sequence = slot;                   // WHOLE
  Span all, span;
  if constexpr (CUT) {
    all = {span_of(p, 0).first, span_of(p, p.sequences - 1).end};
    all.end = max(all.end, all.first);
    span = part_of(all, BACK ? p.parts - 1 - slot : slot, p.parts);
  } else {
    if (NW > 1 && p.starts != nullptr && p.sequences <= kRanked) sequence = __builtin_amdgcn_readfirstlane(nth_longest<NW * kWave>(p, sequence));
    all = span = span_of(p, sequence);
  }
  const int length = span.end - span.first;
  // of channel c_wg + lane % CH, in every wavefront alike
  const int own = lane % CH;
  const bool owns = c_wg + own < p.width;
  float2* joint = CUT ? p.joint + c_wg + own : nullptr;    // of the parts: their compositions
  float state = 0.0f, product = 1.0f;
  if (!CUT && owns) {
    if (BACK) state = p.dlast != nullptr ? p.dlast[sequence * p.dlast_row + c_wg + own] : 0.0f;
    else state = p.initial != nullptr ? p.initial[sequence * p.initial_row + c_wg + own] : 0.0f;
  }
  struct Rows { Raw8<T> gate, v, dh, h; };
  Rows ahead[R];
  // Row `at` of this lane, counted from the span's end backward, and what lies one row and one pass further on.
  int at = (wave * PARTS + part) * R, parity = 0;
  constexpr int64_t kOn = BACK ? -1 : 1;
  const int64_t row0 = BACK ? (int64_t)span.end - 1 - at : (int64_t)span.first + at;
  const T* gate_at = reinterpret_cast<const T*>(p.gate) + row0 * p.gate_row + c;
  const T* v_at = reinterpret_cast<const T*>(p.v) + row0 * p.v_row + c;
  const T* dh_at = BACK ? reinterpret_cast<const T*>(p.dh) + row0 * p.dh_row + c : nullptr;
  const T* h_at = BACK ? reinterpret_cast<const T*>(p.h_in) + (row0 - 1) * p.h_in_row + c : nullptr;
  T* out_at = reinterpret_cast<T*>(p.h) + row0 * p.h_row + c;
  T* dgate_at = BACK ? reinterpret_cast<T*>(p.dgate) + row0 * p.dgate_row + c : nullptr;
  auto request = [&](int from) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < R; ++j)
      if (from + j < length && n > 0) {
        load_channels<VEC>(ahead[j].gate, gate_at + j * kOn * p.gate_row, n, p.gate);
        if constexpr (!BACK || MODE != COMPOSE) load_channels<VEC>(ahead[j].v, v_at + j * kOn * p.v_row, n, p.v);
        if constexpr (BACK) load_channels<VEC>(ahead[j].dh, dh_at + j * kOn * p.dh_row, n, p.dh);
        if constexpr (BACK && MODE != COMPOSE) {
          if (from + j < length - 1 || span.first > all.first) load_channels<VEC>(ahead[j].h, h_at + j * kOn * p.h_in_row, n, p.h_in);
        }
      } else {
        // past the end a gate that is open, and nothing else: such a row leaves what comes to it as it is
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
          constexpr uint32_t kOpen = sizeof(T) == 4 ? 0x7F800000u : 0x7F807F80u;
          ahead[j].gate.q[i] = (u32x4_t){kOpen, kOpen, kOpen, kOpen};
          ahead[j].v.q[i] = ahead[j].dh.q[i] = (u32x4_t){0, 0, 0, 0};
        }
      }
    gate_at += PASS * kOn * p.gate_row;
    v_at += PASS * kOn * p.v_row;
    if constexpr (BACK) {
      dh_at += PASS * kOn * p.dh_row;
      h_at += PASS * kOn * p.h_in_row;
    }
  };
  // CUT: the state of sequence s that comes to its first row; kept aside by the first launch, as the second one may write `last` over it
  auto entering = [&](int s, float (&v)[8]) __attribute__((always_inline)) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = 0.0f;
    const float* from = BACK ? p.dlast : p.initial;
    if (from == nullptr || n <= 0) return;
    float* aside = p.aside + (int64_t)s * p.width + c;
    if constexpr (MODE == COMPOSE) {
      load8(from + s * (BACK ? p.dlast_row : p.initial_row) + c, n, v);
      store8(aside, n, v);
    } else {
      load8(aside, n, v);
    }
  };
  request(at);
  if constexpr (MODE == APPLY) {
    // the parts before this one: a wavefront composes its share of them, then each those of all
    const int each = (slot + NW - 1) / NW, q1 = min(slot, (wave + 1) * each);
    float a = 1.0f, b = 0.0f;
    if (owns) {
#pragma unroll 8
      for (int q = wave * each; q < q1; ++q) compose<true>(a, b, joint[(int64_t)q * p.width]);
    }
    if (lane < CH) *reinterpret_cast<float2*>(&total[1][wave][own][0]) = make_float2(a, b);
    __syncthreads();
#pragma unroll
    for (int q = 0; q < NW; ++q) compose<true>(product, state, *reinterpret_cast<const float2*>(&total[1][q][own][0]));
  }
  for (int base = 0; base < length; base += PASS, at += PASS, parity ^= 1) {
    if constexpr (CUT) {
      if (base % kTableRows == 0) {
        __syncthreads();
        for (int i = tid; i < kTableRows; i += NW * kWave) head[i] = tail[i] = -1;
        __syncthreads();
        for (int i = tid; i < p.sequences; i += NW * kWave) {
          const Span q = span_of(p, i);
          if (q.end <= q.first) continue;
          const int from = (BACK ? span.end - q.end : q.first - span.first) - base, to = (BACK ? span.end - 1 - q.first : q.end - 1 - span.first) - base;
          if ((unsigned)from < (unsigned)kTableRows) head[from] = i;
          if ((unsigned)to < (unsigned)kTableRows) tail[to] = i;
        }
        __syncthreads();
      }
    }
    // forward: u = (1 - f) v; backward: u = dh, w = (1 - f) (h_{t-1} - v)
    float f[R][8], u[R][8], rest[BACK ? R : 1][8], w[BACK ? R : 1][8], a[8], b[8];
    int first_of[R], last_of[R];         // CUT: the sequence whose first row, as the scan goes, this is, and whose last row
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      a[e] = 1.0f;
      b[e] = 0.0f;
    }
#pragma unroll
    for (int j = 0; j < R; ++j) {
      if constexpr (CUT) {
        const bool row = at + j < length;
        first_of[j] = row ? head[(at + j) % kTableRows] : -1;
        last_of[j] = row ? tail[(at + j) % kTableRows] : -1;
        if (first_of[j] >= 0) {
          entering(first_of[j], b);
#pragma unroll
          for (int e = 0; e < 8; ++e) a[e] = -1.0f;
        }
      }
      if constexpr (!VEC) {
        place_channels(ahead[j].gate, n);
        if constexpr (!BACK || MODE != COMPOSE) place_channels(ahead[j].v, n);
        if constexpr (BACK) place_channels(ahead[j].dh, n);
        if constexpr (BACK && MODE != COMPOSE) place_channels(ahead[j].h, n);
      }
      float past[8];
      if constexpr (BACK && MODE != COMPOSE) {
#pragma unroll
        for (int e = 0; e < 8; ++e) past[e] = raw_at(ahead[j].h, e);
        const int s = CUT ? last_of[j] : at + j == length - 1 ? sequence : -1;
        if (s >= 0) {                                      // the sequence's first row
#pragma unroll
          for (int e = 0; e < 8; ++e) past[e] = 0.0f;
          if (p.initial != nullptr && n > 0) load8(p.initial + s * p.initial_row + c, n, past);
        }
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float r;
        gates(raw_at(ahead[j].gate, e), f[j][e], r);
        if constexpr (BACK) {
          u[j][e] = raw_at(ahead[j].dh, e);
          if constexpr (MODE != COMPOSE) {
            rest[j][e] = r;
            w[j][e] = r * (past[e] - raw_at(ahead[j].v, e));
          }
          b[e] = f[j][e] * (u[j][e] + b[e]);
        } else {
          u[j][e] = r * raw_at(ahead[j].v, e);
          b[e] = fmaf(f[j][e], b[e], u[j][e]);
        }
        a[e] = CUT && a[e] < 0.0f ? -1.0f : a[e] * f[j][e];
      }
    }
    request(at + PASS);
    float* to = &composed[wave][part][cl][0];
#pragma unroll
    for (int e = 0; e < 8; e += 2) *reinterpret_cast<float4*>(to + 2 * e) = make_float4(a[e], b[e], a[e + 1], b[e + 1]);
    __builtin_amdgcn_wave_barrier();
    // of a channel: what lies before each of the lanes' rows, then that of the wavefront as a whole
    float before_a[PARTS], before_b[PARTS], sum_a = 1.0f, sum_b = 0.0f;
#pragma unroll
    for (int q = 0; q < PARTS; ++q) {
      before_a[q] = sum_a;
      before_b[q] = sum_b;
      compose<CUT>(sum_a, sum_b, *reinterpret_cast<const float2*>(&composed[wave][q][own][0]));
    }
    if (lane < CH) *reinterpret_cast<float2*>(&total[parity][wave][own][0]) = make_float2(sum_a, sum_b);
    __syncthreads();
    float mine = state;
#pragma unroll
    for (int q = 0; q < NW; ++q) {
      mine = q == wave ? state : mine;
      compose<CUT>(product, state, *reinterpret_cast<const float2*>(&total[parity][q][own][0]));
    }
    if constexpr (MODE == COMPOSE) continue;
    float* states = &composed[wave][0][0][0];              // [PARTS][CH]
    if (lane < CH) {
#pragma unroll
      for (int q = 0; q < PARTS; ++q) {
        float none = 1.0f, x = mine;
        compose<CUT>(none, x, make_float2(before_a[q], before_b[q]));
        states[q * CH + own] = x;
      }
    }
    __builtin_amdgcn_wave_barrier();
    float h[8];
#pragma unroll
    for (int e = 0; e < 8; e += 4) {
      const float4 x = *reinterpret_cast<const float4*>(states + part * CH + cl + e);
      h[e] = x.x;
      h[e + 1] = x.y;
      h[e + 2] = x.z;
      h[e + 3] = x.w;
    }
#pragma unroll
    for (int j = 0; j < R; ++j)
      if (at + j < length && n > 0) {
        if constexpr (CUT) {
          if (first_of[j] >= 0) entering(first_of[j], h);
        }
        if constexpr (BACK) {
          float dv[8], dgate[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float g = u[j][e] + h[e];
            dv[e] = rest[j][e] * g;
            h[e] = f[j][e] * g;
            dgate[e] = w[j][e] * h[e];
          }
          store8(out_at + j * kOn * p.h_row, VEC ? 8 : n, dv);
          store8(dgate_at + j * kOn * p.dgate_row, VEC ? 8 : n, dgate);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) h[e] = fmaf(f[j][e], h[e], u[j][e]);
          store8(out_at + j * kOn * p.h_row, VEC ? 8 : n, h);
        }
        if constexpr (CUT) {
          if (last_of[j] >= 0 && p.last != nullptr) store8(p.last + last_of[j] * p.last_row + c, n, h);
        }
      }
    out_at += PASS * kOn * p.h_row;
    if constexpr (BACK) dgate_at += PASS * kOn * p.dgate_row;
    __builtin_amdgcn_wave_barrier();
  }
  if (wave == 0 && lane < CH && owns) {
    if (MODE == COMPOSE) joint[(int64_t)slot * p.width] = make_float2(product, state);
    if (MODE == WHOLE && p.last != nullptr) p.last[sequence * p.last_row + c_wg + own] = state;
  }
}

// Sequences of one row: a token of each.
template <typename T, bool BACK> __global__ void __launch_bounds__(kThreads) scan_step_kernel(ScanArgs p, int lanes_log2) {
  const int lanes = 1 << lanes_log2, slots = kThreads >> lanes_log2;
  for (int64_t row = (int64_t)blockIdx.x * slots + (threadIdx.x >> lanes_log2); row < p.rows; row += (int64_t)gridDim.x * slots)
    for (int c = (threadIdx.x & (lanes - 1)) * 8; c < p.width; c += lanes * 8) {
      const int n = p.width - c;
      float gate[8], v[8], state[8] = {0, 0, 0, 0, 0, 0, 0, 0}, dlast[8] = {0, 0, 0, 0, 0, 0, 0, 0}, dh[8], out[8];
      load8(reinterpret_cast<const T*>(p.gate) + row * p.gate_row + c, n, gate);
      load8(reinterpret_cast<const T*>(p.v) + row * p.v_row + c, n, v);
      if (p.initial != nullptr) load8(p.initial + row * p.initial_row + c, n, state);
      if constexpr (BACK) {
        load8(reinterpret_cast<const T*>(p.dh) + row * p.dh_row + c, n, dh);
        if (p.dlast != nullptr) load8(p.dlast + row * p.dlast_row + c, n, dlast);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float f, rest;
        gates(gate[e], f, rest);
        if constexpr (BACK) {
          const float g = dh[e] + dlast[e];
          v[e] = f * rest * (state[e] - v[e]) * g;
          out[e] = rest * g;
          state[e] = f * g;
        } else {
          out[e] = state[e] = fmaf(f, state[e], rest * v[e]);
        }
      }
      store8(reinterpret_cast<T*>(p.h) + row * p.h_row + c, n, out);
      if constexpr (BACK) store8(reinterpret_cast<T*>(p.dgate) + row * p.dgate_row + c, n, v);
      if (p.last != nullptr) store8(p.last + row * p.last_row + c, n, state);
    }
}

// Sequences first .. first + n of p.
template <typename T> ScanArgs sequences_of(const ScanArgs& p, int first, int n) {
  ScanArgs q = p;
  q.sequences = n;
  q.clear = 0;
  if (p.starts != nullptr) {
    q.starts += first;
  } else {
    const int64_t length = p.rows / p.sequences, row = first * length;
    q.rows = n * length;
    auto on = [&](auto& at, int64_t distance) {
      if (at != nullptr) at = (decltype(+at))((const T*)at + row * distance);
    };
    on(q.v, p.v_row);
    on(q.gate, p.gate_row);
    on(q.h_in, p.h_in_row);
    on(q.dh, p.dh_row);
    on(q.h, p.h_row);
    on(q.dgate, p.dgate_row);
  }
  if (p.initial != nullptr) q.initial += first * p.initial_row;
  if (p.dlast != nullptr) q.dlast += first * p.dlast_row;
  if (p.last != nullptr) q.last += first * p.last_row;
  return q;
}
template <typename T, bool BACK> __global__ void __launch_bounds__(kThreads) clear_kernel(ScanArgs p) { clear_rest<T, BACK, WHOLE>(p, (int)blockIdx.x); }
// An axis of a grid holds fewer than 2^32 threads, and a launch of more is cut without an error: more sequences than that go by several launches.
constexpr int kMostWorkgroups = 1 << 22;
template <typename T, bool BACK, int NW, int R, int CL, bool VEC, int OCC> hipError_t launch_in_turn(const ScanArgs& p, int tiles, hipStream_t s) {
  const int most = kMostWorkgroups / tiles;
  for (int first = 0; first < p.sequences; first += most) {
    const ScanArgs q = sequences_of<T>(p, first, std::min(most, p.sequences - first));
    hipLaunchKernelGGL((scan_kernel<T, BACK, NW, R, CL, VEC, OCC, WHOLE>), dim3((unsigned)tiles * (unsigned)q.sequences), dim3(NW * kWave), 0, s, q, tiles);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  }
  if (p.starts == nullptr || p.clear == 0) return hipSuccess;
  hipLaunchKernelGGL((clear_kernel<T, BACK>), dim3(kClearers), dim3(kThreads), 0, s, p);
  return hipGetLastError();
}

// Rows in hand such that no vector register goes to scratch.  Scalar registers do not all fit: in 22 of these 44 kernels 2 to 105 of them are kept in lanes of vector registers.
template <typename T, bool VEC, int MODE> constexpr bool kLarge = sizeof(T) == 4 && !VEC && MODE == APPLY;
template <typename T, bool BACK, int NW, bool VEC, int MODE, int R = BACK && kLarge<T, VEC, MODE> ? 1 : 2, int CL = kTile / 8>
hipError_t launch_scan(const ScanArgs& p, hipStream_t s) {
  constexpr int OCC = BACK || CL < 8 || kLarge<T, VEC, MODE> ? 2 : 4;
  const int tiles = (p.width + 8 * CL - 1) / (8 * CL);
  if constexpr (MODE == WHOLE) {
    if (p.sequences > kMostWorkgroups / tiles) return launch_in_turn<T, BACK, NW, R, CL, VEC, OCC>(p, tiles, s);
  }
  const unsigned others = MODE != COMPOSE && p.starts != nullptr && (p.clear != 0 || MODE == APPLY) ? kClearers : 0;
  const unsigned grid = (unsigned)tiles * (unsigned)(MODE == WHOLE ? p.sequences : p.parts) + others;
  hipLaunchKernelGGL((scan_kernel<T, BACK, NW, R, CL, VEC, OCC, MODE>), dim3(grid), dim3(NW * kWave), 0, s, p, tiles);
  return hipGetLastError();
}
template <typename T, bool BACK, bool VEC> hipError_t launch_passes(const ScanArgs& p, hipStream_t s) {
  if (p.parts > 1) {
    const hipError_t e = launch_scan<T, BACK, kWaves, VEC, COMPOSE>(p, s);
    return e != hipSuccess ? e : launch_scan<T, BACK, kWaves, VEC, APPLY>(p, s);
  }
  const int64_t workgroups = (int64_t)((p.width + kTile - 1) / kTile) * p.sequences, each = p.rows / p.sequences;
  // one wavefront, where eight would have no rows to walk: 4096 sequences of 12 rows x 512 bf16 24 us, by eight 164.  Where the card has enough of them, equal sequences of up to 64 rows
  // too: 16384 of 17, 32 and 64 rows x 64 bf16 32, 38 and 82 us, by eight 126, 127 and 138 (gradients 46, 67 and 132 of 218, 231 and 243), 1024 of 64 rows 8.8 and 10.7 us, but 256 of
  // them 7.1 and 4.9.  Of packed ones one may be much longer than the others, which a wavefront walks in four times the time that eight take.
  if (each <= 16 || (p.starts == nullptr && each <= 64 && workgroups >= 1024)) return launch_scan<T, BACK, 1, VEC, WHOLE>(p, s);
  // too few workgroups for the card, and walks of some length: half the channels, and for long walks forward twice the rows in hand.  4 sequences of 16384 rows x 2048
  // bf16 330 -> 235 us, gradients 450 -> 397 us, gradients of 3 of 605 rows x 448 fp32 18.9 -> 13.7 us; but 64 of 1024 rows 219 -> 638 us, gradients of 2 packed ones of 900 rows
  // x 1048 17 -> 20 us.  (Odd rows in fp32 backward leave room for one row in hand: 1500 rows x 3001 93 -> 55 us.)
  if (workgroups <= 128 && each >= (p.starts == nullptr ? 256 : 2048)) {
    if constexpr (!BACK) {
      if (each >= 2048) return launch_scan<T, BACK, kWaves, VEC, WHOLE, 4, 4>(p, s);
    }
    return launch_scan<T, BACK, kWaves, VEC, WHOLE, BACK && sizeof(T) == 4 && !VEC ? 1 : 2, 4>(p, s);
  }
  return launch_scan<T, BACK, kWaves, VEC, WHOLE>(p, s);
}

template <typename T, bool BACK> hipError_t launch(const ScanArgs& p, hipStream_t s) {
  if (p.starts == nullptr && p.rows == p.sequences) {
    const int lanes_log2 = lanes_for_row(p.width), slots = kThreads >> lanes_log2;
    const unsigned grid = (unsigned)std::min<int64_t>((p.rows + slots - 1) / slots, 256 * 64);
    hipLaunchKernelGGL((scan_step_kernel<T, BACK>), dim3(grid), dim3(kThreads), 0, s, p, lanes_log2);
    return hipGetLastError();
  }
  const bool vec = p.width % 8 == 0;
  return vec ? launch_passes<T, BACK, true>(p, s) : launch_passes<T, BACK, false>(p, s);
}

}  // namespace

// Parts by what the two ways take, in microseconds: a pass of a workgroup 2, HBM 5.2 TB/s for the rows (and once more for what is composed), a launch more 8.  The
// longest of n packed sequences that are cut at random has 1 + ln n times the rows of the average.
int scan_parts(int sequences, int64_t rows, int width, int element_bytes, bool packed, bool backward) {
  constexpr double kPassTime = 2.0, kLaunch = 8.0, kRate = 5.2e6;
  if (sequences > 4096) return 1;        // a workgroup looks at all of them
  const double tiles = (width + kTile - 1) / kTile, bytes = (double)rows * width * element_bytes;
  const double longest = std::min((double)rows, (double)rows / sequences * (packed ? 1.0 + std::log((double)sequences) : 1.0));
  const double whole = std::max(longest / kPass * kPassTime, (backward ? 6 : 3) * bytes / kRate);
  const int64_t parts = std::min<int64_t>(std::max<int64_t>((int64_t)(512 / tiles), 1), (rows + kPass - 1) / kPass);
  const double passes = std::ceil((double)rows / (double)parts / kPass);
  const double cut = kLaunch + std::max(2.0 * passes * kPassTime, (backward ? 8 : 5) * bytes / kRate);
  return parts > 1 && cut < whole ? (int)parts : 1;
}

hipError_t launch_gated_scan(const ScanArgs& p, bool bf16, bool backward, hipStream_t s) {
  if (bf16) return backward ? launch<uint16_t, true>(p, s) : launch<uint16_t, false>(p, s);
  return backward ? launch<float, true>(p, s) : launch<float, false>(p, s);
}

}  // namespace prsgd
