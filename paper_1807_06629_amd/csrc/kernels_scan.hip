// Gated linear recurrence over packed sequences, forward and backward.
//   f = sigmoid(gate),  h_t = f_t h_{t-1} + (1 - f_t) v_t
//   c_t = f_t (dh_t + c_{t+1}) (c behind the last row is dlast),  g_t = dh_t + c_{t+1},
//   dv_t = (1 - f_t) g_t,  dgate_t = f_t (1 - f_t) (h_{t-1} - v_t) g_t,  dinitial = c of the first row
// Both are x -> a x + b along a sequence, the second one from its end.  A workgroup has 64 channels of one sequence and walks along it: every lane
// holds R rows of eight channels, composes them, and lanes, then wavefronts, compose theirs, so that a pass over NW * 8 * R rows reads
// each of them once and needs no workgroup to wait for another.  States and compositions are fp32.
#include <algorithm>

#include "orth_rows.h"
#include "prsgd_token_internal.h"

namespace prsgd {

namespace {

// sigmoid(x) and sigmoid(-x), neither as a difference from 1.  The hardware's base-2 exponential takes an argument that is rounded, which leaves 1.3 |x| 2^-24 of
// exp(-|x|), and its quotient is good to one rounding.  For gates in bf16, which are off by |x| 2^-9 themselves, that is nothing; for fp32 the rounding is made good.
template <typename T> __device__ __forceinline__ void gates(float x, float& f, float& rest) {
  float e;
  if constexpr (sizeof(T) == 2) {
    e = __builtin_amdgcn_exp2f(fabsf(x) * -1.44269502f);
  } else {
    const float t = fabsf(x) > 128.0f ? 128.0f : fabsf(x);       // NaN stays; from 104 on e is 0 anyway
    const float hi = t * -1.44269502f, lo = fmaf(t, -1.44269502f, -hi), power = __builtin_amdgcn_exp2f(hi);
    e = fmaf(power * 0.693147181f, lo, power);
  }
  const float r = __builtin_amdgcn_rcpf(1.0f + e), s = e * r;
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

// Zeros in the rows that no sequence has, by workgroups behind those of the sequences.
constexpr int kClearers = 64;
template <typename T> __device__ __forceinline__ void clear_rest(const ScanArgs& p, int block) {
  const int first = min(max(p.starts[0], 0), (int)p.rows), end = min(max(p.starts[p.sequences], first), (int)p.rows);
  const float none[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  for (int i = block; i < first + ((int)p.rows - end); i += kClearers) {
    const int64_t row = i < first ? i : end + (i - first);
    for (int c = threadIdx.x * 8; c < p.width; c += blockDim.x * 8) {
      if ((p.clear & 1) != 0) store8(reinterpret_cast<T*>(p.h) + row * p.h_row + c, p.width - c, none);
      if ((p.clear & 2) != 0) store8(reinterpret_cast<T*>(p.dgate) + row * p.dgate_row + c, p.width - c, none);
    }
  }
}

// Eight channels of a row as they lie in memory, and of it n that exist.
template <typename T> struct Raw { u32x4_t q[sizeof(T) / 2]; };
template <typename T> __device__ __forceinline__ float raw_at(const Raw<T>& v, int e) {
  if constexpr (sizeof(T) == 4) return __uint_as_float(v.q[e / 4][e % 4]);
  else return __uint_as_float((e & 1) != 0 ? v.q[0][e / 2] & 0xFFFF0000u : v.q[0][e / 2] << 16);
}
// VEC: rows are whole eights, so that no lane has a part of one
template <typename T, bool VEC> __device__ __forceinline__ void raw_load(Raw<T>& v, const T* p, int n) {
  if (VEC || n >= 8) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) v.q[i] = reinterpret_cast<const Packed16<(int)sizeof(T)>*>(p + i * (16 / (int)sizeof(T)))->v;
  } else {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) v.q[i] = (u32x4_t){0, 0, 0, 0};
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < n) {
        if constexpr (sizeof(T) == 4) v.q[e / 4][e % 4] = __float_as_uint(p[e]);
        else v.q[0][e / 2] |= (uint32_t)p[e] << (16 * (e & 1));
      }
  }
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

// A long sequence may be cut into parts (p.parts), where there are too few workgroups otherwise: the first launch composes each part's rows, the second
// (join_parts_kernel) finds the states in front of the parts, the third is the scan with these.
enum ScanMode { WHOLE = 0, COMPOSE = 1, APPLY = 2 };
__device__ __forceinline__ Span part_of(Span s, int part, int parts) {
  const int each = ((s.end - s.first + parts - 1) / parts + 63) / 64 * 64, from = min(s.first + part * each, s.end);
  return {from, min(from + each, s.end)};
}

// NW wavefronts; CL lanes share a row, R rows a lane.  The next pass's rows are on their way while this one's are composed.
template <typename T, bool BACK, int NW, int R, int CL, bool VEC, int OCC, int MODE> __global__ void __launch_bounds__(NW * kWave, OCC) scan_kernel(ScanArgs p, int tiles) {
  constexpr int CH = 8 * CL, PARTS = kWave / CL, PASS = NW * PARTS * R;
  // compositions of the lanes' rows, then the states in front of them; of a wavefront, which alone reads them
  __shared__ __attribute__((aligned(16))) float composed[NW][PARTS][CH][2];
  __shared__ float total[2][NW][CH][2];
  const int workgroups = tiles * p.sequences * (MODE == WHOLE ? 1 : p.parts);
  if (blockIdx.x >= (unsigned)workgroups) {
    clear_rest<T>(p, (int)(blockIdx.x - workgroups));
    return;
  }
  const int slot = blockIdx.x / tiles, c_wg = (blockIdx.x - slot * tiles) * CH;
  int sequence = MODE == WHOLE ? slot : slot / p.parts;
  const int nth = MODE == WHOLE ? 0 : slot - sequence * p.parts;           // part, counted as the scan goes
  if (MODE == WHOLE && NW > 1 && p.starts != nullptr && p.sequences <= kRanked) sequence = __builtin_amdgcn_readfirstlane(nth_longest<NW * kWave>(p, sequence));
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid / kWave), lane = tid % kWave, part = lane / CL, cl = lane % CL * 8;
  const int c = c_wg + cl, n = p.width - c;
  const Span all = span_of(p, sequence), span = MODE == WHOLE ? all : part_of(all, BACK ? p.parts - 1 - nth : nth, p.parts);
  const int length = span.end - span.first;
  // of channel c_wg + lane % CH, in every wavefront alike
  const int own = lane % CH;
  const bool owns = c_wg + own < p.width;
  float2* joint = MODE == WHOLE ? nullptr : p.joint + (int64_t)slot * p.width + c_wg + own;
  float state = 0.0f;
  if (owns && MODE == APPLY) state = joint->x;
  if (owns && MODE == WHOLE) {
    if (BACK) state = p.dlast != nullptr ? p.dlast[sequence * p.dlast_row + c_wg + own] : 0.0f;
    else state = p.initial != nullptr ? p.initial[sequence * p.initial_row + c_wg + own] : 0.0f;
  }
  float product = 1.0f;                  // COMPOSE: of all f
  struct Rows { Raw<T> gate, v, dh, h; };
  Rows ahead[R];
  // Row `at` of this lane, counted from the sequence's end backward, and what lies one row and one pass further on.
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
        raw_load<T, VEC>(ahead[j].gate, gate_at + j * kOn * p.gate_row, n);
        if constexpr (!BACK || MODE != COMPOSE) raw_load<T, VEC>(ahead[j].v, v_at + j * kOn * p.v_row, n);
        if constexpr (BACK) raw_load<T, VEC>(ahead[j].dh, dh_at + j * kOn * p.dh_row, n);
        if constexpr (BACK && MODE != COMPOSE) {
          if (from + j < length - 1 || span.first > all.first) raw_load<T, VEC>(ahead[j].h, h_at + j * kOn * p.h_in_row, n);
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
  request(at);
  for (int base = 0; base < length; base += PASS, at += PASS, parity ^= 1) {
    // forward: u = (1 - f) v; backward: u = dh, w = (1 - f) (h_{t-1} - v)
    float f[R][8], u[R][8], rest[BACK ? R : 1][8], w[BACK ? R : 1][8], a[8], b[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      a[e] = 1.0f;
      b[e] = 0.0f;
    }
#pragma unroll
    for (int j = 0; j < R; ++j) {
      float past[8];
      if constexpr (BACK && MODE != COMPOSE) {
#pragma unroll
        for (int e = 0; e < 8; ++e) past[e] = raw_at<T>(ahead[j].h, e);
        if (at + j == length - 1 && span.first == all.first) {           // the first row
#pragma unroll
          for (int e = 0; e < 8; ++e) past[e] = 0.0f;
          if (p.initial != nullptr && n > 0) load8(p.initial + sequence * p.initial_row + c, n, past);
        }
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float r;
        gates<T>(raw_at<T>(ahead[j].gate, e), f[j][e], r);
        if constexpr (BACK) {
          u[j][e] = raw_at<T>(ahead[j].dh, e);
          if constexpr (MODE != COMPOSE) {
            rest[j][e] = r;
            w[j][e] = r * (past[e] - raw_at<T>(ahead[j].v, e));
          }
          b[e] = f[j][e] * (u[j][e] + b[e]);
        } else {
          u[j][e] = r * raw_at<T>(ahead[j].v, e);
          b[e] = fmaf(f[j][e], b[e], u[j][e]);
        }
        a[e] *= f[j][e];
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
      const float2 x = *reinterpret_cast<const float2*>(&composed[wave][q][own][0]);
      before_a[q] = sum_a;
      before_b[q] = sum_b;
      sum_b = fmaf(x.x, sum_b, x.y);
      sum_a *= x.x;
    }
    if (lane < CH) *reinterpret_cast<float2*>(&total[parity][wave][own][0]) = make_float2(sum_a, sum_b);
    __syncthreads();
    float mine = state;
#pragma unroll
    for (int q = 0; q < NW; ++q) {
      const float2 x = *reinterpret_cast<const float2*>(&total[parity][q][own][0]);
      mine = q == wave ? state : mine;
      state = fmaf(x.x, state, x.y);
      if (MODE == COMPOSE) product *= x.x;
    }
    if constexpr (MODE == COMPOSE) continue;
    float* states = &composed[wave][0][0][0];              // [PARTS][CH]
    if (lane < CH) {
#pragma unroll
      for (int q = 0; q < PARTS; ++q) states[q * CH + own] = fmaf(before_a[q], mine, before_b[q]);
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
      }
    out_at += PASS * kOn * p.h_row;
    if constexpr (BACK) dgate_at += PASS * kOn * p.dgate_row;
    __builtin_amdgcn_wave_barrier();
  }
  if (wave == 0 && lane < CH && owns) {
    if (MODE == COMPOSE) *joint = make_float2(product, state);
    if (MODE == WHOLE && p.last != nullptr) p.last[sequence * p.last_row + c_wg + own] = state;
  }
}

// The state in front of every part, in the place of the part's composition.
template <bool BACK> __global__ void __launch_bounds__(kThreads) join_parts_kernel(ScanArgs p) {
  const int channels = (p.width + kThreads - 1) / kThreads, sequence = blockIdx.x / channels, c = (blockIdx.x - sequence * channels) * kThreads + threadIdx.x;
  if (c >= p.width) return;
  const float* from = BACK ? p.dlast : p.initial;
  float state = from != nullptr ? from[sequence * (BACK ? p.dlast_row : p.initial_row) + c] : 0.0f;
  float2* joint = p.joint + (int64_t)sequence * p.parts * p.width + c;
#pragma unroll 8
  for (int q = 0; q < p.parts; ++q, joint += p.width) {
    const float2 x = *joint;
    joint->x = state;
    state = fmaf(x.x, state, x.y);
  }
  if (p.last != nullptr) p.last[sequence * p.last_row + c] = state;
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
        gates<T>(gate[e], f, rest);
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

template <typename T, bool BACK, int NW, bool VEC, int MODE> hipError_t launch_scan(const ScanArgs& p, hipStream_t s) {
  constexpr int OCC = BACK ? 2 : 4;
  const int tiles = (p.width + kTile - 1) / kTile;
  const unsigned grid = (unsigned)tiles * (unsigned)p.sequences * (MODE == WHOLE ? 1u : (unsigned)p.parts) +
                        (MODE != COMPOSE && p.starts != nullptr && p.clear != 0 ? kClearers : 0);
  hipLaunchKernelGGL((scan_kernel<T, BACK, NW, 2, kTile / 8, VEC, OCC, MODE>), dim3(grid), dim3(NW * kWave), 0, s, p, tiles);
  return hipGetLastError();
}
template <typename T, bool BACK, bool VEC> hipError_t launch_passes(const ScanArgs& p, hipStream_t s) {
  if (p.parts > 1) {
    hipError_t e = launch_scan<T, BACK, kWaves, VEC, COMPOSE>(p, s);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(join_parts_kernel<BACK>, dim3((unsigned)p.sequences * (unsigned)((p.width + kThreads - 1) / kThreads)), dim3(kThreads), 0, s, p);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    return launch_scan<T, BACK, kWaves, VEC, APPLY>(p, s);
  }
  if (p.rows / p.sequences <= 16) return launch_scan<T, BACK, 1, VEC, WHOLE>(p, s);
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

int scan_parts(int sequences, int64_t rows, int width) {
  const int64_t workgroups = (int64_t)sequences * ((width + kTile - 1) / kTile), passes = rows / sequences / kPass;
  if (workgroups > 64 || passes < 8) return 1;
  return (int)std::min<int64_t>(std::min<int64_t>(512 / workgroups, 64), passes / 2);
}

hipError_t launch_gated_scan(const ScanArgs& p, bool bf16, bool backward, hipStream_t s) {
  if (bf16) return backward ? launch<uint16_t, true>(p, s) : launch<uint16_t, false>(p, s);
  return backward ? launch<float, true>(p, s) : launch<float, false>(p, s);
}

}  // namespace prsgd
