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

constexpr int kChannels = 64;            // of a workgroup; eight lanes share a row

// sigmoid(x) and sigmoid(-x), neither as a difference from 1
__device__ __forceinline__ void gates(float x, float& f, float& rest) {
  const float e = expf(-fabsf(x)), r = 1.0f / (1.0f + e);
  f = x >= 0.0f ? r : e * r;
  rest = x >= 0.0f ? e * r : r;
}

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

template <typename T, bool BACK, int NW, int R> __global__ void __launch_bounds__(NW * kWave) scan_kernel(ScanArgs p, int tiles) {
  __shared__ float total[NW][2][kChannels], before[NW][kChannels];
  if (blockIdx.x >= (unsigned)(tiles * p.sequences)) {
    clear_rest<T>(p, (int)(blockIdx.x - tiles * p.sequences));
    return;
  }
  const int sequence = blockIdx.x / tiles, c_wg = (blockIdx.x - sequence * tiles) * kChannels;
  const int tid = threadIdx.x, wave = tid / kWave, lane = tid % kWave, part = lane / 8, c = c_wg + lane % 8 * 8, n = p.width - c;
  const Span span = span_of(p, sequence);
  const int length = span.end - span.first;
  float state = 0.0f;                    // threads 0 .. 63: of channel c_wg + tid
  const bool keeps = tid < kChannels && c_wg + tid < p.width;
  if (keeps) {
    if (BACK) state = p.dlast != nullptr ? p.dlast[sequence * p.dlast_row + c_wg + tid] : 0.0f;
    else state = p.initial != nullptr ? p.initial[sequence * p.initial_row + c_wg + tid] : 0.0f;
  }
  for (int base = 0; base < length; base += NW * 8 * R) {
    const int at = base + (wave * 8 + part) * R;           // backward: counted from the sequence's end
    float f[R][8], x[R][8], u[R][8], w[R][8];              // forward: u = (1 - f) v; backward: u = dh, w = h_{t-1} - v
#pragma unroll
    for (int j = 0; j < R; ++j) {
#pragma unroll
      for (int e = 0; e < 8; ++e) f[j][e] = x[j][e] = u[j][e] = w[j][e] = 0.0f;
      if (at + j < length && n > 0) {
        const int64_t row = BACK ? span.end - 1 - (at + j) : span.first + at + j;
        load8(reinterpret_cast<const T*>(p.gate) + row * p.gate_row + c, n, f[j]);
        load8(reinterpret_cast<const T*>(p.v) + row * p.v_row + c, n, x[j]);
        if constexpr (BACK) {
          load8(reinterpret_cast<const T*>(p.dh) + row * p.dh_row + c, n, u[j]);
          if (row > span.first) load8(reinterpret_cast<const T*>(p.h_in) + (row - 1) * p.h_in_row + c, n, w[j]);
          else if (p.initial != nullptr) load8(p.initial + sequence * p.initial_row + c, n, w[j]);
        }
      }
    }
    float a[8], b[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      a[e] = 1.0f;
      b[e] = 0.0f;
    }
#pragma unroll
    for (int j = 0; j < R; ++j)
      if (at + j < length) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          float rest;
          gates(f[j][e], f[j][e], rest);
          if constexpr (BACK) {
            w[j][e] = (w[j][e] - x[j][e]) * rest;
            x[j][e] = rest;
            b[e] = f[j][e] * (u[j][e] + b[e]);
          } else {
            u[j][e] = rest * x[j][e];
            b[e] = fmaf(f[j][e], b[e], u[j][e]);
          }
          a[e] *= f[j][e];
        }
      }
    // of this lane's rows and all before them in the wavefront, then of those before them alone
#pragma unroll
    for (int d = 8; d < kWave; d <<= 1)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float pa = __shfl_up(a[e], d), pb = __shfl_up(b[e], d);
        if (lane >= d) {
          b[e] = fmaf(a[e], pb, b[e]);
          a[e] *= pa;
        }
      }
    if (part == 7) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        total[wave][0][lane % 8 * 8 + e] = a[e];
        total[wave][1][lane % 8 * 8 + e] = b[e];
      }
    }
    __syncthreads();
    if (tid < kChannels) {
#pragma unroll
      for (int q = 0; q < NW; ++q) {
        before[q][tid] = state;
        state = fmaf(total[q][0][tid], state, total[q][1][tid]);
      }
    }
    __syncthreads();
    float h[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float pa = __shfl_up(a[e], 8), pb = __shfl_up(b[e], 8);
      h[e] = before[wave][lane % 8 * 8 + e];
      if (part > 0) h[e] = fmaf(pa, h[e], pb);
    }
#pragma unroll
    for (int j = 0; j < R; ++j)
      if (at + j < length && n > 0) {
        const int64_t row = BACK ? span.end - 1 - (at + j) : span.first + at + j;
        if constexpr (BACK) {
          float dv[8], dgate[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float g = u[j][e] + h[e];
            dv[e] = x[j][e] * g;
            dgate[e] = f[j][e] * w[j][e] * g;
            h[e] = f[j][e] * g;
          }
          store8(reinterpret_cast<T*>(p.h) + row * p.h_row + c, n, dv);
          store8(reinterpret_cast<T*>(p.dgate) + row * p.dgate_row + c, n, dgate);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) h[e] = fmaf(f[j][e], h[e], u[j][e]);
          store8(reinterpret_cast<T*>(p.h) + row * p.h_row + c, n, h);
        }
      }
  }
  if (keeps && p.last != nullptr) p.last[sequence * p.last_row + c_wg + tid] = state;
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

template <typename T, bool BACK> hipError_t launch(const ScanArgs& p, hipStream_t s) {
  if (p.starts == nullptr && p.rows == p.sequences) {
    const int lanes_log2 = lanes_for_row(p.width), slots = kThreads >> lanes_log2;
    const unsigned grid = (unsigned)std::min<int64_t>((p.rows + slots - 1) / slots, 256 * 64);
    hipLaunchKernelGGL((scan_step_kernel<T, BACK>), dim3(grid), dim3(kThreads), 0, s, p, lanes_log2);
    return hipGetLastError();
  }
  const int tiles = (p.width + kChannels - 1) / kChannels;
  const dim3 grid((unsigned)tiles * (unsigned)p.sequences + (p.starts != nullptr && p.clear != 0 ? kClearers : 0));
  constexpr int R = BACK ? 2 : 4;
  if (p.rows / p.sequences > 8 * R) hipLaunchKernelGGL((scan_kernel<T, BACK, 8, R>), grid, dim3(8 * kWave), 0, s, p, tiles);
  else hipLaunchKernelGGL((scan_kernel<T, BACK, 1, R>), grid, dim3(kWave), 0, s, p, tiles);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_gated_scan(const ScanArgs& p, bool bf16, bool backward, hipStream_t s) {
  if (bf16) return backward ? launch<uint16_t, true>(p, s) : launch<uint16_t, false>(p, s);
  return backward ? launch<float, true>(p, s) : launch<float, false>(p, s);
}

}  // namespace prsgd
