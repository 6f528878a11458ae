// Rows of the workers' tables by token, and the tables' gradients by sorted tokens.
//   y[r] = scale T[token[r]],   dT[v] = scale * sum of dy[r] over the rows r whose token is v
// Bound by HBM: a lookup moves rows, a gradient reads every row of dy once and writes every row of dT, mostly zeros, once.  So that a row of
// dT has one writer and its sum one order, tokens are sorted with their rows (equal tokens stay in order): tiles of 2048 in LDS, then each
// token finds its place by binary search in the other tiles.  Text has a few tokens that are a large share of all: sorted tokens are cut into chunks, a
// workgroup each, which sum what of a run passes their ends; a row of dT then adds its own rows of dy, or such sums.
#include <algorithm>

#include "orth_rows.h"
#include "prsgd_token_internal.h"

namespace prsgd {

namespace {

constexpr int kTileBits = 11;
static_assert(1 << kTileBits == kSortTile, "place in a tile");
static_assert((uint64_t)(kMaxClasses + 1) << kTileBits < 0xFFFFFFFFull, "a token and its place in its tile fit 32 bits, with a value to spare");
constexpr uint32_t kNoKey = 0xFFFFFFFFu;
constexpr int kLeastChunk = 64;

template <typename T> __global__ void __launch_bounds__(kThreads) embedding_kernel(EmbeddingArgs p, int lanes_log2) {
  const int lanes = 1 << lanes_log2, slots = kThreads >> lanes_log2;
  const int64_t rows = p.rows * p.workers;
  for (int64_t row = (int64_t)blockIdx.x * slots + (threadIdx.x >> lanes_log2); row < rows; row += (int64_t)gridDim.x * slots) {
    const int token = p.tokens[row];
    const bool real = (unsigned)token < (unsigned)p.classes;
    const T* from = reinterpret_cast<const T*>(p.table) + (int64_t)((uint32_t)row / (uint32_t)p.rows) * p.table_gs + (int64_t)(real ? token : 0) * p.table_row;
    for (int c = (threadIdx.x & (lanes - 1)) * 8; c < p.width; c += lanes * 8) {
      float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
      if (real) load8(from + c, p.width - c, v);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = real ? v[e] * p.scale : 0.0f;   // a scale of infinity leaves padding alone
      store8(reinterpret_cast<T*>(p.y) + row * p.y_row + c, p.width - c, v);
    }
  }
}

// ---- sorting -----------------------------------------------------------------------------------

// A tile's tokens in order, each above its place in the tile; what is no token is above all that are.  Also clears the runs.
__global__ void __launch_bounds__(kSortTile / 2) sort_tiles_kernel(EmbeddingArgs p, EmbeddingPlan plan, char* ws) {
  __shared__ uint32_t key[kSortTile];
  const int64_t g = blockIdx.y, first = (int64_t)blockIdx.x * kSortTile;
  const int n = (int)min((int64_t)kSortTile, p.rows - first), t = threadIdx.x, threads = blockDim.x;
  const int32_t* tokens = p.tokens + g * p.rows + first;
  for (int i = t; i < 2 * threads; i += threads) {
    uint32_t k = kNoKey;
    if (i < n) {
      const int32_t v = tokens[i];
      k = ((unsigned)v < (unsigned)p.classes ? (uint32_t)v : (uint32_t)p.classes) << kTileBits | (uint32_t)i;
    }
    key[i] = k;
  }
  int2* runs = reinterpret_cast<int2*>(ws + plan.runs) + g * p.classes;
  for (int i = blockIdx.x * threads + t; i < p.classes; i += gridDim.x * threads) runs[i] = make_int2(0, 0);
  __syncthreads();
  // bitonic: pairs j apart within blocks of k
  for (int k = 2; k <= 2 * threads; k <<= 1)
    for (int j = k >> 1; j > 0; j >>= 1) {
      const int lo = ((t & ~(j - 1)) << 1) | (t & (j - 1)), hi = lo | j;
      const uint32_t a = key[lo], b = key[hi];
      if ((a > b) == ((lo & k) == 0)) {
        key[lo] = b;
        key[hi] = a;
      }
      __syncthreads();
    }
  if (plan.tiles == 1) {
    int* order = reinterpret_cast<int*>(ws + plan.order) + g * p.rows;
    int* sorted = reinterpret_cast<int*>(ws + plan.sorted) + g * p.rows;
    for (int i = t; i < n; i += threads) {
      order[i] = (int)(key[i] & (kSortTile - 1));
      sorted[i] = (int)(key[i] >> kTileBits);
    }
  } else {
    uint32_t* keys = reinterpret_cast<uint32_t*>(ws + plan.keys) + (g * plan.tiles + blockIdx.x) * kSortTile;
    for (int i = t; i < kSortTile; i += threads) keys[i] = key[i];
  }
}

// Place of a tile's tokens among those of all tiles: equal ones of earlier tiles come before, of later ones behind.
__global__ void __launch_bounds__(kSortTile / 2) place_tokens_kernel(EmbeddingArgs p, EmbeddingPlan plan, char* ws) {
  __shared__ uint32_t other[2][kSortTile];
  const int64_t g = blockIdx.y;
  const int t = threadIdx.x, mine = blockIdx.x, n = (int)min((int64_t)kSortTile, p.rows - (int64_t)mine * kSortTile);
  const uint32_t* keys = reinterpret_cast<const uint32_t*>(ws + plan.keys) + g * plan.tiles * kSortTile;
  uint32_t k[2];
  int rank[2];
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    k[e] = keys[(int64_t)mine * kSortTile + 2 * t + e];
    rank[e] = 2 * t + e;
  }
  for (int b = 0, stage = 0; b < plan.tiles; ++b) {
    if (b == mine) continue;
#pragma unroll
    for (int e = 0; e < 2; ++e) other[stage][e * (kSortTile / 2) + t] = keys[(int64_t)b * kSortTile + e * (kSortTile / 2) + t];
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const uint32_t below = ((k[e] >> kTileBits) + (b < mine ? 1u : 0u)) << kTileBits;
      int lo = 0;
#pragma unroll
      for (int half = kSortTile / 2; half > 0; half >>= 1) lo += other[stage][lo + half - 1] < below ? half : 0;
      rank[e] += lo + (other[stage][lo] < below ? 1 : 0);
    }
    stage ^= 1;
  }
  int* order = reinterpret_cast<int*>(ws + plan.order) + g * p.rows;
  int* sorted = reinterpret_cast<int*>(ws + plan.sorted) + g * p.rows;
#pragma unroll
  for (int e = 0; e < 2; ++e)
    if (2 * t + e < n) {
      order[rank[e]] = mine * kSortTile + (int)(k[e] & (kSortTile - 1));
      sorted[rank[e]] = (int)(k[e] >> kTileBits);
    }
}

// ---- sums --------------------------------------------------------------------------------------

constexpr int kSlice = 512;              // columns of a workgroup's sums: eight a lane, rows dealt to the wavefronts
__host__ __device__ constexpr int part_width(int width) { return (width + 7) / 8 * 8; }

// Where the runs of a chunk of sorted tokens begin and end, and the sums of those that pass its ends: of the chunk's first run (part 0) and of
// its last one if that is another (part 1).
template <typename T> __global__ void __launch_bounds__(kThreads) chunk_sums_kernel(EmbeddingArgs p, EmbeddingPlan plan, char* ws) {
  __shared__ float share[kThreads / kWave][kSlice];
  const int64_t g = blockIdx.z;
  const int n = (int)p.rows, c0 = blockIdx.x * plan.chunk, c1 = min(n, c0 + plan.chunk), t = threadIdx.x;
  const int* sorted = reinterpret_cast<const int*>(ws + plan.sorted) + g * p.rows;
  const int* order = reinterpret_cast<const int*>(ws + plan.order) + g * p.rows;
  int2* runs = reinterpret_cast<int2*>(ws + plan.runs) + g * p.classes;
  const int first = sorted[c0], last = sorted[c1 - 1];
  const bool on = c1 < n && sorted[c1] == last;            // the last run goes on
  const bool part0 = first < p.classes && ((c0 > 0 && sorted[c0 - 1] == first) || (on && first == last));
  const bool part1 = last < p.classes && on && first != last;
  int firsts = 0, lasts = 0;                               // tokens of the first and of the last run in the chunk
  for (int i0 = c0; i0 < c1; i0 += kThreads) {
    const int i = i0 + t, v = i < c1 ? sorted[i] : -1;
    if (blockIdx.y == 0 && i < c1 && v < p.classes) {
      if (i == 0 || sorted[i - 1] != v) runs[v].x = i;
      if (i == n - 1 || sorted[i + 1] != v) runs[v].y = i + 1;
    }
    firsts += __syncthreads_count(v == first);
    lasts += __syncthreads_count(v == last);
  }
  const int wave = t / kWave, lane = t % kWave, c = blockIdx.y * kSlice + lane * 8;
  for (int part = 0; part < 2; ++part) {
    if (part == 0 ? !part0 : !part1) continue;
    const int from = part == 0 ? c0 : c1 - lasts, to = part == 0 ? c0 + firsts : c1;
    float sum[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (c < p.width)
      for (int i = from + wave; i < to; i += kThreads / kWave) {
        float v[8];
        load8(reinterpret_cast<const T*>(p.y) + (g * p.rows + order[i]) * p.y_row + c, p.width - c, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[e] += v[e];
      }
#pragma unroll
    for (int e = 0; e < 8; ++e) share[wave][lane * 8 + e] = sum[e];
    __syncthreads();
    float* out = reinterpret_cast<float*>(ws + plan.parts) + ((g * plan.chunks + blockIdx.x) * 2 + part) * part_width(p.width);
    for (int j = t; j < kSlice; j += kThreads) {
      float s = share[0][j];
#pragma unroll
      for (int w = 1; w < kThreads / kWave; ++w) s += share[w][j];
      if (blockIdx.y * kSlice + j < part_width(p.width)) out[blockIdx.y * kSlice + j] = s;
    }
    __syncthreads();
  }
}

template <typename T> __global__ void __launch_bounds__(kThreads) table_rows_kernel(EmbeddingArgs p, EmbeddingPlan plan, const char* ws, int lanes_log2) {
  const int lanes = 1 << lanes_log2, slots = kThreads >> lanes_log2;
  const int64_t rows = (int64_t)p.classes * p.workers;
  for (int64_t row = (int64_t)blockIdx.x * slots + (threadIdx.x >> lanes_log2); row < rows; row += (int64_t)gridDim.x * slots) {
    const int64_t g = row / p.classes;
    const int2 run = reinterpret_cast<const int2*>(ws + plan.runs)[row];
    const int* order = reinterpret_cast<const int*>(ws + plan.order) + g * p.rows;
    const int q0 = run.x / plan.chunk, q1 = run.y > run.x ? (run.y - 1) / plan.chunk : q0;
    for (int c = (threadIdx.x & (lanes - 1)) * 8; c < p.width; c += lanes * 8) {
      float sum[8] = {0, 0, 0, 0, 0, 0, 0, 0};
      if (q0 == q1) {
        for (int i = run.x; i < run.y; ++i) {
          float v[8];
          load8(reinterpret_cast<const T*>(p.y) + (g * p.rows + order[i]) * p.y_row + c, p.width - c, v);
#pragma unroll
          for (int e = 0; e < 8; ++e) sum[e] += v[e];
        }
      } else {
        const float* parts = reinterpret_cast<const float*>(ws + plan.parts) + g * plan.chunks * 2 * part_width(p.width) + c;
        for (int q = q0; q <= q1; ++q) {
          float v[8];
          load8(parts + (int64_t)(q * 2 + (q * plan.chunk < run.x ? 1 : 0)) * part_width(p.width), 8, v);
#pragma unroll
          for (int e = 0; e < 8; ++e) sum[e] += v[e];
        }
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) sum[e] *= p.scale;
      store8(reinterpret_cast<T*>(p.dtable) + g * p.dtable_gs + (row - g * p.classes) * p.dtable_row + c, p.width - c, sum);
    }
  }
}

template <typename K> hipError_t launch_rows(K kernel_of, int64_t rows, int width) {
  const int lanes_log2 = lanes_for_row(width), slots = kThreads >> lanes_log2;
  kernel_of(dim3((unsigned)std::min<int64_t>((rows + slots - 1) / slots, 256 * 64)), lanes_log2);
  return hipGetLastError();
}

template <typename T> hipError_t backward(const EmbeddingArgs& p, const EmbeddingPlan& plan, char* ws, hipStream_t s) {
  int threads = kWave;
  while (threads < kSortTile / 2 && 2 * threads < p.rows) threads *= 2;
  const dim3 tiles((unsigned)plan.tiles, (unsigned)p.workers);
  hipLaunchKernelGGL(sort_tiles_kernel, tiles, dim3(threads), 0, s, p, plan, ws);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (plan.tiles > 1) {
    hipLaunchKernelGGL(place_tokens_kernel, tiles, dim3(kSortTile / 2), 0, s, p, plan, ws);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  if (plan.chunks > 0)
    hipLaunchKernelGGL(chunk_sums_kernel<T>, dim3((unsigned)plan.chunks, (unsigned)((p.width + kSlice - 1) / kSlice), (unsigned)p.workers), dim3(kThreads),
                       0, s, p, plan, ws);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  return launch_rows([&](dim3 grid, int lanes_log2) {
    hipLaunchKernelGGL(table_rows_kernel<T>, grid, dim3(kThreads), 0, s, p, plan, (const char*)ws, lanes_log2);
  }, (int64_t)p.classes * p.workers, p.width);
}

}  // namespace

hipError_t launch_embedding(const EmbeddingArgs& p, bool bf16, hipStream_t s) {
  return launch_rows([&](dim3 grid, int lanes_log2) {
    if (bf16) hipLaunchKernelGGL(embedding_kernel<uint16_t>, grid, dim3(kThreads), 0, s, p, lanes_log2);
    else hipLaunchKernelGGL(embedding_kernel<float>, grid, dim3(kThreads), 0, s, p, lanes_log2);
  }, p.rows * p.workers, p.width);
}

EmbeddingPlan embedding_plan(int workers, int64_t rows, int classes, int width) {
  EmbeddingPlan e{};
  e.tiles = (int)std::max<int64_t>(1, (rows + kSortTile - 1) / kSortTile);
  // chunks grow with the rows, so that the commonest token's row has at most 256 of them to add
  e.chunk = (int)std::max<int64_t>(kLeastChunk, ((rows + 255) / 256 + 63) / 64 * 64);
  e.chunks = (int)((rows + e.chunk - 1) / e.chunk);
  size_t at = 0;
  auto take = [&](size_t bytes) { const size_t v = at; at += (bytes + 255) / 256 * 256; return v; };
  const size_t n = (size_t)workers, r = (size_t)rows;
  e.keys = e.tiles > 1 ? take(n * e.tiles * kSortTile * sizeof(uint32_t)) : 0;
  e.order = take(n * r * sizeof(int));
  e.sorted = take(n * r * sizeof(int));
  e.runs = take(n * classes * sizeof(int2));
  e.parts = take(n * e.chunks * 2 * part_width(width) * sizeof(float));
  e.total = at;
  return e;
}

hipError_t launch_embedding_backward(const EmbeddingArgs& p, const EmbeddingPlan& plan, char* ws, bool bf16, hipStream_t s) {
  return bf16 ? backward<uint16_t>(p, plan, ws, s) : backward<float>(p, plan, ws, s);
}

}  // namespace prsgd
