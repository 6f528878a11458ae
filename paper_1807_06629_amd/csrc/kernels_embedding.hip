// Rows of the workers' tables by token, and the tables' gradients by sorted tokens.
//   y[r] = scale T[token[r]],   dT[v] = scale * sum of dy[r] over the rows r whose token is v
// Bound by HBM: a lookup moves rows, a gradient reads every row of dy once and writes every row of dT, mostly zeros, once (named rows twice: zeros are written
// beside the sort, which they take much longer than).  So that a row of dT has one writer and its sum one order, tokens are sorted with their rows (equal tokens stay
// in order): tiles of 2048 in LDS, then each token finds its place by binary search in the other tiles.  Text has a few tokens that are a large share of all: sorted
// tokens are cut into chunks, whose runs a few lanes sum and write; a run that passes a chunk's end leaves its parts, which another launch adds.
// Rows of 8 x 2048 tokens out of 32768 x 1024 bf16 take 10.6 us; the gradient of 8 x 8192 tokens 175 us: zeros 89 (6 TB/s), places 7, sums 67, parts 13.
#include <algorithm>

#include "orth_rows.h"
#include "prsgd_token_internal.h"
#include "row_pieces.h"

namespace prsgd {

namespace {

constexpr int kTileBits = 11;
static_assert(1 << kTileBits == kSortTile, "place in a tile");
static_assert((uint64_t)(kMaxClasses + 1) << kTileBits < 0xFFFFFFFFull, "a token and its place in its tile fit 32 bits, with a value to spare");
constexpr uint32_t kNoKey = 0xFFFFFFFFu;
constexpr int kLeastChunk = 8;

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
      for (int e = 0; e < 8; ++e) v[e] = real ? v[e] * p.scale : 0.0f;   // +0 in padding, also under a negative scale
      store8(reinterpret_cast<T*>(p.y) + row * p.y_row + c, p.width - c, v);
    }
  }
}

// ---- sorting -----------------------------------------------------------------------------------

// Zeros in a worker's rows of dT, by `blocks` workgroups: 16 aligned bytes a lane where rows lie one behind another.
template <typename T> __device__ __forceinline__ void clear_table(const EmbeddingArgs& p, int64_t g, int block, int blocks) {
  constexpr int V = 16 / (int)sizeof(T);
  T* table = reinterpret_cast<T*>(p.dtable) + g * p.dtable_gs;
  const int64_t start = (int64_t)block * blockDim.x + threadIdx.x, step = (int64_t)blocks * blockDim.x;
  if (p.dtable_row == p.width) {
    const int64_t n = (int64_t)p.classes * p.width, front = min((int64_t)((16 - (uintptr_t)table % 16) % 16 / sizeof(T)), n), units = (n - front) / V;
    u32x4_t* at = reinterpret_cast<u32x4_t*>(table + front);
#pragma unroll 4
    for (int64_t i = start; i < units; i += step) at[i] = (u32x4_t){0, 0, 0, 0};
    if (start < front) table[start] = 0;
    if (start < n - front - units * V) table[front + units * V + start] = 0;
  } else {
    const float none[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    const int64_t per_row = (p.width + 7) / 8;
    for (int64_t i = start; i < per_row * p.classes; i += step) {
      const int64_t r = i / per_row, c = (i - r * per_row) * 8;
      store8(table + r * p.dtable_row + c, (int)min(p.width - c, (int64_t)8), none);
    }
  }
}

// A tile's tokens in order, each above its place in the tile; what is no token is above all that are.  Workgroups behind the tiles' clear dT.
template <typename T> __global__ void __launch_bounds__(kSortTile / 2) sort_tiles_kernel(EmbeddingArgs p, EmbeddingPlan plan, char* ws) {
  __shared__ uint32_t key[kSortTile];
  const int64_t g = blockIdx.y, first = (int64_t)blockIdx.x * kSortTile;
  const int t = threadIdx.x, threads = blockDim.x;
  if ((int)blockIdx.x >= plan.tiles) {
    clear_table<T>(p, g, blockIdx.x - plan.tiles, gridDim.x - plan.tiles);
    return;
  }
  const int n = (int)min((int64_t)kSortTile, p.rows - first);
  const int32_t* tokens = p.tokens + g * p.rows + first;
  for (int i = t; i < 2 * threads; i += threads) {
    uint32_t k = kNoKey;
    if (i < n) {
      const int32_t v = tokens[i];
      k = ((unsigned)v < (unsigned)p.classes ? (uint32_t)v : (uint32_t)p.classes) << kTileBits | (uint32_t)i;
    }
    key[i] = k;
  }
  __syncthreads();
  // bitonic: pairs j apart within blocks of k.  Up to 64 apart a wavefront's 64 pairs are 128 keys that no other one has.
  bool across = false;
  for (int k = 2; k <= 2 * threads; k <<= 1)
    for (int j = k >> 1; j > 0; j >>= 1) {
      if (across || j > 64) __syncthreads();
      else __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      across = j > 64;
      const int lo = ((t & ~(j - 1)) << 1) | (t & (j - 1)), hi = lo | j;
      const uint32_t a = key[lo], b = key[hi];
      if ((a > b) == ((lo & k) == 0)) {
        key[lo] = b;
        key[hi] = a;
      }
    }
  __syncthreads();
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

constexpr int kSlice = 8 * kWave;        // columns that a chunk's lanes take, at most
__host__ __device__ constexpr int part_width(int width) { return (width + 7) / 8 * 8; }

// An axis of a grid holds fewer than 2^32 threads, and a launch of more is cut without an error: workgroups lie along two, the last of which may be too many.
constexpr int kGridBits = 22;
dim3 grid_of(int64_t workgroups) {
  const int64_t along = (int64_t)1 << kGridBits;
  return dim3((unsigned)std::min(workgroups, along), (unsigned)((workgroups + along - 1) / along));
}

// A chunk of sorted tokens and a slice of the columns, for lanes_log2 lanes: which these are, and what follows from them.
struct ChunkPlace {
  int64_t g;
  int chunk, c, first, end;              // sorted tokens first .. end - 1; c: this lane's first column
  const int *sorted, *order;
  float* parts;                          // [2][part_width]: of the chunk's first run if it began before, of its last one if it goes on
  __device__ __forceinline__ bool set(const EmbeddingArgs& p, const EmbeddingPlan& plan, char* ws, int lanes_log2) {
    const int lanes = 1 << lanes_log2, slices = (p.width + kSlice - 1) / kSlice;
    const int64_t unit = (int64_t)(blockIdx.y << kGridBits | blockIdx.x) * (kThreads >> lanes_log2) + (threadIdx.x >> lanes_log2), at = unit / slices;
    if (at >= (int64_t)plan.chunks * p.workers) return false;
    g = at / plan.chunks;
    chunk = (int)(at - g * plan.chunks);
    c = (int)(unit - at * slices) * kSlice + (threadIdx.x & (lanes - 1)) * 8;
    first = chunk * plan.chunk;
    end = (int)min(p.rows, (int64_t)first + plan.chunk);
    sorted = reinterpret_cast<const int*>(ws + plan.sorted) + g * p.rows;
    order = reinterpret_cast<const int*>(ws + plan.order) + g * p.rows;
    parts = reinterpret_cast<float*>(ws + plan.parts) + (g * plan.chunks + chunk) * 2 * part_width(p.width) + c;
    return c < p.width;
  }
};
template <typename T> __device__ __forceinline__ void store_row(const EmbeddingArgs& p, const ChunkPlace& at, int token, float (&sum)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) sum[e] *= p.scale;
  store8(reinterpret_cast<T*>(p.dtable) + at.g * p.dtable_gs + (int64_t)token * p.dtable_row + at.c, p.width - at.c, sum);
}

template <typename T> __global__ void __launch_bounds__(kThreads) chunk_sums_kernel(EmbeddingArgs p, EmbeddingPlan plan, char* ws, int lanes_log2) {
  constexpr int U = 8;                   // rows on their way
  ChunkPlace at;
  if (!at.set(p, plan, ws, lanes_log2)) return;
  const int n = p.width - at.c, before = at.first > 0 ? at.sorted[at.first - 1] : -1, behind = at.end < p.rows ? at.sorted[at.end] : -1;
  const T* dy = reinterpret_cast<const T*>(p.y) + at.g * p.rows * p.y_row + at.c;
  int token[U], row[U], now = -1;        // the run that is being summed
  bool from_before = false;
  float sum[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  auto places = [&](int i) __attribute__((always_inline)) {
#pragma unroll
    for (int k = 0; k < U; ++k) {
      const int j = min(i + k, at.end - 1);
      token[k] = i + k < at.end ? at.sorted[j] : -1;
      row[k] = at.order[j];
    }
  };
  auto finish_run = [&](bool goes_on) __attribute__((always_inline)) {
    if ((unsigned)now >= (unsigned)p.classes) return;
    if (from_before || goes_on) store8(at.parts + (from_before ? 0 : part_width(p.width)), 8, sum);
    else store_row<T>(p, at, now, sum);
  };
  places(at.first);
  for (int i = at.first; i < at.end; i += U) {
    // no token comes last: nothing of its row is read
    if ((unsigned)token[0] >= (unsigned)p.classes) break;
    Raw8<T> v[U];
    int of[U];
#pragma unroll
    for (int k = 0; k < U; ++k) {
      of[k] = token[k];
      raw_load(v[k], dy + row[k] * p.y_row, n, narrow_row<T>(p.width));
    }
    places(i + U);
#pragma unroll
    for (int k = 0; k < U; ++k) {
      if ((unsigned)of[k] < (unsigned)p.classes) {
        raw_place(v[k], n);
        if (of[k] != now) {
          finish_run(false);
          now = of[k];
          from_before = i + k == at.first && before == now;
#pragma unroll
          for (int e = 0; e < 8; ++e) sum[e] = 0.0f;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[e] += raw_at(v[k], e);
      }
    }
  }
  finish_run(behind == now);
}

// A run that passes ends of chunks: the parts that it left, by the lanes of the chunk that it begins in.
template <typename T> __global__ void __launch_bounds__(kThreads) join_chunks_kernel(EmbeddingArgs p, EmbeddingPlan plan, char* ws, int lanes_log2) {
  constexpr int U = 8;
  ChunkPlace at;
  if (!at.set(p, plan, ws, lanes_log2)) return;
  const int token = at.sorted[at.end - 1];
  if (at.end == p.rows || (unsigned)token >= (unsigned)p.classes || at.sorted[at.end] != token) return;
  if (at.first > 0 && at.sorted[at.first] == token && at.sorted[at.first - 1] == token) return;
  const int64_t apart = 2 * part_width(p.width);
  float sum[8];
  load8(at.parts + part_width(p.width), 8, sum);
  bool more = true;
  for (int q = at.chunk + 1; more; q += U) {
    float part[U][8];
    bool of_run[U];
#pragma unroll
    for (int k = 0; k < U; ++k) {
      const int chunk = min(q + k, plan.chunks - 1);
      of_run[k] = q + k < plan.chunks && at.sorted[chunk * plan.chunk] == token;
      load8(at.parts + (chunk - at.chunk) * apart, 8, part[k]);
    }
#pragma unroll
    for (int k = 0; k < U; ++k) {
      more = more && of_run[k];
#pragma unroll
      for (int e = 0; e < 8; ++e) sum[e] += more ? part[k][e] : 0.0f;
    }
  }
  store_row<T>(p, at, token, sum);
}

// Few rows a worker: a workgroup has a range of a table's rows to itself.  It writes zeros, sorts those of the tokens that lie in its range beside that, and sums
// their runs.  No other workgroup writes there, so that one launch is all: 2 x 65 tokens of 19 x 126 fp32 18.4 -> 9.5 us, 59 of 43011 x 265 bf16 18.6 -> 13.1 us, 64 x 100 of
// 1001 x 250 fp32 28 -> 23 us.
constexpr int kFewRows = kThreads, kPlaceBits = 8;
static_assert(1 << kPlaceBits == kFewRows, "place among a worker's rows");
static_assert((uint64_t)kMaxClasses << kPlaceBits < 0xFFFFFFFFull, "a token and its place fit 32 bits, with a value to spare");

// Sum of the threads' flags before this one, and of all: count is a wavefront's.
__device__ __forceinline__ int rank_of(bool flag, int (&count)[kThreads / kWave], int* all) {
  const uint64_t bits = __ballot(flag);
  const int wave = threadIdx.x / kWave;
  if (threadIdx.x % kWave == 0) count[wave] = __popcll(bits);
  __syncthreads();
  int before = __popcll(bits & ((1ull << (threadIdx.x % kWave)) - 1));
  *all = 0;
#pragma unroll
  for (int w = 0; w < kThreads / kWave; ++w) {
    before += w < wave ? count[w] : 0;
    *all += count[w];
  }
  __syncthreads();
  return before;
}

template <typename T> __global__ void __launch_bounds__(kThreads) few_rows_kernel(EmbeddingArgs p, int range, int lanes_log2) {
  constexpr int U = 8;
  __shared__ uint32_t key[kFewRows];
  __shared__ int start[kFewRows + 1], count[kThreads / kWave];
  const int t = threadIdx.x;
  const int64_t g = blockIdx.y;
  const int first = blockIdx.x * range, classes = min(range, p.classes - first);
  EmbeddingArgs part = p;                // of this workgroup's rows of the table
  part.dtable = reinterpret_cast<T*>(p.dtable) + (int64_t)first * p.dtable_row;
  part.classes = classes;
  clear_table<T>(part, g, 0, 1);
  const int token = t < p.rows ? p.tokens[g * p.rows + t] : -1;
  const bool mine = (unsigned)token < (unsigned)p.classes && (unsigned)token - (unsigned)first < (unsigned)classes;
  int n;
  const int at = rank_of(mine, count, &n);
  key[t] = kNoKey;
  __syncthreads();
  if (mine) key[at] = (uint32_t)token << kPlaceBits | (uint32_t)t;
  __syncthreads();
  int size = 2;
  while (size < n) size *= 2;
  bool across = false;
  for (int k = 2; k <= size; k <<= 1)
    for (int j = k >> 1; j > 0; j >>= 1) {
      if (across || j > 64) __syncthreads();
      else __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      across = j > 64;
      if (t < size / 2) {
        const int lo = ((t & ~(j - 1)) << 1) | (t & (j - 1)), hi = lo | j;
        const uint32_t a = key[lo], b = key[hi];
        if ((a > b) == ((lo & k) == 0)) {
          key[lo] = b;
          key[hi] = a;
        }
      }
    }
  __syncthreads();
  const bool begins = t < n && (t == 0 || key[t] >> kPlaceBits != key[t - 1] >> kPlaceBits);
  int runs;
  const int run = rank_of(begins, count, &runs);
  if (begins) start[run] = t;
  if (t == 0) start[runs] = n;
  __syncthreads();                       // and the zeros are written
  const int lanes = 1 << lanes_log2, groups = kThreads >> lanes_log2, slices = (p.width + 8 * lanes - 1) / (8 * lanes);
  for (int unit = t >> lanes_log2; unit < runs * slices; unit += groups) {
    const int r = unit / slices, c = (unit - r * slices) * 8 * lanes + (t & (lanes - 1)) * 8, width = p.width - c;
    if (width <= 0) continue;
    const int i0 = start[r], i1 = start[r + 1];
    const T* dy = reinterpret_cast<const T*>(p.y) + g * p.rows * p.y_row + c;
    float sum[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    for (int i = i0; i < i1; i += U) {
      Raw8<T> v[U];
#pragma unroll
      for (int k = 0; k < U; ++k) {
        const int64_t row = key[min(i + k, i1 - 1)] & (kFewRows - 1);
        raw_load(v[k], dy + row * p.y_row, width, narrow_row<T>(p.width));
      }
#pragma unroll
      for (int k = 0; k < U; ++k) {
        raw_place(v[k], width);
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[e] += i + k < i1 ? raw_at(v[k], e) : 0.0f;
      }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) sum[e] *= p.scale;
    store8(reinterpret_cast<T*>(p.dtable) + g * p.dtable_gs + (int64_t)(key[i0] >> kPlaceBits) * p.dtable_row + c, width, sum);
  }
}
template <typename T> hipError_t few_rows(const EmbeddingArgs& p, hipStream_t s) {
  // 32 KiB of a table a workgroup, and two workgroups a compute unit where it has the rows
  const int64_t bytes = (int64_t)p.classes * p.width * (int64_t)sizeof(T);
  const int64_t wanted = std::max<int64_t>((bytes + 32767) / 32768, (512 + p.workers - 1) / p.workers);
  const int range = (int)std::max<int64_t>((p.classes + wanted - 1) / wanted, 1);
  const int lanes_log2 = std::min(lanes_for_row(p.width), 6);
  hipLaunchKernelGGL(few_rows_kernel<T>, dim3((unsigned)((p.classes + range - 1) / range), (unsigned)p.workers), dim3(kThreads), 0, s, p, range, lanes_log2);
  return hipGetLastError();
}

template <typename T> hipError_t backward(const EmbeddingArgs& p, const EmbeddingPlan& plan, char* ws, hipStream_t s) {
  if (p.rows <= kFewRows) return few_rows<T>(p, s);
  int threads = kThreads;
  while (threads < kSortTile / 2 && 2 * threads < p.rows) threads *= 2;
  // 64 KiB of zeros a workgroup, 16384 in all at most
  const int64_t units = ((int64_t)p.classes * p.width * (int64_t)sizeof(T) + 65535) / 65536;
  const int clearers = (int)std::min<int64_t>(units, std::max<int64_t>(16384 / p.workers, 1));
  hipLaunchKernelGGL(sort_tiles_kernel<T>, dim3((unsigned)(plan.tiles + clearers), (unsigned)p.workers), dim3(threads), 0, s, p, plan, ws);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (plan.tiles > 1) {
    hipLaunchKernelGGL(place_tokens_kernel, dim3((unsigned)plan.tiles, (unsigned)p.workers), dim3(kSortTile / 2), 0, s, p, plan, ws);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  const int lanes_log2 = std::min(lanes_for_row(p.width), 6), slots = kThreads >> lanes_log2;
  const int64_t chunks = (int64_t)plan.chunks * p.workers * ((p.width + kSlice - 1) / kSlice);
  const dim3 grid = grid_of((chunks + slots - 1) / slots);
  hipLaunchKernelGGL(chunk_sums_kernel<T>, grid, dim3(kThreads), 0, s, p, plan, ws, lanes_log2);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  hipLaunchKernelGGL(join_chunks_kernel<T>, grid, dim3(kThreads), 0, s, p, plan, ws, lanes_log2);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_embedding(const EmbeddingArgs& p, bool bf16, hipStream_t s) {
  const int lanes_log2 = lanes_for_row(p.width), slots = kThreads >> lanes_log2;
  const dim3 grid((unsigned)std::min<int64_t>((p.rows * p.workers + slots - 1) / slots, 256 * 64));
  if (bf16) hipLaunchKernelGGL(embedding_kernel<uint16_t>, grid, dim3(kThreads), 0, s, p, lanes_log2);
  else hipLaunchKernelGGL(embedding_kernel<float>, grid, dim3(kThreads), 0, s, p, lanes_log2);
  return hipGetLastError();
}

EmbeddingPlan embedding_plan(int workers, int64_t rows, int width) {
  EmbeddingPlan e{};
  e.total = 256;
  if (rows <= kFewRows) return e;        // no rows, or few: nothing of the workspace is used
  e.tiles = (int)((rows + kSortTile - 1) / kSortTile);
  // Few rows a chunk, so that many lanes work on them; chunks grow with the rows, so that the commonest token's row has at most 256 parts to add: chunks of 8, 16,
  // 32 and 64 of 8 x 8192 tokens, 1024 wide, take 107, 89, 81 and 75 us for sums and parts, of 16 x 2013, 21 wide, 19, 21, 29 and 48 us.
  e.chunk = (int)std::max<int64_t>(kLeastChunk, ((rows + 255) / 256 + kLeastChunk - 1) / kLeastChunk * kLeastChunk);
  e.chunks = (int)((rows + e.chunk - 1) / e.chunk);
  size_t at = 0;
  auto take = [&](size_t bytes) { const size_t v = at; at += (bytes + 255) / 256 * 256; return v; };
  const size_t n = (size_t)workers, r = (size_t)rows;
  e.keys = e.tiles > 1 ? take(n * e.tiles * kSortTile * sizeof(uint32_t)) : 0;
  e.order = take(n * r * sizeof(int));
  e.sorted = take(n * r * sizeof(int));
  e.parts = take(n * e.chunks * 2 * part_width(width) * sizeof(float));
  e.total = at;
  return e;
}

hipError_t launch_embedding_backward(const EmbeddingArgs& p, const EmbeddingPlan& plan, char* ws, bool bf16, hipStream_t s) {
  return bf16 ? backward<uint16_t>(p, plan, ws, s) : backward<float>(p, plan, ws, s);
}

}  // namespace prsgd
