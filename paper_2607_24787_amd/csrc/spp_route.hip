// Tokens to their experts and back: the pairs (token, expert) sorted by expert,
// the tokens' rows copied to their places, the experts' rows summed with the
// gates, and that sum's gradients.  The calls' contracts are in spp.h.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <type_traits>

#include "spp.h"
#include "spp_fp4.h"
#include "spp_internal.h"

namespace {

// ------------------------------------------------------------------------ sort

constexpr int kSortThreads = 1024;
constexpr int kSortWaves = kSortThreads / 64;
constexpr int kMaxParts = 64;         // workgroups of a sort
constexpr int kMinPart = 4096;        // pairs of one at least
constexpr int64_t kMaxPairs = int64_t{1} << 24;

struct SortArgs {
  const int32_t* topk;
  int32_t *start, *pair, *place;
  int32_t* total;  // [parts][n] pairs of each expert in each part (parts > 1)
  int P, n, bits;  // bits of the largest id
  int parts, each;  // pairs of a part: a multiple of kSortThreads
};

// The lanes of this wave that hold the same id, as a mask; 0 for id < 0
__device__ __forceinline__ uint64_t alike(int id, int bits) {
  uint64_t m = __ballot(id >= 0);
  for (int b = 0; b < bits; ++b) {
    const uint64_t one = __ballot((id >> b) & 1);
    m &= (id >> b) & 1 ? one : ~one;
  }
  return id >= 0 ? m : 0;
}

__device__ __forceinline__ int id_at(const SortArgs& a, int p, int end) {
  const int id = p < end ? a.topk[p] : -1;
  return static_cast<unsigned>(id) < static_cast<unsigned>(a.n) ? id : -1;
}

// Counts of a wave's run of pairs [from, to) into its row of LDS, or with
// `each`(pair, id, pairs of that id before it in the row) called for every pair.
// A wave takes its pairs in order, 64 at a time, and only it writes its row: the
// places do not depend on which lane comes first.
template <typename Each>
__device__ __forceinline__ void take_run(const SortArgs& a, int* row, int from, int to, Each each) {
  const int lane = threadIdx.x & 63;
  for (int p0 = from; p0 < to; p0 += 64) {
    const int id = id_at(a, p0 + lane, to);
    const uint64_t same = alike(id, a.bits);
    const int before = __popcll(same & ((uint64_t{1} << lane) - 1));
    const int base = id >= 0 ? row[id] : 0;
    if (p0 + lane < to) each(p0 + lane, id, base + before);
    __builtin_amdgcn_wave_barrier();
    if (id >= 0 && before == 0) row[id] = base + __popcll(same);
    __builtin_amdgcn_wave_barrier();
  }
}

// Starts of the experts from their pairs (thread e: expert e; n is at most the
// threads), and all pairs
__device__ __forceinline__ int starts_of(int all, int* s_sum, int* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int incl = all;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int o = __shfl_up(incl, d);
    if (lane >= d) incl += o;
  }
  if (lane == 63) s_sum[wave] = incl;
  __syncthreads();
  int base = incl - all;
  *total = 0;
  for (int w = 0; w < kSortWaves; ++w) {
    base += w < wave ? s_sum[w] : 0;
    *total += s_sum[w];
  }
  return base;
}

constexpr int kCountedPairs = 1 << 14;  // sorts that count all pairs in every part
constexpr int kHeldPairs = 1 << 18;     // sorts whose parts are held in registers
constexpr int kHeld = 4;                // pairs of a thread

// A stable counting sort: a workgroup places kEach * 1024 pairs, which it holds
// in registers.  The others it counts by itself (at most 2^14: a launch that
// would count them costs more than the reads), or finds counted (kCounted).  A
// wave takes its run of pairs in order and only it writes its row of counts, so
// a pair's rank does not depend on which lane comes first.  Latency: 512 pairs of
// 128 experts take 4 us, 6,144 of 64 take 8.4 (two parts), 65,536 of 128 take 4.7 +
// 7.9; with the pairs read twice, in a loop, 12, and 5.9 + 13.
template <int kEach, bool kCounted>
__global__ __launch_bounds__(kSortThreads) void expert_sort_once_kernel(SortArgs a) {
  extern __shared__ int s_row[];  // [kSortWaves][n], then pairs before this part and behind it [2][n]
  __shared__ int s_sum[kSortWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int part = static_cast<int>(blockIdx.x) * kEach * kSortThreads, from = part + wave * 64 * kEach;
  int id[kEach], rank[kEach];
#pragma unroll
  for (int j = 0; j < kEach; ++j) id[j] = id_at(a, from + 64 * j + lane, a.P);
  constexpr int kMost = kCounted ? 1 : kCountedPairs / kSortThreads;
  int e[kMost];  // pairs of other parts
  if constexpr (!kCounted) {
#pragma unroll
    for (int j = 0; j < kMost; ++j) {
      const int p = j * kSortThreads + tid;
      e[j] = gridDim.x == 1 || (p >= part && p < part + kEach * kSortThreads) ? -1 : id_at(a, p, a.P);
    }
  }
  for (int i = tid; i < (kSortWaves + 2) * a.n; i += kSortThreads) s_row[i] = 0;
  __syncthreads();
  int* row = s_row + wave * a.n;
  int* other = s_row + kSortWaves * a.n;
#pragma unroll
  for (int j = 0; j < kEach; ++j) {
    const uint64_t same = alike(id[j], a.bits);
    const int before = __popcll(same & ((uint64_t{1} << lane) - 1));
    const int base = id[j] >= 0 ? row[id[j]] : 0;
    rank[j] = base + before;
    __builtin_amdgcn_wave_barrier();
    if (id[j] >= 0 && before == 0) row[id[j]] = base + __popcll(same);
    __builtin_amdgcn_wave_barrier();
  }
  // counts alone: their order does not matter
  if constexpr (!kCounted) {
#pragma unroll
    for (int j = 0; j < kMost; ++j)
      if (e[j] >= 0) atomicAdd(other + (j * kSortThreads + tid < part ? 0 : a.n) + e[j], 1);
  }
  __syncthreads();
  int all = 0, mine = 0, of_wave[kSortWaves];
  if (tid < a.n) {
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) of_wave[w] = s_row[w * a.n + tid];
    if constexpr (kCounted) {
      constexpr int kBatch = 8;
      for (int k0 = 0; k0 < a.parts; k0 += kBatch) {
        int c[kBatch];
#pragma unroll
        for (int k = 0; k < kBatch; ++k) c[k] = k0 + k < a.parts ? a.total[(k0 + k) * a.n + tid] : 0;
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
          all += c[k];
          mine += k0 + k < static_cast<int>(blockIdx.x) ? c[k] : 0;
        }
      }
    } else {
      mine = other[tid];
      all = mine + other[a.n + tid];
#pragma unroll
      for (int w = 0; w < kSortWaves; ++w) all += of_wave[w];
    }
  }
  int total;
  const int base = starts_of(all, s_sum, &total);
  if (tid < a.n) {
    if (blockIdx.x == 0) {
      a.start[tid] = base;
      if (tid == a.n - 1) a.start[a.n] = total;
    }
    int at = base + mine;
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) {
      s_row[w * a.n + tid] = at;
      at += of_wave[w];
    }
  }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < kEach; ++j) {
    const int p = from + 64 * j + lane;
    const int at = id[j] >= 0 ? row[id[j]] + rank[j] : -1;
    if (p < a.P) a.place[p] = at;
    if (id[j] >= 0) a.pair[at] = p;
  }
  // the places of pairs without an expert name no pair
  for (int i = total + static_cast<int>(blockIdx.x) * kSortThreads + tid; i < a.P;
       i += static_cast<int>(gridDim.x) * kSortThreads)
    a.pair[i] = -1;
}

// Pairs of each expert in each part of kHeld * 1024 pairs; counts alone
__global__ __launch_bounds__(kSortThreads) void expert_count_held_kernel(SortArgs a) {
  extern __shared__ int s_row[];  // [n]
  const int tid = threadIdx.x, part = static_cast<int>(blockIdx.x) * kHeld * kSortThreads;
  int id[kHeld];
#pragma unroll
  for (int j = 0; j < kHeld; ++j) id[j] = id_at(a, part + j * kSortThreads + tid, a.P);
  for (int i = tid; i < a.n; i += kSortThreads) s_row[i] = 0;
  __syncthreads();
#pragma unroll
  for (int j = 0; j < kHeld; ++j)
    if (id[j] >= 0) atomicAdd(s_row + id[j], 1);
  __syncthreads();
  if (tid < a.n) a.total[blockIdx.x * a.n + tid] = s_row[tid];
}

// Pairs of each expert in each part, for larger sorts
__global__ __launch_bounds__(kSortThreads) void expert_count_kernel(SortArgs a) {
  extern __shared__ int s_row[];  // [kSortWaves][n]
  const int wave = threadIdx.x >> 6, run = a.each / kSortWaves;
  for (int i = threadIdx.x; i < kSortWaves * a.n; i += kSortThreads) s_row[i] = 0;
  __syncthreads();
  const int64_t from = static_cast<int64_t>(blockIdx.x) * a.each + wave * run;
  const int to = static_cast<int>(min<int64_t>(from + run, a.P));
  if (from < to) take_run(a, s_row + wave * a.n, static_cast<int>(from), to, [](int, int, int) {});
  __syncthreads();
  for (int e = threadIdx.x; e < a.n; e += kSortThreads) {
    int sum = 0;
    for (int w = 0; w < kSortWaves; ++w) sum += s_row[w * a.n + e];
    a.total[static_cast<size_t>(blockIdx.x) * a.n + e] = sum;
  }
}

// A stable counting sort of more pairs.  A wave counts its run of pairs by expert; the counts
// become starts (experts before, parts before, waves before); the wave goes
// through its run again and gives every pair its place.
__global__ __launch_bounds__(kSortThreads) void expert_sort_kernel(SortArgs a) {
  extern __shared__ int s_row[];  // [kSortWaves][n]
  __shared__ int s_sum[kSortWaves];
  const int tid = threadIdx.x, wave = tid >> 6, run = a.each / kSortWaves;
  for (int i = tid; i < kSortWaves * a.n; i += kSortThreads) s_row[i] = 0;
  __syncthreads();
  const int64_t from64 = static_cast<int64_t>(blockIdx.x) * a.each + wave * run;
  const int to = static_cast<int>(min<int64_t>(from64 + run, a.P));
  const int from = static_cast<int>(min<int64_t>(from64, a.P));
  int* row = s_row + wave * a.n;
  take_run(a, row, from, to, [](int, int, int) {});
  __syncthreads();
  // thread e: expert e (n is at most the threads)
  int all = 0, mine = 0;  // pairs of the expert: in all parts, and in the parts before this one
  if (tid < a.n) {
    for (int k = 0; k < a.parts; ++k) {
      const int c = a.total[static_cast<size_t>(k) * a.n + tid];
      all += c;
      mine += k < static_cast<int>(blockIdx.x) ? c : 0;
    }
  }
  int total;
  const int base = starts_of(all, s_sum, &total);
  if (tid < a.n) {
    if (blockIdx.x == 0) {
      a.start[tid] = base;
      if (tid == a.n - 1) a.start[a.n] = total;
    }
    int at = base + mine;
    for (int w = 0; w < kSortWaves; ++w) {
      const int c = s_row[w * a.n + tid];
      s_row[w * a.n + tid] = at;
      at += c;
    }
  }
  __syncthreads();
  take_run(a, row, from, to, [&](int p, int id, int at) {
    a.place[p] = id >= 0 ? at : -1;
    if (id >= 0) a.pair[at] = p;
  });
  // the places of pairs without an expert name no pair
  for (int64_t i = static_cast<int64_t>(total) + blockIdx.x * kSortThreads + tid; i < a.P;
       i += static_cast<int64_t>(a.parts) * kSortThreads)
    a.pair[i] = -1;
}

// ------------------------------------------------- rows there, back, gradients

struct RowArgs {
  const void* x;       // gather: tokens' rows; combine and its gradient: pairs' rows
  int64_t x_stride;    // bytes, as every stride here
  const void* res;     // combine: added rows, or NULL; gradient: the outputs' gradient
  int64_t res_stride;
  void* out;
  int64_t out_stride;
  const int32_t* place;  // or NULL: pair p's row is row p, where its id is an expert
  const int32_t* ids;
  const float* weight;  // or NULL: 1
  float* d_weight;
  int T, K, n, pieces;  // pieces: of 16 bytes, of an output row
  int shift;         // threads of a row: 1 << shift
};

constexpr int kRowThreads = 256;

// 16 bytes to fp32 values and back
template <typename T>
__device__ __forceinline__ void widen(u32x4 v, float* f) {
  if constexpr (std::is_same<T, float>::value) {
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(v[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) f[2 * i] = bf16_lo(v[i]), f[2 * i + 1] = bf16_hi(v[i]);
  }
}

template <typename T>
__device__ __forceinline__ u32x4 narrow(const float* f) {
  u32x4 v;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (std::is_same<T, float>::value)
      v[i] = __float_as_uint(f[i]);
    else
      v[i] = pack_bf16(f[2 * i], f[2 * i + 1]);
  }
  return v;
}

__device__ __forceinline__ const u32x4* row_at(const void* base, int64_t stride, int64_t row) {
  return reinterpret_cast<const u32x4*>(static_cast<const uint8_t*>(base) + row * stride);
}
__device__ __forceinline__ u32x4* row_at(void* base, int64_t stride, int64_t row) {
  return reinterpret_cast<u32x4*>(static_cast<uint8_t*>(base) + row * stride);
}

// This thread's token and first piece; its row's next piece is `step` further
struct RowOf {
  int t, first, step;
  __device__ __forceinline__ explicit RowOf(const RowArgs& a) {
    const int per = kRowThreads >> a.shift;
    t = static_cast<int>(blockIdx.x) * per + (static_cast<int>(threadIdx.x) >> a.shift);
    step = 1 << a.shift;
    first = static_cast<int>(threadIdx.x) & (step - 1);
  }
};

constexpr int kRowBatch = 8;  // rows whose loads are in flight together

// A token's row is read once and written to its pairs' places.  Bound by the
// writes: 8,192 bf16 rows of 2,048 to 8 places each take 47 to 58 us (302 MB, 5.2 to
// 6.4 TB/s).
__global__ __launch_bounds__(kRowThreads) void expert_gather_kernel(RowArgs a) {
  const RowOf r(a);
  if (r.t >= a.T) return;
  const int P = a.T * a.K;
  const int32_t* place = a.place + static_cast<int64_t>(r.t) * a.K;
  const u32x4* from = row_at(a.x, a.x_stride, r.t);
  for (int i = r.first; i < a.pieces; i += r.step) {
    const u32x4 v = from[i];
    for (int k0 = 0; k0 < a.K; k0 += kRowBatch) {
      int at[kRowBatch];
#pragma unroll
      for (int k = 0; k < kRowBatch; ++k) at[k] = k0 + k < a.K ? place[k0 + k] : -1;
#pragma unroll
      for (int k = 0; k < kRowBatch; ++k)
        if (static_cast<unsigned>(at[k]) < static_cast<unsigned>(P)) row_at(a.out, a.out_stride, at[k])[i] = v;
    }
  }
}

// Where pair p's row is; negative or too large: nowhere
__device__ __forceinline__ int place_of(const RowArgs& a, int64_t p) {
  if (a.place) return a.place[p];
  return static_cast<unsigned>(a.ids[p]) < static_cast<unsigned>(a.n) ? static_cast<int>(p) : -1;
}

// Sums in fp32, in the order of a token's experts.  Rows in T, or fp32 rows of
// bf16 outputs.  Bound by the rows' reads, which go past the caches: 65,536 bf16
// rows of 2,048 take 64 us with weights and a residual (335 MB, 5.2 TB/s), 98
// through the caches.
template <typename T, typename Rows, bool kWeights>
__global__ __launch_bounds__(kRowThreads) void expert_combine_kernel(RowArgs a) {
  constexpr int E = 16 / static_cast<int>(sizeof(T));
  constexpr int Q = static_cast<int>(sizeof(Rows) / sizeof(T));  // pieces of a row for one of the output
  const RowOf r(a);
  if (r.t >= a.T) return;
  const int P = a.T * a.K;
  const int64_t p0 = static_cast<int64_t>(r.t) * a.K;
  for (int i = r.first; i < a.pieces; i += r.step) {
    float sum[E];
#pragma unroll
    for (int j = 0; j < E; ++j) sum[j] = 0.f;
    for (int k0 = 0; k0 < a.K; k0 += kRowBatch) {
      u32x4 v[kRowBatch][Q];
      float w[kRowBatch];
      bool have[kRowBatch];
#pragma unroll
      for (int k = 0; k < kRowBatch; ++k) {
        const int at = k0 + k < a.K ? place_of(a, p0 + k0 + k) : -1;
        have[k] = static_cast<unsigned>(at) < static_cast<unsigned>(P);
#pragma unroll
        for (int q = 0; q < Q; ++q)
          if (have[k]) v[k][q] = __builtin_nontemporal_load(row_at(a.x, a.x_stride, at) + i * Q + q);
        if constexpr (kWeights) w[k] = have[k] ? a.weight[p0 + k0 + k] : 0.f;
      }
#pragma unroll
      for (int k = 0; k < kRowBatch; ++k) {
        if (!have[k]) continue;
        float f[E];
#pragma unroll
        for (int q = 0; q < Q; ++q) widen<Rows>(v[k][q], f + q * (E / Q));
#pragma unroll
        for (int j = 0; j < E; ++j) {
          if constexpr (kWeights)
            sum[j] = fmaf(w[k], f[j], sum[j]);
          else
            sum[j] += f[j];
        }
      }
    }
    if (a.res) {
      float f[E];
      widen<T>(row_at(a.res, a.res_stride, r.t)[i], f);
#pragma unroll
      for (int j = 0; j < E; ++j) sum[j] += f[j];
    }
    row_at(a.out, a.out_stride, r.t)[i] = narrow<T>(sum);
  }
}

// One wave per pair: d_row = w * d_out, d_w = <d_out, row>.  The waves of a
// token are neighbours and find its d_out in the caches.  Bound by memory: 65,536
// bf16 rows of 2,048 read and written take 126 us (570 MB, 4.5 TB/s; a copy reaches
// 5.2).
template <typename T>
__global__ __launch_bounds__(kRowThreads) void expert_combine_grad_kernel(RowArgs a) {
  constexpr int E = 16 / static_cast<int>(sizeof(T));
  const int lane = static_cast<int>(threadIdx.x) & 63;
  const int P = a.T * a.K;
  const int64_t p = static_cast<int64_t>(blockIdx.x) * (kRowThreads / 64) + (threadIdx.x >> 6);
  if (p >= P) return;
  const int at = a.place[p];
  float dot = 0.f;
  if (static_cast<unsigned>(at) < static_cast<unsigned>(P)) {
    const float w = a.weight ? a.weight[p] : 1.f;
    const u32x4* d = row_at(a.res, a.res_stride, p / a.K);
    const u32x4* y = row_at(a.x, a.x_stride, at);
    u32x4* o = a.out ? row_at(a.out, a.out_stride, at) : nullptr;
    for (int i = lane; i < a.pieces; i += 64) {
      float f[E], g[E];
      widen<T>(d[i], f);
      if (a.d_weight) {
        widen<T>(__builtin_nontemporal_load(y + i), g);
#pragma unroll
        for (int j = 0; j < E; ++j) dot = fmaf(f[j], g[j], dot);
      }
      if (o) {
#pragma unroll
        for (int j = 0; j < E; ++j) f[j] *= w;
        o[i] = narrow<T>(f);
      }
    }
  }
  if (!a.d_weight) return;
#pragma unroll
  for (int m = 32; m > 0; m >>= 1) dot += __shfl_xor(dot, m);
  if (lane == 0) a.d_weight[p] = dot;
}

// ------------------------------------------------------------------ host side

const char* pairs_why(int32_t T, int32_t K) {
  if (T < 0 || K < 1) return "T must be >= 0 and K >= 1";
  if (static_cast<int64_t>(T) * K > kMaxPairs) return "T * K must be at most 2^24";
  return nullptr;
}

// Parts of a sort at most
int64_t most_parts(int64_t P) { return std::min<int64_t>(kMaxParts, std::max<int64_t>(1, (P + kMinPart - 1) / kMinPart)); }

// Parts of a sort whose parts are not held, and pairs of one
void parts_of(int64_t P, int* parts, int* each) {
  const int64_t e = ((P + kMaxParts - 1) / kMaxParts + kSortThreads - 1) / kSortThreads * kSortThreads;
  *each = static_cast<int>(e);
  *parts = static_cast<int>((P + e - 1) / e);
}

const char* width_why(int32_t D, int elem) {
  return D < 1 || D > 1 << 20 || static_cast<int64_t>(D) * elem % 16 != 0
             ? "D must be positive, at most 2^20, and a row a multiple of 16 bytes"
             : nullptr;
}

RowArgs rows_of(int32_t T, int32_t K, int32_t D, int elem) {
  RowArgs a{};
  a.T = T;
  a.K = K;
  a.pieces = D * elem / 16;
  // a launch has fewer than 2^32 threads: of 2^24 tokens none gets a whole workgroup
  const int most = T < kMaxPairs ? 8 : 7;
  while (a.shift < most && 1 << a.shift < a.pieces) ++a.shift;
  return a;
}

unsigned row_grid(const RowArgs& a) {
  const int per = kRowThreads >> a.shift;
  return static_cast<unsigned>((a.T + per - 1) / per);
}

}  // namespace

namespace spp {

size_t expert_sort_bytes(int64_t P, int32_t n) {
  const int64_t parts = most_parts(P);
  return parts > 1 ? static_cast<size_t>(parts) * n * sizeof(int32_t) : 0;
}

hipError_t launch_expert_sort(const int32_t* topk, int64_t P, int32_t n, int32_t* start, int32_t* pair, int32_t* place,
                              void* workspace, hipStream_t st) {
  SortArgs a{};
  a.topk = topk;
  a.start = start;
  a.pair = pair;
  a.place = place;
  a.total = static_cast<int32_t*>(workspace);
  a.P = static_cast<int>(P);
  a.n = n;
  while (1 << a.bits < n) ++a.bits;
  void* params[] = {&a};
  if (P <= kHeldPairs) {
    const int each = (P <= kSortThreads ? 1 : kHeld) * kSortThreads;
    a.parts = static_cast<int>(std::max<int64_t>(1, (P + each - 1) / each));
    const bool counted = P > kCountedPairs;
    if (counted) {
      const hipError_t e = hipLaunchKernel(reinterpret_cast<const void*>(expert_count_held_kernel), dim3(a.parts),
                                           dim3(kSortThreads), params, static_cast<unsigned>(n * sizeof(int)), st);
      if (e != hipSuccess) return e;
    }
    const auto kernel = counted               ? expert_sort_once_kernel<kHeld, true>
                        : P <= kSortThreads ? expert_sort_once_kernel<1, false>
                                            : expert_sort_once_kernel<kHeld, false>;
    return hipLaunchKernel(reinterpret_cast<const void*>(kernel), dim3(a.parts), dim3(kSortThreads), params,
                           static_cast<unsigned>((kSortWaves + 2) * n * sizeof(int)), st);
  }
  parts_of(P, &a.parts, &a.each);
  const unsigned lds = static_cast<unsigned>(kSortWaves * n * sizeof(int));
  const hipError_t e = hipLaunchKernel(reinterpret_cast<const void*>(expert_count_kernel), dim3(a.parts),
                                       dim3(kSortThreads), params, lds, st);
  if (e != hipSuccess) return e;
  return hipLaunchKernel(reinterpret_cast<const void*>(expert_sort_kernel), dim3(a.parts), dim3(kSortThreads), params,
                         lds, st);
}

hipError_t launch_expert_combine(const ExpertSum& c, hipStream_t st) {
  const int elem = c.dtype == SPP_DTYPE_BF16 ? 2 : 4, rows_elem = c.fp32_rows ? 4 : elem;
  RowArgs a = rows_of(c.T, c.K, c.D, elem);
  a.x = c.rows;
  a.x_stride = c.rows_stride * rows_elem;
  a.res = c.residual;
  a.res_stride = c.residual_stride * elem;
  a.out = c.out;
  a.out_stride = c.out_stride * elem;
  a.place = c.place;
  a.ids = c.ids;
  a.n = c.n;
  a.weight = c.weights;
  const auto kernel =
      c.dtype == SPP_DTYPE_BF16
          ? (c.fp32_rows ? expert_combine_kernel<__bf16, float, true>
                         : c.weights ? expert_combine_kernel<__bf16, __bf16, true>
                                     : expert_combine_kernel<__bf16, __bf16, false>)
          : (c.weights ? expert_combine_kernel<float, float, true> : expert_combine_kernel<float, float, false>);
  return launch(kernel, row_grid(a), kRowThreads, a, st);
}

}  // namespace spp

extern "C" size_t spp_expert_sort_workspace(int32_t T, int32_t K, int32_t n) {
  if (const char* w = pairs_why(T, K)) return bad(w), 0;
  if (n < 1 || n > spp::kMaxExpertsTopK) return bad("n must be in [1, 1024]"), 0;
  return std::max<size_t>(16, spp::expert_sort_bytes(static_cast<int64_t>(T) * K, n));
}

extern "C" spp_status spp_expert_sort(const int32_t* topk, int32_t T, int32_t K, int32_t n, int32_t* start,
                                      int32_t* pair, int32_t* place, void* workspace, size_t workspace_bytes,
                                      void* hip_stream) {
  SPP_BAD(pairs_why(T, K));
  if (n < 1 || n > spp::kMaxExpertsTopK) return bad("n must be in [1, 1024]");
  if (!start || (T > 0 && (!topk || !pair || !place))) return bad("topk, start, pair and place must not be NULL");
  if (!aligned(topk, 4) || !aligned(start, 4) || !aligned(pair, 4) || !aligned(place, 4))
    return bad("topk, start, pair and place must be aligned to their elements");
  const int64_t P = static_cast<int64_t>(T) * K;
  const size_t need = spp::expert_sort_bytes(P, n);
  if (need > 0) {
    if (!workspace || !aligned16(workspace)) return bad("workspace must not be NULL, and 16-byte aligned");
    if (workspace_bytes < need) return bad("the workspace is too small");
  }
  const Rows all[] = {array(topk, P * 4), array(pair, P * 4), array(place, P * 4), array(start, (n + 1) * 4),
                      array(need > 0 ? workspace : nullptr, static_cast<int64_t>(need))};
  for (const Rows& one : all)
    for (const Rows* other = all; other < &one; ++other)
      if (meet(one, *other)) return bad("topk, start, pair, place and workspace must not overlap");
  return launched(spp::launch_expert_sort(topk, P, n, start, pair, place, workspace, static_cast<hipStream_t>(hip_stream)));
}

extern "C" spp_status spp_expert_gather(int32_t dtype, const void* x, int64_t x_stride, const int32_t* place, int32_t T,
                                        int32_t K, int32_t D, void* rows, int64_t rows_stride, void* hip_stream) {
  SPP_BAD(dtype_why(dtype));
  SPP_BAD(pairs_why(T, K));
  const int elem = dtype == SPP_DTYPE_BF16 ? 2 : 4;
  SPP_BAD(width_why(D, elem));
  if (T == 0) return SPP_OK;
  SPP_BAD(rows_why(x, x_stride, D, elem));
  SPP_BAD(rows_why(rows, rows_stride, D, elem));
  if (!place || !aligned(place, 4)) return bad("place must not be NULL, and aligned to its elements");
  const Rows to = rows_from(rows, rows_stride, D, static_cast<int64_t>(T) * K, elem);
  if (meet(to, rows_from(x, x_stride, D, T, elem))) return bad("rows must not overlap x");
  if (meet(to, array(place, static_cast<int64_t>(T) * K * 4))) return bad("rows must not overlap place");
  RowArgs a = rows_of(T, K, D, elem);
  a.x = x;
  a.x_stride = x_stride * elem;
  a.out = rows;
  a.out_stride = rows_stride * elem;
  a.place = place;
  return launched(launch(expert_gather_kernel, row_grid(a), kRowThreads, a, static_cast<hipStream_t>(hip_stream)));
}

extern "C" spp_status spp_expert_combine(int32_t dtype, const void* rows, int64_t rows_stride, const int32_t* place,
                                         const float* weights, int32_t T, int32_t K, int32_t D, const void* residual,
                                         int64_t residual_stride, void* out, int64_t out_stride, void* hip_stream) {
  SPP_BAD(dtype_why(dtype));
  SPP_BAD(pairs_why(T, K));
  const int elem = dtype == SPP_DTYPE_BF16 ? 2 : 4;
  SPP_BAD(width_why(D, elem));
  if (T == 0) return SPP_OK;
  SPP_BAD(rows_why(rows, rows_stride, D, elem));
  SPP_BAD(rows_why(out, out_stride, D, elem));
  if (!place || !aligned(place, 4) || !aligned(weights, 4))
    return bad("place must not be NULL, place and weights aligned to their elements");
  const Rows to = rows_from(out, out_stride, D, T, elem);
  if (meet(to, rows_from(rows, rows_stride, D, static_cast<int64_t>(T) * K, elem))) return bad("out must not overlap rows");
  const int64_t each = static_cast<int64_t>(T) * K * 4;
  if (meet(to, array(place, each)) || meet(to, array(weights, each))) return bad("out must not overlap place or weights");
  if (residual) {
    SPP_BAD(rows_why(residual, residual_stride, D, elem));
    if (!(residual == out && residual_stride == out_stride) && meet(to, rows_from(residual, residual_stride, D, T, elem)))
      return bad("out must be residual with the same stride, or not overlap it");
  }
  const spp::ExpertSum sum{rows, rows_stride, place,    nullptr,         weights, 0,          dtype,
                           0,    T,           K,        D,               residual, residual_stride, out, out_stride};
  return launched(spp::launch_expert_combine(sum, static_cast<hipStream_t>(hip_stream)));
}

extern "C" spp_status spp_expert_combine_grad(int32_t dtype, const void* d_out, int64_t d_out_stride, const void* rows,
                                              int64_t rows_stride, const int32_t* place, const float* weights, int32_t T,
                                              int32_t K, int32_t D, void* d_rows, int64_t d_rows_stride,
                                              float* d_weights, void* hip_stream) {
  SPP_BAD(dtype_why(dtype));
  SPP_BAD(pairs_why(T, K));
  const int elem = dtype == SPP_DTYPE_BF16 ? 2 : 4;
  SPP_BAD(width_why(D, elem));
  if (T == 0 || (!d_rows && !d_weights)) return SPP_OK;
  SPP_BAD(rows_why(d_out, d_out_stride, D, elem));
  if (!place || !aligned(place, 4) || !aligned(weights, 4) || !aligned(d_weights, 4))
    return bad("place must not be NULL, place, weights and d_weights aligned to their elements");
  const int64_t P = static_cast<int64_t>(T) * K;
  if (d_weights) SPP_BAD(rows_why(rows, rows_stride, D, elem));
  if (d_rows) {
    SPP_BAD(rows_why(d_rows, d_rows_stride, D, elem));
    const Rows to = rows_from(d_rows, d_rows_stride, D, P, elem);
    if (meet(to, rows_from(d_out, d_out_stride, D, T, elem))) return bad("d_rows must not overlap d_out");
    if (d_weights && !(rows == d_rows && rows_stride == d_rows_stride) && meet(to, rows_from(rows, rows_stride, D, P, elem)))
      return bad("d_rows must be rows with the same stride, or not overlap them");
    if (meet(to, array(place, P * 4)) || meet(to, array(weights, P * 4)))
      return bad("d_rows must not overlap place or weights");
    if (meet(to, array(d_weights, P * 4))) return bad("d_weights must not overlap d_rows");
  }
  const Rows dots = array(d_weights, P * 4);
  if (meet(dots, array(place, P * 4)) || meet(dots, array(weights, P * 4)) || meet(dots, rows_from(d_out, d_out_stride, D, T, elem)) ||
      meet(dots, rows_from(rows, rows_stride, D, P, elem)))
    return bad("d_weights must not overlap an input");
  RowArgs a = rows_of(T, K, D, elem);
  a.x = rows;
  a.x_stride = rows_stride * elem;
  a.res = d_out;
  a.res_stride = d_out_stride * elem;
  a.out = d_rows;
  a.out_stride = d_rows_stride * elem;
  a.place = place;
  a.weight = weights;
  a.d_weight = d_weights;
  const unsigned grid = static_cast<unsigned>((P + kRowThreads / 64 - 1) / (kRowThreads / 64));
  const auto kernel = dtype == SPP_DTYPE_BF16 ? expert_combine_grad_kernel<__bf16> : expert_combine_grad_kernel<float>;
  return launched(launch(kernel, grid, kRowThreads, a, static_cast<hipStream_t>(hip_stream)));
}
