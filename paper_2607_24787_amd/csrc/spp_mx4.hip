// Matrices in microscaled 4 bits: quantisation, products with them, and an MoE
// layer's routed experts on them.  The calls' contracts and the format are in
// spp.h.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <cstring>
#include <type_traits>
#include <utility>

#include "spp.h"
#include "spp_fp4.h"
#include "spp_internal.h"

namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));

constexpr int kOne = 127;  // the scale byte of 1

// ------------------------------------------------------- quantisation and back

struct RowsQ {
  const void* x;
  void* out;
  int64_t x_stride, out_stride;  // elements
  uint8_t *codes, *scales;
  int64_t words;  // of codes: 8 elements each
  int per_row;    // words of a row
};

constexpr int kQuantThreads = 256;

// A lane takes 8 elements, four lanes a block: a row's reads and writes are whole
// cache lines.  Bound by memory: 98,304 bf16 rows of 2,048 take 113 us (510 MB, 4.5
// TB/s) here, and 97 us (5.3 TB/s) to be read back by mx4_load_kernel.
template <typename T>
__global__ __launch_bounds__(kQuantThreads) void mx4_quantize_kernel(RowsQ a) {
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * kQuantThreads + threadIdx.x; i < a.words;
       i += static_cast<int64_t>(gridDim.x) * kQuantThreads) {
    const int64_t row = i / a.per_row;
    float y[8];
    load8(static_cast<const T*>(a.x) + row * a.x_stride + (i - row * a.per_row) * 8, y);
    uint32_t byte;
    reinterpret_cast<uint32_t*>(a.codes)[i] = quantise8(y, &byte);
    if (i % 4 == 0) a.scales[i / 4] = static_cast<uint8_t>(byte);
  }
}

template <typename T>
__global__ __launch_bounds__(kQuantThreads) void mx4_load_kernel(RowsQ a) {
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * kQuantThreads + threadIdx.x; i < a.words;
       i += static_cast<int64_t>(gridDim.x) * kQuantThreads) {
    const int64_t row = i / a.per_row;
    const uint32_t byte = a.scales[i / 4];
    const u32x4 v = cvt8(reinterpret_cast<const uint32_t*>(a.codes)[i], scale_of(byte));
    T* out = static_cast<T*>(a.out) + row * a.out_stride + (i - row * a.per_row) * 8;
    if constexpr (std::is_same<T, float>::value) {
      float f[8];
#pragma unroll
      for (int j = 0; j < 4; ++j) f[2 * j] = bf16_lo(v[j]), f[2 * j + 1] = bf16_hi(v[j]);
      store8(out, f);
    } else {
      *reinterpret_cast<u32x4*>(out) = v;
    }
  }
}

// --------------------------------------------------------- products of few rows

// What a product's rows of x are
// (rows of two bf16 terms, the second one half a stride behind: kXTerms multiplies
// one after the other, kXTermRows as neighbouring rows of x, of one row)
enum { kXBf16 = 0, kXCodes = 1, kXQuantBf16 = 2, kXQuantF32 = 3, kXTerms = 4, kXTermRows = 5 };
// A result as such terms, which keep 16 bits
struct Terms {};
// Which rows a group has: start[g] .. start[g+1] - 1 (or all), or the pairs
// with its id
enum { kRowsStart = 0, kRowsIds = 1 };

struct ProductArgs {
  const uint8_t *codes, *scales;  // the groups' weights
  int64_t blocks;                 // of all weights
  int N, nb;                      // outputs of a group; blocks of 32 of a row
  const void* x;
  int64_t x_stride;               // bytes
  const uint8_t* x_scales;        // kXCodes: [rows][nb]
  int64_t x_blocks;               // of all rows of x
  const int32_t* start;
  int M, groups;
  const int32_t* ids;             // kRowsIds: [M]
  const int32_t* pair;            // row i of a group is row pair[i] / xdiv of x (NULL: i / xdiv)
  int xdiv;
  int run;                        // few rows: tiles of a workgroup
  int by_pair;                    // kRowsIds: blockIdx.y is a pair, and the first with its id takes the group
  void* out;
  int64_t out_stride;             // elements
  uint8_t* out_scales;            // SwiGLU results in 4 bits
  int columns;                    // workgroups over a group's outputs
  int wide_out;                   // rows of out are 16-byte aligned
};

// A row's scale bytes, four blocks at a time, read whole and in bounds: near the
// end of all scales (at least four) the word starts earlier.
struct ScaleRow {
  const uint8_t* p;
  int last;  // the last block at which a word may start
  __device__ __forceinline__ ScaleRow(const uint8_t* scales, int64_t row, int nb, int64_t total) {
    p = scales + row * nb;
    last = static_cast<int>(min(total - 4 - row * nb, int64_t{1} << 20));
  }
  __device__ __forceinline__ uint32_t load(int b) const {
    uint32_t w;
    __builtin_memcpy(&w, p + min(b, last), 4);
    return w;
  }
};

__device__ __forceinline__ f32x4 mfma_bf16(u32x4 a, u32x4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// 32 values of a block, in fp32, to codes
__device__ __forceinline__ u32x4 quantise32(const float* y, uint32_t* byte) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 32; ++i) top = max(top, __float_as_uint(y[i]) & 0x7fffffffu);
  *byte = byte_of(top);
  if (*byte == kNanByte) return u32x4{0, 0, 0, 0};
  const float scale = scale_of(*byte);
  u32x4 c;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[8 * i], y[8 * i + 1], scale, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[8 * i + 2], y[8 * i + 3], scale, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[8 * i + 4], y[8 * i + 5], scale, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[8 * i + 6], y[8 * i + 7], scale, 3);
    c[i] = w;
  }
  return c;
}

__device__ __forceinline__ i32x8 wide(u32x4 c) {
  return i32x8{static_cast<int>(c[0]), static_cast<int>(c[1]), static_cast<int>(c[2]), static_cast<int>(c[3]), 0, 0, 0, 0};
}

// A barrier for LDS reads and writes that leaves loads into LDS on their way:
// __syncthreads() would wait for them.
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// kStep blocks of a row of x: bf16 rows as four operands of 8 elements each, split
// rows as four and four, rows in 4 bits as codes with their scale byte
template <int X, int kStep>
struct XBlocks {
  static constexpr int kParts = X == kXBf16 || X == kXTermRows ? 4 : X == kXTerms ? 8 : 1;
  u32x4 v[kStep][kParts];
  uint32_t byte[kStep];
  // blocks b .. b + kStep - 1, zeros outside [b0, b1) or for no row (`row` is one
  // that can be read all the same)
  __device__ __forceinline__ void load(const ProductArgs& a, int64_t row, bool have, int b, int b0, int b1) {
    const uint8_t* p = static_cast<const uint8_t*>(a.x) + row * a.x_stride;
    if constexpr (X == kXTermRows) p += threadIdx.x & 1 ? a.x_stride / 2 : 0;
    if constexpr (X != kXQuantBf16 && X != kXQuantF32) {
#pragma unroll
      for (int s = 0; s < kStep; ++s) {
        byte[s] = kOne;
#pragma unroll
        for (int q = 0; q < kParts; ++q) v[s][q] = u32x4{0, 0, 0, 0};
        if (!have || b + s < b0 || b + s >= b1) continue;
        if constexpr (X == kXCodes) {
          v[s][0] = reinterpret_cast<const u32x4*>(p)[b + s];
          byte[s] = a.x_scales[row * a.nb + b + s];
        } else {
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            v[s][q] = reinterpret_cast<const u32x4*>(p)[4 * (b + s) + q];
            if constexpr (X == kXTerms) v[s][4 + q] = reinterpret_cast<const u32x4*>(p + a.x_stride / 2)[4 * (b + s) + q];
          }
        }
      }
      return;
    }
    // converted: all lanes load, so that no load is waited for inside a branch
    using T = typename std::conditional<X == kXQuantBf16, __bf16, float>::type;
    float y[kStep][32];
#pragma unroll
    for (int s = 0; s < kStep; ++s)
#pragma unroll
      for (int q = 0; q < 4; ++q) load8(reinterpret_cast<const T*>(p) + 32 * min(b + s, a.nb - 1) + 8 * q, y[s] + 8 * q);
#pragma unroll
    for (int s = 0; s < kStep; ++s) {
      const bool ok = have && b + s >= b0 && b + s < b1;
      uint32_t scale;
      const u32x4 codes = quantise32(y[s], &scale);
      v[s][0] = ok ? codes : u32x4{0, 0, 0, 0};
      byte[s] = ok ? scale : kOne;
    }
  }
};

__device__ __forceinline__ f32x4 mfma_mx4(u32x4 w, uint32_t w_byte, u32x4 x, uint32_t x_byte, f32x4 c) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wide(w), wide(x), c, 4, 4, 0, static_cast<int>(w_byte), 0,
                                                          static_cast<int>(x_byte));
}

// Two results as bf16 terms of 16 bits together (the first ones; *low: the
// second): the first is cut off, not rounded, so that a finite result's is finite;
// the second holds what that leaves, nothing beside an infinity.
__device__ __forceinline__ uint32_t terms_of(float a, float b, uint32_t* low) {
  const uint32_t high = __float_as_uint(a) >> 16 | (__float_as_uint(b) & 0xffff0000u);
  *low = pack_bf16(a == bf16_lo(high) ? 0.f : a - bf16_lo(high), b == bf16_hi(high) ? 0.f : b - bf16_hi(high));
  return high;
}

__device__ __forceinline__ float swiglu(float g, float u) { return g / (1.f + expf(-g)) * u; }

constexpr int kFewThreads = 256;
constexpr int kFewWaves = kFewThreads / 64;
// Up to kStep blocks of a lane, of kTiles weight rows: codes and scale bytes.
// Lane l holds weight row and row of x l % 16.  Which blocks a lane takes is
// free as long as both operands agree: the matrix instruction's sum goes by lane
// and place, whatever the blocks' order in K.  Here a lane's blocks follow one
// another, so that its loads share cache lines and its scales a word.  kTiny:
// rows of fewer blocks, or fewer scales than a word's in all.
template <int kTiles, int kStep, bool kTiny>
struct WeightBlocks {
  u32x4 codes[kTiles][kStep];
  uint32_t scales[kTiles];
  int shift[kTiles];
  // The first of kStep blocks that are in the row, from block b on
  static __device__ __forceinline__ int window(const ProductArgs& a, int b) { return max(min(b, a.nb - kStep), 0); }
  // blocks b .. b + kStep - 1 of a window
  __device__ __forceinline__ void load(const ProductArgs& a, const int64_t* row, int b) {
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
      if constexpr (kTiny) {
        const uint8_t* p = a.scales + row[t] * a.nb;
        scales[t] = 0, shift[t] = 0;
        for (int s = 0; s < kStep && b + s < a.nb; ++s) scales[t] |= static_cast<uint32_t>(p[b + s]) << (8 * s);
      } else {
        const ScaleRow r(a.scales, row[t], a.nb, a.blocks);
        scales[t] = r.load(b);
        shift[t] = 8 * (b - min(b, r.last));
      }
      const u32x4* p = reinterpret_cast<const u32x4*>(a.codes) + row[t] * a.nb + b;
#pragma unroll
      for (int s = 0; s < kStep; ++s) codes[t][s] = p[kTiny && b + s >= a.nb ? 0 : s];
    }
  }
  // those in [b0, b1)
  template <int X>
  __device__ __forceinline__ void products(const XBlocks<X, kStep>& x, int b, int b0, int b1, f32x4* acc) const {
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
      const uint32_t word = scales[t] >> shift[t];
#pragma unroll
      for (int s = 0; s < kStep; ++s) {
        // what is not to be added: x is zero there, and the scale must be none that makes NaN
        const uint32_t byte = b + s >= b0 && b + s < b1 ? (word >> (8 * s)) & 255u : kOne;
        if constexpr (X == kXBf16 || X == kXTerms || X == kXTermRows) {
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const u32x4 w = cvt8(codes[t][s][q], scale_of(byte));
            acc[t] = mfma_bf16(w, x.v[s][q], acc[t]);
            if constexpr (X == kXTerms) acc[t] = mfma_bf16(w, x.v[s][4 + q], acc[t]);
          }
        } else {
          acc[t] = mfma_mx4(codes[t][s], byte, x.v[s][0], x.byte[s], acc[t]);
        }
      }
    }
  }
};

constexpr int kIds = 8;

// Ids of 64 * kIds pairs from p0 on, by lanes
struct Ids {
  int id[kIds];
  __device__ __forceinline__ void load(const ProductArgs& a, int p0) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int j = 0; j < kIds; ++j) id[j] = a.ids[min(p0 + 64 * j + lane, a.M - 1)];
  }
};

// Where a search for a group's pairs stands
struct Search {
  int count;  // pairs with its id
  int first;  // the first of them
  int p0, seen;  // where the next 16 are looked for from, and pairs before that
};

// The pairs with id `group` whose place among them is in [r0, r0 + 16), by one
// wave.  The first search (r0 = 0; ids: the first pairs') counts all of them, the
// others go on where the one before found what it looked for.
__device__ __forceinline__ void find_pairs(const ProductArgs& a, Ids ids, int group, int r0, int* row, Search& s) {
  const int lane = threadIdx.x & 63;
  int p0 = 0, seen = 0;
  if (r0 > 0) {
    p0 = s.p0, seen = s.seen;
  } else {
    s.first = s.p0 = a.M, s.seen = 0;
  }
  bool on = true;  // the next ones' place is not known yet
  for (; p0 < a.M && (r0 == 0 || on); p0 += 64 * kIds) {
    if (p0 > 0) ids.load(a, p0);
    const int before = seen;
#pragma unroll
    for (int j = 0; j < kIds; ++j) {
      const int p = p0 + 64 * j + lane;
      const bool mine = p < a.M && ids.id[j] == group;
      const uint64_t m = __ballot(mine);
      const int at = seen + __popcll(m & ((uint64_t{1} << lane) - 1)) - r0;
      if (mine && at >= 0 && at < 16) row[at] = p;
      if (seen == 0 && m) s.first = p0 + 64 * j + __ffsll(static_cast<long long>(m)) - 1;
      seen += __popcll(m);
    }
    if (on && seen > r0 + 16) s.p0 = p0, s.seen = before, on = false;
  }
  if (r0 == 0) s.count = seen;
}

// A workgroup takes a.run tiles of 16 * NT outputs (of both matrices for SwiGLU)
// of one group, for 16 of its rows at a time (where groups have more, gridDim.z
// workgroups take these in turn); its waves share K, kStep blocks of
// a lane at a time.  A tile's weights are on their way while the one before is
// multiplied, the first one's before the rows are known; the ids that tell them
// go before the weights, since loads return in order.  kHold: K is one step, and
// x stays in registers over the tiles.
// Bound by the weights' reads: the SwiGLU half of 64 tokens over 128 experts (K =
// 2,048, 214 MB) takes 46 us, 4.6 TB/s, the other (K = 768, 107 MB) 28 to 31.  One
// tile a workgroup, rows first and the weights behind them took 67 and 81: a
// workgroup then waits for three round trips one after the other.  One token's 8
// experts are latency (7.7 us: a launch, ids, weights, join), and so are 5,120
// outputs of one row (4.8 us).
template <int X, bool kSwiglu, int NT, int kStep, bool kHold, bool kTiny, typename Out, int kRows>
__global__ __launch_bounds__(kFewThreads) void mx4_few_kernel(ProductArgs a) {
  constexpr int kTiles = kSwiglu ? 2 * NT : NT;
  __shared__ f32x4 s_part[2][kFewWaves][kTiles][64];
  __shared__ int s_rows[kFewWaves][16];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 4, l16 = lane & 15;
  int* s_row = s_rows[wave];
  int group = blockIdx.y, begin = 0, count = 0;
  Ids ids;
  if constexpr (kRows == kRowsIds) {
    ids.load(a, 0);
    if (a.by_pair) group = a.ids[blockIdx.y];
    if (static_cast<unsigned>(group) >= static_cast<unsigned>(a.groups)) return;
  } else {
    count = a.M;
    if (a.start) {
      begin = min(max(a.start[group], 0), a.M);
      count = min(max(a.start[group + 1], 0), a.M) - begin;
    }
    if (count <= 16 * static_cast<int>(blockIdx.z)) return;
  }
  const int per = (a.nb + 4 * kFewWaves - 1) / (4 * kFewWaves);
  const int b0 = (wave * 4 + g) * per, b1 = min(b0 + per, a.nb);
  const int tiles = (a.N + 16 * NT - 1) / (16 * NT);
  const int from = static_cast<int>(blockIdx.x) * a.run, to = min(from + a.run, tiles);
  const int64_t first_row = static_cast<int64_t>(group) * (kSwiglu ? 2 : 1) * a.N;
  using Weights = WeightBlocks<kTiles, kStep, kTiny>;
  const auto load = [&](Weights& w, int tile, int s0) {
    int64_t row[kTiles];
#pragma unroll
    for (int t = 0; t < kTiles; ++t) row[t] = first_row + t / NT * a.N + min((tile * NT + t % NT) * 16 + l16, a.N - 1);
    w.load(a, row, Weights::window(a, b0 + s0));
  };
  Search search;
  Weights even, odd;
  load(even, from, 0);
  const int r_first = 16 * static_cast<int>(blockIdx.z), r_step = 16 * static_cast<int>(gridDim.z);
  for (int r0 = r_first;; r0 += r_step) {
    if constexpr (kRows == kRowsIds) {
      find_pairs(a, ids, group, r0, s_row, search);
      count = search.count;
      if (r0 >= count || (a.by_pair && search.first != static_cast<int>(blockIdx.y))) return;
      __builtin_amdgcn_wave_barrier();
    }
    const bool x_ok = r0 + l16 < count;
    int64_t x_row = 0;
    if (x_ok) x_row = kRows == kRowsIds ? s_row[l16] / a.xdiv : begin + r0 + l16;
    XBlocks<X, kStep> x;
    if (kHold) x.load(a, x_row, x_ok, Weights::window(a, b0), b0, b1);
    const auto take = [&](Weights& w, Weights& next, int tile) {
      if (tile + 1 < to) load(next, tile + 1, 0);
      f32x4 acc[kTiles];
#pragma unroll
      for (int t = 0; t < kTiles; ++t) acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
      if constexpr (kHold) {
        w.template products<X>(x, Weights::window(a, b0), b0, b1, acc);
      } else {
        for (int s0 = 0; s0 < per; s0 += kStep) {
          if (s0 > 0) load(w, tile, s0);
          const int b = Weights::window(a, b0 + s0);
          x.load(a, x_row, x_ok, b, b0 + s0, b1);
          w.template products<X>(x, b, b0 + s0, b1, acc);
        }
      }
      // outputs 4g .. 4g+3 of row l16
      const auto part = s_part[tile & 1];
#pragma unroll
      for (int t = 0; t < kTiles; ++t) part[wave][t][l16 * 4 + g] = acc[t];
      lds_barrier();
      for (int j = tid; j < 64 * NT; j += kFewThreads) {
        const int i = j / (4 * NT), q = j % (4 * NT), t = q / 4, at = i * 4 + q % 4;  // row i, four outputs
        f32x4 y = part[0][t][at];
#pragma unroll
        for (int v = 1; v < kFewWaves; ++v) y += part[v][t][at];
        if constexpr (kSwiglu) {
          f32x4 u = part[0][NT + t][at];
#pragma unroll
          for (int v = 1; v < kFewWaves; ++v) u += part[v][NT + t][at];
#pragma unroll
          for (int e = 0; e < 4; ++e) y[e] = swiglu(y[e], u[e]);
        }
        const int f = tile * 16 * NT + 4 * q;
        if (r0 + i >= count || f >= a.N) continue;
        const int64_t row = kRows == kRowsIds ? s_row[i] : begin + r0 + i;
        if constexpr (std::is_same<Out, Terms>::value) {  // N is a multiple of 32
          __bf16* out = static_cast<__bf16*>(a.out) + row * 2 * a.N + f;
          uint32_t low0, low1;
          *reinterpret_cast<u32x2*>(out) = u32x2{terms_of(y[0], y[1], &low0), terms_of(y[2], y[3], &low1)};
          *reinterpret_cast<u32x2*>(out + a.N) = u32x2{low0, low1};
          continue;
        } else {
          Out* out = static_cast<Out*>(a.out) + row * a.out_stride + f;
          if (a.wide_out && f + 4 <= a.N) {
            if constexpr (std::is_same<Out, float>::value)
              *reinterpret_cast<f32x4*>(out) = y;
            else
              *reinterpret_cast<u32x2*>(out) = u32x2{pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3])};
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (f + e < a.N) out[e] = static_cast<Out>(y[e]);
          }
        }
      }
    };
    for (int tile = from; tile < to; tile += 2) {
      take(even, odd, tile);
      if (tile + 1 < to) take(odd, even, tile + 1);
    }
    if (r0 + r_step >= count) return;
    load(even, from, 0);
    lds_barrier();
  }
}

// The second product of one or a few tokens with the gates' sum, one launch for
// both (5.3 us for 8 experts of 2048 x 768; two launches took 6.3 and 4.4): a
// workgroup takes 16 outputs of token blockIdx.y, its waves its experts
// (and shares of K where there are fewer experts than waves).
struct LastArgs {
  ProductArgs p;  // x: the SwiGLU's results, row t * K + k; ids
  const float* gates;
  const void* residual;
  int64_t residual_stride;
  int K;
};

constexpr int kLastThreads = 512;
constexpr int kLastWaves = kLastThreads / 64;

template <int X, int kStep, bool kTiny>
__global__ __launch_bounds__(kLastThreads) void mx4_last_kernel(LastArgs a) {
  constexpr int kTerms = X == kXTermRows ? 2 : 1;  // columns of the matrix instruction that the token takes
  __shared__ f32x4 s_part[kLastWaves][4];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 4, l16 = lane & 15;
  const int parts = a.K >= kLastWaves ? 1 : kLastWaves / a.K;
  const int per = (a.p.nb + 4 * parts - 1) / (4 * parts);
  const int f0 = blockIdx.x * 16, token = blockIdx.y;
  f32x4 sum = {0.f, 0.f, 0.f, 0.f};
  for (int i = wave; i < a.K * parts; i += kLastWaves) {
    const int pair = token * a.K + i / parts, e = a.p.ids[pair];
    if (static_cast<unsigned>(e) >= static_cast<unsigned>(a.p.groups)) continue;
    const float gate = a.gates[pair];
    const int b0 = (i % parts * 4 + g) * per, b1 = min(b0 + per, a.p.nb);
    const int64_t row = static_cast<int64_t>(e) * a.p.N + min(f0 + l16, a.p.N - 1);
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    WeightBlocks<1, kStep, kTiny> w;
    XBlocks<X, kStep> x;
    for (int s0 = 0; s0 < per; s0 += kStep) {
      const int b = WeightBlocks<1, kStep, kTiny>::window(a.p, b0 + s0);
      w.load(a.p, &row, b);
      x.load(a.p, pair, l16 < kTerms, b, b0 + s0, b1);
      w.template products<X>(x, b, b0 + s0, b1, &acc);
    }
    sum += gate * acc;
  }
  if constexpr (kTerms == 2)
#pragma unroll
    for (int j = 0; j < 4; ++j) sum[j] += __shfl_down(sum[j], 1);
  if (l16 == 0) s_part[wave][g] = sum;
  __syncthreads();
  if (tid >= 16 || f0 + tid >= a.p.N) return;
  float y = 0.f;
#pragma unroll
  for (int w = 0; w < kLastWaves; ++w) y += reinterpret_cast<const float*>(s_part[w])[tid];
  if (a.residual) y += static_cast<float>(static_cast<const __bf16*>(a.residual)[token * a.residual_stride + f0 + tid]);
  static_cast<__bf16*>(a.p.out)[token * a.p.out_stride + f0 + tid] = static_cast<__bf16>(y);
}

// -------------------------------------------------------- products of many rows

typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kTileThreads = 512;
constexpr int kTileWaves = kTileThreads / 64;
constexpr int kTileRows = 256;  // weight rows of a tile
constexpr int kXcds = 8;
constexpr int kTileWorkgroups = 256;  // one on each compute unit
constexpr int kBuffers = 3;
constexpr int kBand = 8;

__device__ const u32x4 kZeros = {0, 0, 0, 0};

template <int N>
using Const = std::integral_constant<int, N>;

template <int... I, typename F>
__device__ __forceinline__ void each_of(std::integer_sequence<int, I...>, F f) {
  (f(Const<I>{}), ...);
}
// f(0), f(1), .. f(N - 1), as constants
template <int N, typename F>
__device__ __forceinline__ void for_each(F f) {
  each_of(std::make_integer_sequence<int, N>{}, f);
}

// 16 bytes from global memory to `to` + 16 * lane of LDS
__device__ __forceinline__ void to_lds(const uint8_t* from, uint8_t* to) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) uint32_t*)from,
                                   (__attribute__((address_space(3))) uint32_t*)to, 16, 0, 0);
}

// Waits until at most kLeft of this wave's loads are on their way
template <int kLeft>
__device__ __forceinline__ void wait_loads() {
  // vmcnt in bits 3:0 and 15:14; the other counters' bits all ones: not waited for
  __builtin_amdgcn_s_waitcnt((kLeft & 15) | 0x0f70 | (kLeft >> 4) << 14);
  __builtin_amdgcn_sched_barrier(0);
}

// Where 16-byte piece c of a row of `kPieces` goes: piece c of the neighbouring
// rows that 16 lanes read together is spread over 256 bytes, all of the banks.
template <int kPieces>
__device__ __forceinline__ int swizzled(int row, int c) {
  return c ^ ((row / (16 / kPieces)) % kPieces);
}

template <int SEL>
__device__ __forceinline__ f32x16 mfma_mx4_32(u32x4 w, uint32_t w_scales, u32x4 x, uint32_t x_scales, f32x16 c) {
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(wide(w), wide(x), c, 4, 4, SEL, static_cast<int>(w_scales), SEL,
                                                         static_cast<int>(x_scales));
}

// Rows of a group
__device__ __forceinline__ int rows_of(const ProductArgs& a, int g, int* first) {
  *first = min(max(a.start[g], 0), a.M);
  return max(min(max(a.start[g + 1], 0), a.M) - *first, 0);
}

// Rows of x of a tile: with rows of two terms each of them takes two places
template <int X, int CT>
constexpr int kTileOf = X == kXTermRows ? 32 * CT : 64 * CT;

// A tile is 256 weight rows (128 outputs of both matrices for SwiGLU) by 64 * CT
// rows of one group (kXTermRows: 64 rows of two terms, each of a wave's 32 rows in
// two of its columns, which are added at the tile's end).  A workgroup stays on its compute unit and takes tiles one
// after the other, neighbouring tiles on one XCD.  K goes through LDS in stages
// of 128 bytes of a row in 4 bits (64 beside bf16 rows of x, whose stages are 256
// bytes), in three buffers that are loaded two stages ahead, over the tiles'
// borders: the next tile's first stages are on their way while this one's last
// are multiplied and its results written.  A wave takes 64 of the weight rows
// and half of the rows of x.
//
// What bounds it: with bf16 rows the matrix instructions (32 of each wave a stage,
// 37 cycles each in a loop of nothing else, 2,370 cycles of a SIMD; 8,192 x 5,120
// outputs at K = 2,048 take 152 to 164 us, 1.05 to 1.13 PFLOP/s, a library's bf16
// product of 8,192^3 reaches 1.14 to 1.35).  With both sides in 4 bits (41 cycles
// each, 1,320) what a compute unit gets from L2, 48 KB a stage, which takes 890
// cycles where nothing else is read: 60 us, 2.9 PFLOP/s, of them about 12 for the
// results' 84 MB, the matrix units busy for 41,000 of the 130,000 cycles that a wave
// lives; 3.6 PFLOP/s at K = 16,384 (the instructions by themselves reach 8.0, and 2.2
// in bf16).  Whole lines matter: L2 gives 55 bytes a cycle where a load's rows are 128
// bytes and 29 where they are 64, and a 64-byte stage of 256 x 128 tiles, two
// workgroups of four waves a compute unit, took 87 us.  Loads that are issued
// together hold up the products behind them, so they go between them, one at a time.
// Rows of two terms: 1,024 tokens of 6 of 64 experts, 1280 outputs of K = 896, take 50
// us, which bf16 rows took 37 for, with twice the products.
template <int X, bool kSwiglu, typename Out, int CT>
__global__ __launch_bounds__(kTileThreads, 2) void mx4_tile_kernel(ProductArgs a) {
  constexpr bool kMx4 = X == kXCodes;
  constexpr int KB = kMx4 ? 4 : 2;                  // blocks of a lane and stage
  constexpr int BL = 2 * KB;                        // blocks of a row and stage
  constexpr int AC = BL, BC = kMx4 ? BL : 4 * BL;   // 16-byte pieces of a row
  constexpr bool kTerms = X == kXTermRows;
  static_assert(!kTerms || CT == 2, "a column for each term");
  constexpr int TM = 64 * CT, TR = kTileOf<X, CT>;  // places for rows of x, and rows
  constexpr int kA = kTileRows * AC * 16, kB = TM * BC * 16;
  constexpr int AI = kTileRows * AC / kTileThreads, BI = TM * BC / kTileThreads;  // loads of a wave
  using Word = typename std::conditional<kMx4, uint64_t, uint32_t>::type;  // a row's scales of a stage
  // Scales come four stages at a time, in pieces of 16 bytes: by the stage, every
  // row would ask for a cache line of its own, as many as its codes do.
  constexpr int kAtOnce = 4, SC = kAtOnce * BL / 16;
  constexpr int SI = kMx4 ? 2 : 1;  // loads of a wave: the weights', x's
  // an array for each buffer: the compiler then sees that reads of one need not
  // wait for loads into another
  __shared__ __attribute__((aligned(16))) uint8_t s_a0[kA], s_a1[kA], s_a2[kA];
  __shared__ __attribute__((aligned(16))) uint8_t s_b0[kB], s_b1[kB], s_b2[kB];
  __shared__ Word s_sa[kAtOnce][kTileRows];
  __shared__ Word s_sb[kAtOnce][kMx4 ? TM : 1];
  // Tiles of the groups before each one, and where they are few their first rows
  // and rows, which would take a round trip a tile
  constexpr int kKept = spp::kMaxExpertsTopK / 3;
  __shared__ int s_before[spp::kMaxExpertsTopK];
  int* s_sum = reinterpret_cast<int*>(s_sa);
  const auto a_of = [&](auto buf) -> uint8_t* { return buf == 0 ? s_a0 : buf == 1 ? s_a1 : s_a2; };
  const auto b_of = [&](auto buf) -> uint8_t* { return buf == 0 ? s_b0 : buf == 1 ? s_b1 : s_b2; };
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int half = lane >> 5, l32 = lane & 31, wf = wave & 3, wt = wave >> 2;

  // tiles of the groups before each one (thread t: groups 2t and 2t + 1)
  int row_tiles = (a.M + TR - 1) / TR;
  if (a.start) {
    int n[2], first[2], rows[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      rows[j] = 2 * tid + j < a.groups ? rows_of(a, 2 * tid + j, &first[j]) : 0;
      n[j] = (rows[j] + TR - 1) / TR;
    }
    int incl = n[0] + n[1];
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int o = __shfl_up(incl, d);
      if (lane >= d) incl += o;
    }
    if (lane == 63) s_sum[wave] = incl;
    __syncthreads();
    int base = incl - n[0] - n[1];
    row_tiles = 0;
#pragma unroll
    for (int w = 0; w < kTileWaves; ++w) {
      base += w < wave ? s_sum[w] : 0;
      row_tiles += s_sum[w];
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int g = 2 * tid + j;
      if (g >= a.groups) break;
      s_before[g] = base + (j ? n[0] : 0);
      if (a.groups <= kKept) s_before[kKept + g] = first[j], s_before[2 * kKept + g] = rows[j];
    }
    __syncthreads();
  }
  row_tiles = __builtin_amdgcn_readfirstlane(row_tiles);
  const int64_t total = static_cast<int64_t>(row_tiles) * a.columns;
  const int64_t each = (total + kXcds - 1) / kXcds;
  const int64_t xcd_first = blockIdx.x % kXcds * each, xcd_end = min(xcd_first + each, total);
  const int64_t stride = gridDim.x / kXcds;
  int64_t job = xcd_first + blockIdx.x / kXcds;
  if (job >= xcd_end) return;

  struct Tile {
    int group, first, count, column;
  };
  const auto find = [&](int64_t j) {
    // bands of kBand row tiles, in each of them column by column: those that run
    // together on an XCD share weights and rows of x in its L2
    const int band = static_cast<int>(j / (kBand * a.columns)), tiles = min(kBand, row_tiles - band * kBand);
    const int in_band = static_cast<int>(j - static_cast<int64_t>(band) * kBand * a.columns);
    const int tile = band * kBand + in_band % tiles;
    Tile t{0, tile * TR, min(a.M - tile * TR, TR), in_band / tiles};
    if (a.start) {
      int n = 0;
      for (int g = lane; g - lane < a.groups; g += 64) n += __popcll(__ballot(g < a.groups && s_before[g] <= tile));
      t.group = n - 1;  // the last one with no more tiles before it: those without rows have as many as the next
      int first, rows;
      if (a.groups <= kKept)
        first = s_before[kKept + t.group], rows = s_before[2 * kKept + t.group];
      else
        rows = rows_of(a, t.group, &first);
      const int at = (tile - s_before[t.group]) * TR;
      t.first = __builtin_amdgcn_readfirstlane(first + at);
      t.count = __builtin_amdgcn_readfirstlane(min(rows - at, TR));
    }
    return t;
  };

  // what this lane loads: pieces that go to its places, and a row's scales (of the
  // weights in the first four waves, of x in the others)
  int ca[AI], cb[BI];
#pragma unroll
  for (int i = 0; i < AI; ++i) {
    const int idx = (i * kTileWaves + wave) * 64 + lane;
    ca[i] = swizzled<AC>(idx / AC, idx % AC);
  }
#pragma unroll
  for (int i = 0; i < BI; ++i) {
    const int idx = (i * kTileWaves + wave) * 64 + lane;
    cb[i] = swizzled<BC>(idx / BC, idx % BC);
  }
  // of scales: piece scale_c of a row of the weights, and of x (the last row's
  // again where there are more lanes than rows)
  const int scale_q = wave * 64 + lane, scale_c = scale_q % SC;
  const int scale_ra = min(scale_q / SC, kTileRows - 1), scale_rb = min(scale_q / SC, TM - 1);

  // The place in LDS that load i of this lane goes to, of TM
  const auto place_at = [&](int i) { return ((i * kTileWaves + wave) * 64 + lane) / BC; };
  // Rows of x of a tile; the pairs' loads are on their way until they are used
  int x_pair[BI], x_pair_scale = 0;
  const auto fetch = [&](const Tile& t) {
#pragma unroll
    for (int i = 0; i < BI; ++i) {
      const int r = place_at(i), p = t.first + min(kTerms ? r / 64 * 32 + r % 32 : r, t.count - 1);
      x_pair[i] = a.pair ? a.pair[p] : p;
    }
    if (kMx4) {
      const int p = t.first + min(scale_rb, t.count - 1);
      x_pair_scale = a.pair ? a.pair[p] : p;
    }
  };
  uint32_t pa[AI];         // bytes from the start of a window of weight rows
  const uint8_t* base[2];  // the windows: one, or SwiGLU's two (a load's rows are in one of them)
  const uint8_t* pb[BI];
  int64_t scale_at[SI];
  int scale_last[SI], stage = 0;
  const auto setup = [&](const Tile& t) {
    // LDS row r holds the weight row whose sums come to lie where the results are
    // written from: a lane then has neighbouring outputs
    const int window = t.column * (kSwiglu ? kTileRows / 2 : kTileRows);
    const auto weight_row = [&](int r) {
      const int rho = r & 31, w = r >> 6, hh = (rho >> 2) & 1, j = 4 * (rho >> 3) + (rho & 3), up = (r >> 5) & 1;
      return min(window + (kSwiglu ? w * 32 + 16 * hh + j : w * 64 + 32 * hh + 16 * up + j), a.N - 1);
    };
    const int64_t first_row = static_cast<int64_t>(t.group) * (kSwiglu ? 2 : 1) * a.N;
    base[0] = a.codes + (first_row + window) * a.nb * 16;
    base[1] = kSwiglu ? base[0] + static_cast<int64_t>(a.N) * a.nb * 16 : base[0];
#pragma unroll
    for (int i = 0; i < AI; ++i)
      pa[i] = static_cast<uint32_t>(weight_row(((i * kTileWaves + wave) * 64 + lane) / AC) - window) *
              static_cast<uint32_t>(a.nb) * 16;
#pragma unroll
    for (int i = 0; i < BI; ++i)
      pb[i] = static_cast<const uint8_t*>(a.x) + (x_pair[i] / a.xdiv) * a.x_stride + cb[i] * 16 +
              (kTerms && place_at(i) & 32 ? a.x_stride / 2 : 0);
#pragma unroll
    for (int i = 0; i < SI; ++i) {
      const int64_t row = i == 0 ? first_row + (kSwiglu && (scale_ra >> 5 & 1) ? a.N : 0) + weight_row(scale_ra) : x_pair_scale / a.xdiv;
      scale_at[i] = row * a.nb;
      scale_last[i] = static_cast<int>(min((i == 0 ? a.blocks : a.x_blocks) - 16 - scale_at[i], int64_t{1} << 20));
    }
    stage = 0;
  };

  const int stages = max((a.nb + BL - 1) / BL, 2);  // two at least: one may be of zeros
  struct Scales {
    u32x4 v[SI];
    int last[SI];
  };
  // A lane's piece of four stages from `st` on, read whole and in bounds: near the
  // end of all scales it starts earlier, by up to 15 bytes.  All are at least 16, but
  // for those of x that the experts' call quantises itself: its codes, 256 bytes or
  // more of the workspace, lie in front of them
  const auto load_scales = [&](Scales& to, int st) {
    const int b = st * BL + 16 * scale_c;
#pragma unroll
    for (int i = 0; i < SI; ++i) {
      to.last[i] = scale_last[i];
      __builtin_memcpy(&to.v[i], (i == 0 ? a.scales : a.x_scales) + scale_at[i] + min(b, to.last[i]), 16);
    }
  };
  const auto put_scales = [&](const Scales& from, int st) {
    const int b = st * BL + 16 * scale_c;
#pragma unroll
    for (int i = 0; i < SI; ++i) {
      uint64_t lo = from.v[i][0] | static_cast<uint64_t>(from.v[i][1]) << 32, hi = from.v[i][2] | static_cast<uint64_t>(from.v[i][3]) << 32;
      int skip = min(b - min(b, from.last[i]), 15);  // bytes before block b
      if (skip >= 8) lo = hi, hi = 0, skip -= 8;
      if (skip > 0) {
        lo = lo >> (8 * skip) | hi << (64 - 8 * skip);
        hi >>= 8 * skip;
      }
      const auto whole = [](uint64_t w, int left) {  // past the row's end: 1
        const uint64_t keep = left >= 8 ? ~uint64_t{0} : left <= 0 ? 0 : (uint64_t{1} << (8 * left)) - 1;
        return (w & keep) | (0x7f7f7f7f7f7f7f7full & ~keep);
      };
      lo = whole(lo, a.nb - b), hi = whole(hi, a.nb - b - 8);
      const int r = scale_q / SC;
      if constexpr (kMx4) {
        if (i == 0) {
          s_sa[2 * scale_c][r] = lo, s_sa[2 * scale_c + 1][r] = hi;
        } else if (r < TM) {
          s_sb[2 * scale_c][r] = lo, s_sb[2 * scale_c + 1][r] = hi;
        }
      } else if (r < kTileRows) {
        s_sa[0][r] = static_cast<uint32_t>(lo), s_sa[1][r] = static_cast<uint32_t>(lo >> 32);
        s_sa[2][r] = static_cast<uint32_t>(hi), s_sa[3][r] = static_cast<uint32_t>(hi >> 32);
      }
    }
  };
  // Load l of the next stage into a buffer: always as many, since waits count them
  constexpr int kLoads = AI + BI;
  const auto issue = [&](auto l, auto buf) {
    const int b0 = stage * BL;
    if constexpr (l < AI) {
      constexpr int i = l;
      to_lds(base[((i * kTileWaves + wave) * (64 / AC) >> 5) & 1] + (pa[i] + (b0 + ca[i] < a.nb ? b0 + ca[i] : 0) * 16),
             a_of(buf) + (i * kTileWaves + wave) * 1024);
    } else {
      constexpr int i = l - AI;
      to_lds(b0 + cb[i] / (BC / BL) < a.nb ? pb[i] + static_cast<int64_t>(b0) * (BC / BL * 16)
                                           : reinterpret_cast<const uint8_t*>(&kZeros),
             b_of(buf) + (i * kTileWaves + wave) * 1024);
    }
    if constexpr (l == kLoads - 1) ++stage;
  };
  f32x16 acc[2][CT];
  // where this lane reads: its row's first piece, and the others by exclusive or
  // with their number; its row's scales of its half.  Hidden from the compiler,
  // which would keep an address of its own for every read of every buffer.
  uint32_t at_a = (l32 * AC + swizzled<AC>(l32, half * KB)) * 16 + wf * 64 * AC * 16;
  uint32_t at_b = (l32 * BC + swizzled<BC>(l32, half * (BC / 2))) * 16 + wt * 32 * CT * BC * 16;
  uint32_t at_sa = (wf * 64 + l32) * sizeof(Word) + half * KB, at_sb = (wt * 32 * CT + l32) * sizeof(Word) + half * KB;
  // Half of a stage's operands: two blocks, or one beside bf16 rows of x
  constexpr int HA = kMx4 ? 2 : 1, HB = kMx4 ? 2 : 4;
  struct Half {
    u32x4 a[HA][2], b[HB][CT];
  };
  struct StageScales {
    uint32_t a[2], b[CT];
  };
  constexpr int kReads = 2 * HA + HB * CT;
  const auto read = [&](Half& h, const uint8_t* in_a, const uint8_t* in_b, auto which, auto r) {
    if constexpr (r < 2 * HA) {
      constexpr int k = r / 2, i = r % 2;
      h.a[k][i] = *reinterpret_cast<const u32x4*>(in_a + (at_a ^ ((which * HA + k) << 4)) + i * 32 * AC * 16);
    } else {
      constexpr int k = (r - 2 * HA) / CT, c = (r - 2 * HA) % CT;
      h.b[k][c] = *reinterpret_cast<const u32x4*>(in_b + (at_b ^ ((which * HB + k) << 4)) + c * 32 * BC * 16);
    }
  };
  const auto read_scales = [&](StageScales& to, int st) {
    asm volatile("" : "+v"(at_sa), "+v"(at_sb));
    const auto scale = [&](const Word* in, uint32_t at, int i) -> uint32_t {
      const uint8_t* p = reinterpret_cast<const uint8_t*>(in) + at + i * 32 * sizeof(Word);
      return kMx4 ? *reinterpret_cast<const uint32_t*>(p) : *reinterpret_cast<const uint16_t*>(p);
    };
#pragma unroll
    for (int i = 0; i < 2; ++i) to.a[i] = scale(s_sa[st % kAtOnce], at_sa, i);
#pragma unroll
    for (int c = 0; c < CT; ++c) to.b[c] = kMx4 ? scale(s_sb[st % kAtOnce], at_sb, c) : 0;
  };
  // The products of half a stage.  Between them, one at a time, go the reads of
  // the half after it and half of the next stage's loads: eight waves that issue
  // all of them at once wait 1,300 cycles until they are accepted.
  const auto products = [&](const Half& h, const StageScales& scales, auto which, Half& next, auto next_buf, auto load_buf) {
    asm volatile("" : "+v"(at_a), "+v"(at_b));
    constexpr int kProducts = (kMx4 ? 4 : 8) * CT, kFirst = (kLoads + 1) / 2;
    constexpr int kFrom = which == 0 ? 0 : kFirst, kCount = which == 0 ? kFirst : kLoads - kFirst;
    u32x4 w[2];
    for_each<kProducts>([&](auto k) {
      constexpr int b = k / (2 * CT), i = k / CT % 2, c = k % CT;
      if constexpr (kMx4) {
        acc[i][c] = mfma_mx4_32<2 * which + b>(h.a[b][i], scales.a[i], h.b[b][c], scales.b[c], acc[i][c]);
      } else {
        if constexpr (c == 0) w[i] = cvt8(h.a[0][i][b], scale_of((scales.a[i] >> (8 * which)) & 255u));
        acc[i][c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, w[i]),
                                                            __builtin_bit_cast(bf16x8, h.b[b][c]), acc[i][c], 0, 0, 0);
      }
      for_each<(k + 1) * kReads / kProducts - k * kReads / kProducts>([&](auto r) {
        read(next, a_of(next_buf), b_of(next_buf), Const<1 - which>{}, Const<k * kReads / kProducts + r>{});
      });
      for_each<(k + 1) * kCount / kProducts - k * kCount / kProducts>([&](auto l) {
        issue(Const<kFrom + k * kCount / kProducts + l>{}, load_buf);
      });
      __builtin_amdgcn_sched_barrier(0);
    });
    // else the compiler moves the products over the branches and barriers that follow
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int c = 0; c < CT; ++c) asm volatile("" : "+v"(acc[i][c]));
  };
  // A lane holds 32 neighbouring outputs of a row (16 of both for SwiGLU).  bf16
  // results go through the buffer of the last stage, which nothing is loaded into
  // now, so that whole cache lines are written.
  const auto write_out = [&](const Tile& t, auto buf) {
    wait_loads<0>();  // the next tile's first two stages
    uint8_t* mine = kA >= 8 * 4096 || wave < 4 ? a_of(buf) + wave * 4096 : b_of(buf) + (wave - 4) * 4096;
    constexpr int kColumns = TR / 64;
    if constexpr (kTerms) acc[0][0] += acc[0][1], acc[1][0] += acc[1][1];
#pragma unroll
    for (int c = 0; c < kColumns; ++c) {
      const int r0 = (wt * kColumns + c) * 32, r = r0 + l32;
      const int64_t row = t.first + r;
      const bool ok = r < t.count;
      if constexpr (kSwiglu) {
        const int f0 = t.column * (kTileRows / 2) + wf * 32, f = f0 + 16 * half;
        if (f0 >= a.N) continue;  // N is a multiple of 32
        float y[16];
#pragma unroll
        for (int j = 0; j < 16; ++j) y[j] = swiglu(acc[0][c][j], acc[1][c][j]);
        if constexpr (kMx4) {
          uint32_t top = 0;
#pragma unroll
          for (int j = 0; j < 16; ++j) top = max(top, __float_as_uint(y[j]) & 0x7fffffffu);
          top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), 32)));
          const uint32_t byte = byte_of(top);
          const float scale = scale_of(byte);
          u32x2 w;
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            uint32_t v = 0;
            v = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(v, y[8 * k], y[8 * k + 1], scale, 0);
            v = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(v, y[8 * k + 2], y[8 * k + 3], scale, 1);
            v = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(v, y[8 * k + 4], y[8 * k + 5], scale, 2);
            v = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(v, y[8 * k + 6], y[8 * k + 7], scale, 3);
            w[k] = byte == kNanByte ? 0u : v;
          }
          if (ok) {
            *reinterpret_cast<u32x2*>(static_cast<uint8_t*>(a.out) + (row * a.N + f) / 2) = w;
            if (half == 0) a.out_scales[(row * a.N + f) / 32] = static_cast<uint8_t>(byte);
          }
        } else {
          // two terms (Out), 64 bytes of 32 rows each
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            u32x4 high, low;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              uint32_t l;
              high[j] = terms_of(y[8 * k + 2 * j], y[8 * k + 2 * j + 1], &l);
              low[j] = l;
            }
            uint8_t* to = mine + (l32 * 4 + swizzled<4>(l32, half * 2 + k)) * 16;
            *reinterpret_cast<u32x4*>(to) = high;
            *reinterpret_cast<u32x4*>(to + 2048) = low;
          }
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const int s = k % 2 * 16 + lane / 4, q = lane % 4, term = k / 2;
            const u32x4 v = *reinterpret_cast<const u32x4*>(mine + term * 2048 + (s * 4 + swizzled<4>(s, q)) * 16);
            if (r0 + s < t.count)
              *reinterpret_cast<u32x4*>(static_cast<__bf16*>(a.out) + (int64_t{2} * (t.first + r0 + s) + term) * a.N + f0 + 8 * q) = v;
          }
        }
      } else {
        const int f0 = t.column * kTileRows + wf * 64, f = f0 + 32 * half;
        if (a.wide_out && f0 + 64 <= a.N) {
          // 128 bytes of 32 rows at a time: 64 bf16 outputs, or 32 in fp32, which one
          // half of the lanes holds
          constexpr bool kF32 = std::is_same<Out, float>::value;
          constexpr int kEach = 16 / static_cast<int>(sizeof(Out));
#pragma unroll
          for (int part = 0; part < (kF32 ? 2 : 1); ++part) {
            if (!kF32 || half == part) {
#pragma unroll
              for (int k = 0; k < 32 / kEach; ++k) {
                u32x4 v;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                  const auto y = [&](int m) { return acc[m / 16][c][m % 16]; };
                  v[j] = kF32 ? __float_as_uint(y(4 * k + j)) : pack_bf16(y((8 * k + 2 * j) % 32), y((8 * k + 2 * j + 1) % 32));
                }
                const int piece = kF32 ? k : half * 4 + k;
                *reinterpret_cast<u32x4*>(mine + (l32 * 8 + swizzled<8>(l32, piece)) * 16) = v;
              }
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const int s = k * 8 + lane / 8, q = lane % 8;
              const u32x4 v = *reinterpret_cast<const u32x4*>(mine + (s * 8 + swizzled<8>(s, q)) * 16);
              if (r0 + s < t.count)
                *reinterpret_cast<u32x4*>(static_cast<Out*>(a.out) + (t.first + r0 + s) * a.out_stride + f0 + 32 * part + kEach * q) = v;
            }
          }
          continue;
        }
        if (!ok || f >= a.N) continue;
        Out* out = static_cast<Out*>(a.out) + row * a.out_stride + f;
#pragma unroll
        for (int j = 0; j < 32; ++j)
          if (f + j < a.N) out[j] = static_cast<Out>(acc[j / 16][c][j % 16]);
      }
    }
  };

  Tile t = find(job), next = t;
  fetch(t);
  setup(t);
  Scales scales;
  Half first, second;
  StageScales now, then;
  load_scales(scales, 0);
  for_each<kLoads>([&](auto l) { issue(l, Const<0>{}); });
  for_each<kLoads>([&](auto l) { issue(l, Const<1>{}); });
  wait_loads<0>();
  put_scales(scales, 0);
  lds_barrier();
  read_scales(now, 0);
  for_each<kReads>([&](auto r) { read(first, s_a0, s_b0, Const<0>{}, r); });
  int st = 0;
  bool more;
  const auto begin = [&]() {
    st = 0;
    job += stride;
    more = job < xcd_end;
    if (more) {
      next = find(job);
      fetch(next);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int c = 0; c < CT; ++c)
#pragma unroll
        for (int j = 0; j < 16; ++j) acc[i][c][j] = 0.f;
  };
  // A stage; whether it was the last one.  Its first half is in registers when it
  // begins, and the next one's when it ends, so that the matrix units have work on
  // both sides of the barrier that the stage's loads need.
  const auto step = [&](auto buf) -> bool {
    constexpr int kNext = (buf + 1) % kBuffers, kAfter = (buf + 2) % kBuffers;
    if (st + 2 == stages && more) {
      setup(next);
      __builtin_amdgcn_s_waitcnt(0xc07f);  // scalar loads: not waited for later, with the LDS reads
    }
    products(first, now, Const<0>{}, second, buf, Const<kAfter>{});
    wait_loads<(kLoads + 1) / 2>();  // all but what this stage has issued: the next one is there
    lds_barrier();
    const bool last = st + 1 == stages;
    if (last || st % kAtOnce == kAtOnce - 1) {  // the scales there are no longer read
      put_scales(scales, last ? 0 : st + 1);
      lds_barrier();
    }
    if (st + 2 == stages || (st % kAtOnce == kAtOnce - 2 && st + 2 < stages)) load_scales(scales, st + 2 == stages ? 0 : st + 2);
    read_scales(then, last ? 0 : st + 1);
    products(second, now, Const<1>{}, first, Const<kNext>{}, Const<kAfter>{});
    now = then;
    if (++st < stages) return false;
    write_out(t, buf);
    if (!more) return true;
    lds_barrier();  // the buffer is loaded into again
    t = next;
    begin();
    return false;
  };
  begin();
  if (!step(Const<0>{}))
    while (!step(Const<1>{}) && !step(Const<2>{}) && !step(Const<0>{})) {
    }
  wait_loads<0>();  // nothing may come to this workgroup's LDS after its end
}

// ------------------------------------------------------------------ host side

const char* matrix_why(const spp_mx4_matrix* m) {
  if (!m) return "a matrix is NULL";
  if (m->cols < 32 || m->cols > 1 << 17 || m->cols % 32 != 0) return "cols must be a multiple of 32, at most 2^17";
  if (m->rows < 0 || m->rows > INT32_MAX || m->rows * m->cols > int64_t{1} << 40)
    return "rows must be in [0, 2^31), and rows * cols at most 2^40";
  if (m->rows > 0 && (!m->codes || !m->scales)) return "codes and scales must not be NULL";
  if (!aligned16(m->codes)) return "codes must be 16-byte aligned";
  return nullptr;
}

int64_t code_bytes(const spp_mx4_matrix& m) { return m.rows * (m.cols / 2); }
int64_t scale_bytes(const spp_mx4_matrix& m) { return m.rows * (m.cols / 32); }

bool over(const spp_mx4_matrix& m, const Rows& r) {
  return meet(r, array(m.codes, code_bytes(m))) || meet(r, array(m.scales, scale_bytes(m)));
}

unsigned quant_grid(int64_t words) {
  return static_cast<unsigned>(std::min<int64_t>((words + kQuantThreads - 1) / kQuantThreads, 1 << 20));
}

hipError_t launch3(void (*kernel)(ProductArgs), unsigned x, unsigned y, unsigned z, unsigned threads, const ProductArgs& a,
                   hipStream_t st) {
  void* params[] = {const_cast<ProductArgs*>(&a)};
  return hipLaunchKernel(reinterpret_cast<const void*>(kernel), dim3(x, y, z), dim3(threads), params, 0, st);
}

constexpr int kLastTokens = 2;  // at most, of mx4_last_kernel
constexpr int kMaxM = 1 << 24;
constexpr int kMaxN = 1 << 20;
constexpr int64_t kMaxOutputs = int64_t{1} << 36;  // below 2^24 workgroups in every form

const char* product_why(const spp_mx4_matrix* w, int32_t groups, const int32_t* start, int32_t M, int32_t dtype,
                        const void* out, int64_t out_stride) {
  if (const char* why = matrix_why(w)) return why;
  if (const char* why = dtype_why(dtype)) return why;
  if (groups < 1 || groups > spp::kMaxExpertsTopK) return "groups must be in [1, 1024]";
  if (w->rows < groups || w->rows % groups != 0) return "the weights' rows must be a positive multiple of groups";
  if (w->rows / groups > kMaxN) return "a group's rows of weights must be at most 2^20";
  if (!start && groups != 1) return "start must not be NULL with more than one group";
  if (!aligned(start, 4)) return "start must be aligned to its elements";
  if (M < 0 || M > kMaxM) return "M must be in [0, 2^24]";
  const int64_t N = w->rows / groups;
  if (M * N > kMaxOutputs) return "M times a group's rows of weights must be at most 2^36";
  if (M == 0) return nullptr;
  if (!out || !aligned(out, dtype == SPP_DTYPE_BF16 ? 2 : 4)) return "out must not be NULL, and aligned to its elements";
  if (out_stride < N || out_stride > int64_t{1} << 30) return "out's stride must be at least a row, at most 2^30 elements";
  const Rows to = rows_from(out, out_stride, N, M, dtype == SPP_DTYPE_BF16 ? 2 : 4);
  if (over(*w, to) || meet(to, array(start, (groups + 1) * 4)))
    return "out must not overlap an input";
  return nullptr;
}

ProductArgs product_of(const spp_mx4_matrix& w, int32_t groups, const int32_t* start, int32_t M, void* out,
                       int64_t out_stride) {
  ProductArgs a{};
  a.codes = static_cast<const uint8_t*>(w.codes);
  a.scales = static_cast<const uint8_t*>(w.scales);
  a.nb = w.cols / 32;
  a.blocks = w.rows * a.nb;
  a.N = static_cast<int>(w.rows / groups);
  a.start = start;
  a.groups = groups;
  a.M = M;
  a.xdiv = 1;
  a.out = out;
  a.out_stride = out_stride;
  return a;
}

bool wide_rows(const void* out, int64_t stride, size_t elem) {
  return aligned16(out) && stride * static_cast<int64_t>(elem) % 16 == 0;
}

// Blocks of a lane at a time: the fewest that are loaded in vain, then the most
int few_step(int per) {
  int best = 4;
  for (int s = 3; s > 1; --s)
    if ((per + s - 1) / s * s < (per + best - 1) / best * best) best = s;
  return best;
}

// Sixteens of outputs a workgroup of few rows takes: as many as leave four
// workgroups to a compute unit, and a lane about 8 loads at once
int few_outputs(const ProductArgs& a, int64_t groups, bool swiglu, int step) {
  for (int nt = swiglu ? 2 : 4; nt > 1; nt /= 2)
    if (nt * (swiglu ? 2 : 1) * step <= 8 && groups * ((a.N + 16 * nt - 1) / (16 * nt)) >= 1024) return nt;
  return 1;
}

constexpr int kRunGroups = 512;  // workgroups that are resident together, about

template <int X, bool kSwiglu, int NT, int kStep, typename Out, int kRows>
hipError_t launch_few(ProductArgs a, int64_t groups, bool hold, hipStream_t st) {
  const int tiles = (a.N + 16 * NT - 1) / (16 * NT);
  const int64_t all = groups * tiles, slices = kRows == kRowsStart ? (a.M / groups + 15) / 16 : 1;
  a.run = static_cast<int>(std::min<int64_t>((all + kRunGroups - 1) / kRunGroups, 16));
  // rows beyond 16 of a group beside one another, until the card is full
  const int64_t z = std::min<int64_t>(std::max<int64_t>(kRunGroups * 4 / all, 1), std::max<int64_t>(slices, 1));
  auto kernel = hold ? mx4_few_kernel<X, kSwiglu, NT, kStep, true, false, Out, kRows>
                     : mx4_few_kernel<X, kSwiglu, NT, kStep, false, false, Out, kRows>;
  if constexpr (NT == 1 && kStep == 2)
    if (a.nb < kStep || a.blocks < 4) kernel = mx4_few_kernel<X, kSwiglu, NT, kStep, true, true, Out, kRows>;
  return launch3(kernel, static_cast<unsigned>((tiles + a.run - 1) / a.run), static_cast<unsigned>(groups),
                 static_cast<unsigned>(z), kFewThreads, a, st);
}

template <int X, bool kSwiglu, int NT, typename Out, int kRows>
hipError_t launch_few(const ProductArgs& a, int64_t groups, int step, bool hold, hipStream_t st) {
  return step == 4   ? launch_few<X, kSwiglu, NT, 4, Out, kRows>(a, groups, hold, st)
         : step == 3 ? launch_few<X, kSwiglu, NT, 3, Out, kRows>(a, groups, hold, st)
                     : launch_few<X, kSwiglu, NT, 2, Out, kRows>(a, groups, hold, st);
}

template <int X, bool kSwiglu, typename Out, int kRows>
hipError_t launch_few(ProductArgs a, int64_t groups, hipStream_t st) {
  a.wide_out = wide_rows(a.out, a.out_stride, sizeof(Out));
  const int per = (a.nb + 4 * kFewWaves - 1) / (4 * kFewWaves);
  const bool tiny = a.nb < 4 || a.blocks < 4;
  const int step = tiny ? 2 : few_step(per), nt = tiny ? 1 : few_outputs(a, groups, kSwiglu, step);
  if constexpr (!kSwiglu)
    if (nt == 4) return launch_few<X, kSwiglu, 4, Out, kRows>(a, groups, step, per <= step, st);
  return nt == 2 ? launch_few<X, kSwiglu, 2, Out, kRows>(a, groups, step, per <= step, st)
                 : launch_few<X, kSwiglu, 1, Out, kRows>(a, groups, step, per <= step, st);
}

template <int X, bool kSwiglu, typename Out, int CT>
hipError_t launch_tile(ProductArgs a, hipStream_t st) {
  constexpr int kOutputs = kSwiglu ? kTileRows / 2 : kTileRows;
  a.columns = (a.N + kOutputs - 1) / kOutputs;
  a.wide_out = wide_rows(a.out, a.out_stride, sizeof(Out));
  // groups with a last tile of their own: at most one a group, and one a row
  const int64_t tiles = (a.M / kTileOf<X, CT> + std::min(a.groups, a.M)) * static_cast<int64_t>(a.columns);
  const int64_t grid = std::min<int64_t>((tiles + kXcds - 1) / kXcds * kXcds, kTileWorkgroups);
  return launch(mx4_tile_kernel<X, kSwiglu, Out, CT>, static_cast<unsigned>(grid), kTileThreads, a, st);
}

// What a product takes, about, in us: rounds of 256 tiles, each of them a start
// and its stages; 128 rows instead of 64 take 1.2 (x in 4 bits) to 1.45 times as
// long.  Measured for one round at K = 512 .. 4,096: 7.4 .. 34 (bf16), 6.0 .. 15
// (4 bits).  A group's last tile is half full on average.
float tile_us(int rows, int64_t M, int groups, int outputs, int nb, bool mx4) {
  const int64_t tiles = M / rows + std::max<int64_t>(std::min<int64_t>(groups, M) / 2, 1);
  const int64_t jobs = tiles * ((outputs + kTileRows - 1) / kTileRows);
  const float round = mx4 ? 4.9f + 0.62f * ((nb + 7) / 8) : 4.f + 0.85f * ((nb + 3) / 4);
  return (jobs + kTileWorkgroups - 1) / kTileWorkgroups * round * (rows == 64 ? 1.f : mx4 ? 1.2f : 1.45f);
}

// Rows of x that a tile takes
int tile_rows(int64_t M, int groups, int outputs, int nb, bool mx4) {
  return tile_us(128, M, groups, outputs, nb, mx4) < tile_us(64, M, groups, outputs, nb, mx4) ? 128 : 64;
}

// Whether the experts' products go by tiles, behind a sort: from 10 pairs an
// expert on (8 with 4-bit products), and 1 GFLOP.  Measured, few rows against
// tiles: 128 experts of 2048 x 768 with 6 pairs each 116 : 141 us (bf16), 104 : 93
// (4 bits), with 8 146 : 137 and 127 : 94, with 10 151 : 141 and 132 : 96; 64 of 1280 x
// 896 with 9 each 62 : 82 and 54 : 55, with 10 74 : 70 and 64 : 50; 24 of 1024 x 768
// with 8 each 30 : 36 and 29 : 28, with 12 31 : 37 and 30 : 28, with 16 41 : 37 and
// 39 : 29; 8 of 1024 x 512 with 24 each (0.6 GFLOP) 24 : 31 and 28 : 26.  No one
// number of pairs is the border at every width: at these the rule costs up to 1.2.
// From 64 pairs an expert on in any case: few rows search all pairs.
bool by_tiles(int64_t P, int n, int64_t D, int64_t I, bool mx4) {
  return P >= int64_t{64} * n || (P >= (mx4 ? 8 : 10) * int64_t{n} && 6 * P * D * I >= 1000000000);
}
// The most pairs of a call that goes otherwise
int64_t most_few_pairs(int n, int64_t D, int64_t I) {
  return std::min(int64_t{64} * n, std::max(int64_t{10} * n, 1000000000 / (6 * D * I) + 1));
}

template <int X, bool kSwiglu, typename Out>
hipError_t launch_tiles(const ProductArgs& a, int rows, hipStream_t st) {
  return rows == 128 ? launch_tile<X, kSwiglu, Out, 2>(a, st) : launch_tile<X, kSwiglu, Out, 1>(a, st);
}

template <int X>
hipError_t launch_product(const ProductArgs& a, int32_t dtype, hipStream_t st) {
  constexpr bool kMx4 = X == kXCodes;
  const int rows = tile_rows(a.M, a.groups, a.N, a.nb, kMx4);
  // Few rows: a start, and 108 (173) TFLOP/s, measured with 5,120 outputs at K =
  // 2,048: 9.9 us for 32 rows and 26.5 for 128, which tiles take 17.4 and 17.7 for.
  const float few_us = 3.f + 2e-6f * static_cast<float>(a.M) * static_cast<float>(a.N) * 32.f * static_cast<float>(a.nb) /
                                 (kMx4 ? 173.f : 108.f);
  // (tiles read scales 16 bytes at a time: of fewer, the few rows' kernel alone takes any number)
  if (a.blocks >= 16 && a.M >= 16 && few_us > tile_us(rows, a.M, a.groups, a.N, a.nb, kMx4))
    return dtype == SPP_DTYPE_BF16 ? launch_tiles<X, false, __bf16>(a, rows, st) : launch_tiles<X, false, float>(a, rows, st);
  return dtype == SPP_DTYPE_BF16 ? launch_few<X, false, __bf16, kRowsStart>(a, a.groups, st)
                                 : launch_few<X, false, float, kRowsStart>(a, a.groups, st);
}

// The parts of a workspace of the experts' call
struct Space {
  size_t h, y, start, pair, place, sort, xq, xq_scales, h_scales, bytes;
};

size_t up256(size_t n) { return (n + 255) & ~size_t{255}; }

// h: the SwiGLU's results, y: the experts' results, which are terms of the gates'
// sum and stay in fp32.  h goes into the second product as two bf16 terms, or in 4
// bits.  Few rows an expert: at the pairs' own places, h in fp32 or terms (the
// weights' reads bound such calls).  Many: sorted.  There too both are paid for, so
// that what a call keeps does not go by its number of tokens: with h rounded to bf16
// 1,024 tokens of 6 of 64 experts of 1280 x 896 take 112 us instead of 127, with y in
// bf16 beside 4-bit products 4,096 tokens of 8 of 128 of 2048 x 768 take 252 instead
// of 305 (268 MB less), and each makes 1.4 times the error of the output's rounding.
Space few_space(int64_t P, int32_t D, int32_t I) {
  Space s{};
  s.y = up256(static_cast<size_t>(P) * I * 4);
  s.bytes = s.y + up256(static_cast<size_t>(P) * D * 4);
  return s;
}

Space tile_space(int64_t T, int64_t P, int32_t n, int32_t D, int32_t I, bool mx4) {
  Space s{};
  size_t at = 0;
  const auto take = [&](size_t bytes) {
    const size_t from = at;
    at += up256(bytes);
    return from;
  };
  s.h = take(mx4 ? static_cast<size_t>(P) * I / 2 : static_cast<size_t>(P) * I * 4);
  s.y = take(static_cast<size_t>(P) * D * 4);
  s.start = take((static_cast<size_t>(n) + 1) * 4);
  s.pair = take(static_cast<size_t>(P) * 4);
  s.place = take(static_cast<size_t>(P) * 4);
  s.sort = take(spp::expert_sort_bytes(P, n));
  if (mx4) {
    s.h_scales = take(static_cast<size_t>(P) * I / 32);
    s.xq = take(static_cast<size_t>(T) * D / 2);
    s.xq_scales = take(static_cast<size_t>(T) * D / 32);
  }
  s.bytes = at;
  return s;
}

const char* experts_why(int32_t n, int32_t D, int32_t I, int32_t T, int32_t K) {
  if (n < 1 || n > spp::kMaxExpertsTopK) return "n must be in [1, 1024]";
  if (K < 1 || K > 64) return "K must be in [1, 64]";
  if (T < 0 || static_cast<int64_t>(T) * K > kMaxM) return "T must be >= 0, and T * K at most 2^24";
  if (D < 32 || D % 32 != 0 || D > 1 << 17 || I < 32 || I % 32 != 0 || I > 1 << 17)
    return "D and I must be multiples of 32, at most 2^17";
  if (static_cast<int64_t>(T) * K * std::max(D, I) > kMaxOutputs) return "T * K times D or I must be at most 2^36";
  return nullptr;
}

}  // namespace

extern "C" spp_status spp_mx4_quantize(int32_t dtype, const void* x, int64_t x_stride, const spp_mx4_matrix* q,
                                       void* hip_stream) {
  SPP_BAD(dtype_why(dtype));
  SPP_BAD(matrix_why(q));
  if (q->rows == 0) return SPP_OK;
  const int elem = dtype == SPP_DTYPE_BF16 ? 2 : 4;
  SPP_BAD(rows_why(x, x_stride, q->cols, elem));
  if (over(*q, rows_from(x, x_stride, q->cols, q->rows, elem)) || meet(array(q->codes, code_bytes(*q)), array(q->scales, scale_bytes(*q))))
    return bad("x, codes and scales must not overlap");
  RowsQ a{};
  a.x = x;
  a.x_stride = x_stride;
  a.codes = static_cast<uint8_t*>(q->codes);
  a.scales = static_cast<uint8_t*>(q->scales);
  a.per_row = q->cols / 8;
  a.words = q->rows * a.per_row;
  const auto kernel = dtype == SPP_DTYPE_BF16 ? mx4_quantize_kernel<__bf16> : mx4_quantize_kernel<float>;
  return launched(launch(kernel, quant_grid(a.words), kQuantThreads, a, static_cast<hipStream_t>(hip_stream)));
}

extern "C" spp_status spp_mx4_load(const spp_mx4_matrix* q, int32_t dtype, void* out, int64_t out_stride,
                                   void* hip_stream) {
  SPP_BAD(dtype_why(dtype));
  SPP_BAD(matrix_why(q));
  if (q->rows == 0) return SPP_OK;
  const int elem = dtype == SPP_DTYPE_BF16 ? 2 : 4;
  SPP_BAD(rows_why(out, out_stride, q->cols, elem));
  if (over(*q, rows_from(out, out_stride, q->cols, q->rows, elem))) return bad("out must not overlap codes or scales");
  RowsQ a{};
  a.out = out;
  a.out_stride = out_stride;
  a.codes = static_cast<uint8_t*>(q->codes);
  a.scales = static_cast<uint8_t*>(q->scales);
  a.per_row = q->cols / 8;
  a.words = q->rows * a.per_row;
  const auto kernel = dtype == SPP_DTYPE_BF16 ? mx4_load_kernel<__bf16> : mx4_load_kernel<float>;
  return launched(launch(kernel, quant_grid(a.words), kQuantThreads, a, static_cast<hipStream_t>(hip_stream)));
}

extern "C" spp_status spp_mx4_matmul(const spp_mx4_matrix* w, int32_t groups, const int32_t* start, const void* x,
                                     int64_t x_stride, int32_t M, int32_t dtype, void* out, int64_t out_stride,
                                     void* hip_stream) {
  SPP_BAD(product_why(w, groups, start, M, dtype, out, out_stride));
  if (M == 0) return SPP_OK;
  SPP_BAD(rows_why(x, x_stride, w->cols, 2));
  if (meet(rows_from(out, out_stride, w->rows / groups, M, dtype == SPP_DTYPE_BF16 ? 2 : 4), rows_from(x, x_stride, w->cols, M, 2)))
    return bad("out must not overlap an input");
  ProductArgs a = product_of(*w, groups, start, M, out, out_stride);
  a.x = x;
  a.x_stride = x_stride * 2;
  return launched(launch_product<kXBf16>(a, dtype, static_cast<hipStream_t>(hip_stream)));
}

extern "C" spp_status spp_mx4_matmul_mx4(const spp_mx4_matrix* w, int32_t groups, const int32_t* start,
                                         const spp_mx4_matrix* x, int32_t M, int32_t dtype, void* out,
                                         int64_t out_stride, void* hip_stream) {
  SPP_BAD(product_why(w, groups, start, M, dtype, out, out_stride));
  SPP_BAD(matrix_why(x));
  if (x->rows != M || x->cols != w->cols) return bad("x must have M rows and the weights' cols");
  if (M == 0) return SPP_OK;
  if (over(*x, rows_from(out, out_stride, w->rows / groups, M, dtype == SPP_DTYPE_BF16 ? 2 : 4)))
    return bad("out must not overlap an input");
  ProductArgs a = product_of(*w, groups, start, M, out, out_stride);
  a.x = x->codes;
  a.x_stride = x->cols / 2;
  a.x_scales = static_cast<const uint8_t*>(x->scales);
  a.x_blocks = x->rows * (x->cols / 32);
  return launched(launch_product<kXCodes>(a, dtype, static_cast<hipStream_t>(hip_stream)));
}

extern "C" size_t spp_mx4_experts_workspace(int32_t n, int32_t D, int32_t I, int32_t T, int32_t K) {
  if (const char* w = experts_why(n, D, I, T, K)) return bad(w), 0;
  // every smaller call, with either act: the largest of few rows, and this one
  const int64_t P = static_cast<int64_t>(T) * K, few = std::min<int64_t>(P, most_few_pairs(n, D, I));
  size_t need = std::max(few_space(few, D, I).bytes, size_t{16});
  for (const bool mx4 : {false, true})
    if (by_tiles(P, n, D, I, mx4)) need = std::max(need, tile_space(T, P, n, D, I, mx4).bytes);
  return need;
}

extern "C" spp_status spp_mx4_experts(const spp_mx4_matrix* gate_up, const spp_mx4_matrix* down, int32_t n, int32_t act,
                                      const void* x, int64_t x_stride, const int32_t* topk, const float* gates,
                                      int32_t T, int32_t K, const void* residual, int64_t residual_stride, void* out,
                                      int64_t out_stride, void* workspace, size_t workspace_bytes, void* hip_stream) {
  SPP_BAD(matrix_why(gate_up));
  SPP_BAD(matrix_why(down));
  const int32_t D = gate_up->cols, I = down->cols;
  SPP_BAD(experts_why(n, D, I, T, K));
  if (gate_up->rows != int64_t{2} * n * I || down->rows != static_cast<int64_t>(n) * D)
    return bad("gate_up must have n * 2I rows of D columns, down n * D rows of I columns");
  if (act != SPP_ACT_BF16 && act != SPP_ACT_MX4) return bad("act must be 0 (bf16) or 1 (mx4)");
  if (T == 0) return SPP_OK;
  SPP_BAD(rows_why(x, x_stride, D, 2));
  SPP_BAD(rows_why(out, out_stride, D, 2));
  if (!topk || !gates || !aligned(topk, 4) || !aligned(gates, 4))
    return bad("topk and gates must not be NULL, and aligned to their elements");
  const int64_t P = static_cast<int64_t>(T) * K;
  const Rows to = rows_from(out, out_stride, D, T, 2);
  if (meet(to, rows_from(x, x_stride, D, T, 2)) || meet(to, array(topk, P * 4)) || meet(to, array(gates, P * 4)) ||
      over(*gate_up, to) || over(*down, to))
    return bad("out must not overlap an input");
  if (residual) {
    SPP_BAD(rows_why(residual, residual_stride, D, 2));
    if (!(residual == out && residual_stride == out_stride) && meet(to, rows_from(residual, residual_stride, D, T, 2)))
      return bad("out must be residual with the same stride, or not overlap it");
  }
  const bool mx4 = act == SPP_ACT_MX4;
  const bool tiles = by_tiles(P, n, D, I, mx4);
  const Space s = tiles ? tile_space(T, P, n, D, I, mx4) : few_space(P, D, I);
  if (!workspace || !aligned16(workspace)) return bad("workspace must not be NULL, and 16-byte aligned");
  if (workspace_bytes < s.bytes) return bad("the workspace is too small");
  const Rows used = array(workspace, static_cast<int64_t>(s.bytes));
  if (meet(used, to) || meet(used, rows_from(x, x_stride, D, T, 2)) || meet(used, rows_from(residual, residual_stride, D, T, 2)) ||
      meet(used, array(topk, P * 4)) || meet(used, array(gates, P * 4)) || over(*gate_up, used) || over(*down, used))
    return bad("the workspace must not overlap an input or the output");
  const hipStream_t st = static_cast<hipStream_t>(hip_stream);
  uint8_t* space = static_cast<uint8_t*>(workspace);

  spp::ExpertSum c{};
  c.rows = space + s.y;
  c.rows_stride = D;
  c.weights = gates;
  c.dtype = SPP_DTYPE_BF16;
  c.fp32_rows = 1;
  c.T = T;
  c.K = K;
  c.D = D;
  c.residual = residual;
  c.residual_stride = residual_stride;
  c.out = out;
  c.out_stride = out_stride;

  if (tiles) {
    int32_t* start = reinterpret_cast<int32_t*>(space + s.start);
    int32_t* pair = reinterpret_cast<int32_t*>(space + s.pair);
    int32_t* place = reinterpret_cast<int32_t*>(space + s.place);
    hipError_t e = spp::launch_expert_sort(topk, P, n, start, pair, place, space + s.sort, st);
    if (e != hipSuccess) return launched(e);
    if (mx4) {
      RowsQ q{};
      q.x = x;
      q.x_stride = x_stride;
      q.codes = space + s.xq;
      q.scales = space + s.xq_scales;
      q.per_row = D / 8;
      q.words = static_cast<int64_t>(T) * q.per_row;
      e = launch(mx4_quantize_kernel<__bf16>, quant_grid(q.words), kQuantThreads, q, st);
      if (e != hipSuccess) return launched(e);
    }
    ProductArgs a = product_of(*gate_up, n, start, static_cast<int32_t>(P), space + s.h, I);
    a.N = I;
    a.pair = pair;
    a.xdiv = K;
    a.x = mx4 ? static_cast<const void*>(space + s.xq) : x;
    a.x_stride = mx4 ? D / 2 : x_stride * 2;
    a.x_scales = space + s.xq_scales;
    a.x_blocks = static_cast<int64_t>(T) * a.nb;
    a.out_scales = space + s.h_scales;
    int rows = tile_rows(P, n, 2 * I, a.nb, mx4);
    e = mx4 ? launch_tiles<kXCodes, true, __bf16>(a, rows, st) : launch_tiles<kXBf16, true, Terms>(a, rows, st);
    if (e != hipSuccess) return launched(e);
    ProductArgs d = product_of(*down, n, start, static_cast<int32_t>(P), space + s.y, D);
    d.x = space + s.h;
    d.x_stride = mx4 ? I / 2 : static_cast<int64_t>(I) * 4;
    d.x_scales = space + s.h_scales;
    d.x_blocks = P * d.nb;
    rows = tile_rows(P, n, D, d.nb, mx4);
    e = mx4 ? launch_tiles<kXCodes, false, float>(d, rows, st) : launch_tile<kXTermRows, false, float, 2>(d, st);
    if (e != hipSuccess) return launched(e);
    c.place = place;
    return launched(spp::launch_expert_combine(c, st));
  }

  ProductArgs a = product_of(*gate_up, n, nullptr, static_cast<int32_t>(P), space + s.h, I);
  a.N = I;
  a.x = x;
  a.x_stride = x_stride * 2;
  a.ids = topk;
  a.xdiv = K;
  a.by_pair = P < n;
  const int64_t groups = std::min<int64_t>(P, n);
  hipError_t e = mx4 ? launch_few<kXQuantBf16, true, float, kRowsIds>(a, groups, st)
                     : launch_few<kXBf16, true, Terms, kRowsIds>(a, groups, st);
  if (e != hipSuccess) return launched(e);
  ProductArgs d = product_of(*down, n, nullptr, static_cast<int32_t>(P), space + s.y, D);
  d.x = space + s.h;
  d.x_stride = static_cast<int64_t>(I) * 4;
  d.ids = topk;
  d.by_pair = P < n;
  if (T <= kLastTokens) {
    LastArgs l{};
    l.p = d;
    l.p.out = out;
    l.p.out_stride = out_stride;
    l.gates = gates;
    l.residual = residual;
    l.residual_stride = residual_stride;
    l.K = K;
    void* params[] = {&l};
    const auto last = d.nb < 3 ? (mx4 ? mx4_last_kernel<kXQuantF32, 1, true> : mx4_last_kernel<kXTermRows, 1, true>)
                               : (mx4 ? mx4_last_kernel<kXQuantF32, 3, false> : mx4_last_kernel<kXTermRows, 3, false>);
    const void* kernel = reinterpret_cast<const void*>(last);
    return launched(hipLaunchKernel(kernel, dim3(static_cast<unsigned>((D + 15) / 16), static_cast<unsigned>(T)),
                                    dim3(kLastThreads), params, 0, st));
  }
  e = mx4 ? launch_few<kXQuantF32, false, float, kRowsIds>(d, groups, st)
          : launch_few<kXTerms, false, float, kRowsIds>(d, groups, st);
  if (e != hipSuccess) return launched(e);
  c.ids = topk;
  c.n = n;
  return launched(spp::launch_expert_combine(c, st));
}
