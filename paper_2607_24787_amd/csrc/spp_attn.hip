// Attention over a 4-bit key/value cache: rotary tables, the store that
// rotates and quantises, the load that reads back, and the attention itself.
// The cache's format and the calls' contracts are in spp.h.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <type_traits>
#include <utility>

#include "spp.h"
#include "spp_internal.h"

namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kMaxFreq = 64;
constexpr uint32_t kExpMask = 0x7f800000u;
constexpr int kNanByte = 255;
constexpr int kMinByte = 2;    // scale 2^-125: every nonzero value of a block stays a normal number
constexpr int kMaxByte = 252;  // scale 2^125: 6 * 2^125 is the largest that is finite in bf16 and fp32

// ------------------------------------------------------------------ the cache

struct Cache {
  const uint8_t* base;
  uint32_t page_bytes;  // all heads of a page
  uint32_t head_bytes;  // one head of a page
  int page, shift;      // tokens per page and its logarithm
  int n_pages;
};

// Offsets within a (page, head) block of head size D.
template <int D>
struct Block {
  static __device__ __forceinline__ uint32_t codes(int page, int kv, int off) {
    return static_cast<uint32_t>((kv * page + off) * (D / 2));
  }
  static __device__ __forceinline__ uint32_t scales(int page, int kv, int block, int off) {
    return static_cast<uint32_t>(page * D + (kv * (D / 32) + block) * page + off);
  }
};

__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }

// Byte j of 8 as a scale for cvt2, for which only the exponent field counts
__device__ __forceinline__ float scale_byte(u32x2 w, int j) {
  return __uint_as_float(j % 4 == 3 ? w[j / 4] >> 1 : w[j / 4] << (23 - 8 * (j % 4)));
}

// Whether a byte of w is kMaxByte or more (its upper six bits are ones)
__device__ __forceinline__ bool high_byte(uint32_t w) {
  const uint32_t u = ~w & 0xfcfcfcfcu;
  return ((u - 0x01010101u) & ~u & 0x80808080u) != 0;
}

// Two codes of byte SEL of w to bf16, times the power of two in `scale`'s
// exponent field (its other bits do not count; exponent 255 gives NaN).
template <int SEL>
__device__ __forceinline__ uint32_t cvt2(uint32_t w, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, SEL));
}

// 8 codes to 8 bf16, in order
__device__ __forceinline__ u32x4 cvt8(uint32_t w, float scale) {
  return u32x4{cvt2<0>(w, scale), cvt2<1>(w, scale), cvt2<2>(w, scale), cvt2<3>(w, scale)};
}

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  return __builtin_bit_cast(uint32_t, bf16x2{static_cast<__bf16>(a), static_cast<__bf16>(b)});
}

// 8 consecutive elements of a row (16-byte aligned)
template <typename T>
__device__ __forceinline__ void load8(const T* p, float* f) {
  if constexpr (std::is_same<T, float>::value) {
    const f32x4 a = reinterpret_cast<const f32x4*>(p)[0], b = reinterpret_cast<const f32x4*>(p)[1];
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = a[i], f[4 + i] = b[i];
  } else {
    const u32x4 a = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) f[2 * i] = bf16_lo(a[i]), f[2 * i + 1] = bf16_hi(a[i]);
  }
}

// The same 8 elements past the caches (streams that nothing here reads again)
template <typename T>
__device__ __forceinline__ void stream8(T* p, const float* f) {
  if constexpr (std::is_same<T, float>::value) {
    __builtin_nontemporal_store(f32x4{f[0], f[1], f[2], f[3]}, reinterpret_cast<f32x4*>(p));
    __builtin_nontemporal_store(f32x4{f[4], f[5], f[6], f[7]}, reinterpret_cast<f32x4*>(p) + 1);
  } else {
    __builtin_nontemporal_store(
        u32x4{pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7])},
        reinterpret_cast<u32x4*>(p));
  }
}

template <typename T>
__device__ __forceinline__ void store8(T* p, const float* f) {
  if constexpr (std::is_same<T, float>::value) {
    reinterpret_cast<f32x4*>(p)[0] = f32x4{f[0], f[1], f[2], f[3]};
    reinterpret_cast<f32x4*>(p)[1] = f32x4{f[4], f[5], f[6], f[7]};
  } else {
    *reinterpret_cast<u32x4*>(p) =
        u32x4{pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7])};
  }
}

// --------------------------------------------------------------- rotary table

struct TableArgs {
  const int32_t* pos;
  int64_t pos_stride;
  const float* inv_freq;
  float* table;
  uint32_t axes[kMaxFreq / 16];  // two bits per frequency
  int F, T;
};

constexpr int kTableFreqs = 4;  // per thread: 16-byte stores

// The angle in turns, reduced to [-1/2, 1/2] in 64 bits: its product with 1 / (2
// pi) is not rounded before the whole turns are off it (rounded, it would cost
// 3e-7 of a value at the largest positions, five steps of fp32).  What is left
// beyond fp32 goes in by the first term of the addition theorem (error 2.6e-8 of
// the values, half a step of fp32 2e-8 on average).  16,001 tokens of 64
// frequencies 5.2 us (8.2 MB written), 64 tokens 2.5 us: a launch and one round of
// waves, which are all resident at once; a wave of the 16,001 tokens' lives 2.5
// us, half of it waiting for its positions and frequencies.
__global__ __launch_bounds__(256) void rotary_table_kernel(TableArgs a) {
  const uint32_t per = static_cast<uint32_t>(a.F / kTableFreqs);
  const uint32_t i = blockIdx.x * 256u + threadIdx.x;
  const uint32_t t = i / per;
  if (t >= static_cast<uint32_t>(a.T)) return;
  const int f0 = static_cast<int>(i - t * per) * kTableFreqs;
  f32x4 c, s;
#pragma unroll
  for (int k = 0; k < kTableFreqs; ++k) {
    const int f = f0 + k;
    const int axis = static_cast<int>(a.axes[f / 16] >> (2 * (f % 16))) & 3;
    const double angle = static_cast<double>(a.pos[axis * a.pos_stride + t]) * static_cast<double>(a.inv_freq[f]);
    constexpr double kPerTurn = 0.15915494309189533577, kRest = -9.839338337591243e-18;  // 1 / (2 pi) in two terms
    const double whole = rint(angle * kPerTurn);
    const double turns = fma(angle, kRest, fma(angle, kPerTurn, -whole));
    const double half = 2.0 * turns;  // in units of pi
    const float hi = static_cast<float>(half);
    const float lo = static_cast<float>((half - static_cast<double>(hi)) * 3.14159265358979323846);
    const float ch = cospif(hi), sh = sinpif(hi);
    c[k] = fmaf(-lo, sh, ch);
    s[k] = fmaf(lo, ch, sh);
  }
  float* row = a.table + static_cast<size_t>(t) * 2 * a.F + f0;
  *reinterpret_cast<f32x4*>(row) = c;
  *reinterpret_cast<f32x4*>(row + a.F) = s;
}

// ----------------------------------------------------------------- store, load

struct StoreArgs {
  Cache cache;
  const void *q, *k, *v;
  void* q_out;
  int64_t q_stride, q_out_stride, k_stride, v_stride;
  const float* table;
  const int64_t* slots;
  int Hq, Hkv, F;  // Hq = 0: no queries
  int T;
};

// Codes (one word) and scale byte of this lane's 8 elements of a block of 32,
// which lanes 4j .. 4j+3 hold together.
__device__ __forceinline__ uint32_t quantise8(const float* y, uint32_t* byte) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(y[i]) & 0x7fffffffu);  // ordered as the magnitudes are; NaN above infinity
  top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), 1)));
  top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), 2)));
  if (top >= kExpMask) {
    *byte = kNanByte;
    return 0u;
  }
  // top = 1.m * 2^(E-127) <= 7 * 2^e = 1.75 * 2^(e+2)
  const int E = static_cast<int>(top >> 23);
  int s = (top & 0x7fffffu) <= 0x600000u ? E - 2 : E - 1;
  s = min(max(s, kMinByte), kMaxByte);
  const float scale = scale_of(static_cast<uint32_t>(s));
  *byte = static_cast<uint32_t>(s);
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[0], y[1], scale, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[2], y[3], scale, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[4], y[5], scale, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[6], y[7], scale, 3);
  return w;
}

// Each product and the sum rounded, not contracted: what is quantised next is
// then the same number wherever it is formed.
__device__ __forceinline__ float turn(float y, float z, float c, float s, bool first) {
#pragma clang fp contract(off)
  const float p = y * c, r = z * s;
  return first ? p - r : p + r;
}

// D/8 lanes per head, 8 elements each; a thread reads its elements and those
// they turn with before it writes, and a head lies within one wave, so the
// queries may be rotated in place.  The partner's elements are read a second
// time (from L1) instead of exchanged.  Bound by memory: 8,192 tokens of 32 + 4
// + 4 heads of 128, 160 MB (170 by the counters), in 36.4 us (4.7 TB/s; a large
// copy 5.0); one token 2.5 us.  Queries written past the caches would take 4 us
// off that, but what reads them next then waits for memory: 8,192 tokens with a
// reader behind them 57.6 us so, 59.9 past the caches; 16,384 tokens 113, 111.
template <typename T, int D>
__global__ __launch_bounds__(256) void kv4_store_kernel(StoreArgs a) {
  constexpr int L = D / 8;
  const uint32_t heads = static_cast<uint32_t>(a.Hq + 2 * a.Hkv);
  const uint32_t unit = blockIdx.x * (256u / L) + threadIdx.x / L;
  const uint32_t t = unit / heads;
  if (t >= static_cast<uint32_t>(a.T)) return;
  int h = static_cast<int>(unit - t * heads);
  const int e0 = static_cast<int>(threadIdx.x % L) * 8;
  const int kind = h < a.Hq ? 0 : (h < a.Hq + a.Hkv ? 1 : 2);
  h -= kind == 0 ? 0 : (kind == 1 ? a.Hq : a.Hq + a.Hkv);
  const T* row = kind == 0   ? reinterpret_cast<const T*>(a.q) + static_cast<int64_t>(t) * a.q_stride
                 : kind == 1 ? reinterpret_cast<const T*>(a.k) + static_cast<int64_t>(t) * a.k_stride
                             : reinterpret_cast<const T*>(a.v) + static_cast<int64_t>(t) * a.v_stride;
  row += h * D;
  const int64_t slot = a.slots[t];
  float y[8];
  load8(row + e0, y);
  if (kind < 2 && e0 < 2 * a.F) {
    float z[8], c[8], s[8];
    const bool first = e0 < a.F;
    const int f0 = first ? e0 : e0 - a.F;
    load8(row + (first ? e0 + a.F : f0), z);
    const float* tab = a.table + static_cast<size_t>(t) * 2 * a.F + f0;
    load8(tab, c);
    load8(tab + a.F, s);
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = turn(y[i], z[i], c[i], s[i], first);
  }
  if (kind == 0) {
    T* to = reinterpret_cast<T*>(a.q_out) + static_cast<int64_t>(t) * a.q_out_stride + h * D + e0;
    store8(to, y);
    return;
  }
  uint32_t byte;
  const uint32_t w = quantise8(y, &byte);
  if (static_cast<uint64_t>(slot) >= static_cast<uint64_t>(a.cache.n_pages) << a.cache.shift) return;
  const int off = static_cast<int>(slot) & (a.cache.page - 1);
  uint8_t* blk = const_cast<uint8_t*>(a.cache.base) + static_cast<uint64_t>(slot >> a.cache.shift) * static_cast<uint64_t>(a.cache.page_bytes) +
                 static_cast<uint64_t>(h) * a.cache.head_bytes;
  *reinterpret_cast<uint32_t*>(blk + Block<D>::codes(a.cache.page, kind - 1, off) + e0 / 2) = w;
  if (e0 % 32 == 0) blk[Block<D>::scales(a.cache.page, kind - 1, e0 / 32, off)] = static_cast<uint8_t>(byte);
}

struct LoadArgs {
  Cache cache;
  const int64_t* slots;
  void *k, *v;  // either may be NULL
  int64_t k_stride, v_stride;
  int Hkv, T;
};

// Bound by memory, most of it the rows written: 100,000 tokens of 4 heads of 128
// in bf16, 260 MB, in 45 us (5.8 TB/s) with stores past the caches, 77 us with
// ordinary ones, 66 us with reads past them too; 700 tokens in fp32 3.1 us.  With
// a reader of the rows behind it: 16,000 tokens 19.4 us past the caches, 18.8
// with ordinary stores, 100,000 tokens 124 and 125, 64,000 in fp32 134 and 151.
template <typename T, int D>
__global__ __launch_bounds__(256) void kv4_load_kernel(LoadArgs a) {
  constexpr int L = D / 8;
  const uint32_t both = a.k && a.v ? 2u : 1u;
  const uint32_t heads = static_cast<uint32_t>(a.Hkv) * both;
  const uint32_t unit = blockIdx.x * (256u / L) + threadIdx.x / L;
  const uint32_t t = unit / heads;
  if (t >= static_cast<uint32_t>(a.T)) return;
  int h = static_cast<int>(unit - t * heads);
  const int kv = both == 2u ? (h >= a.Hkv ? 1 : 0) : (a.k ? 0 : 1);
  if (both == 2u) h -= kv * a.Hkv;
  const int e0 = static_cast<int>(threadIdx.x % L) * 8;
  const int64_t slot = a.slots[t];
  if (static_cast<uint64_t>(slot) >= static_cast<uint64_t>(a.cache.n_pages) << a.cache.shift) return;
  const int off = static_cast<int>(slot) & (a.cache.page - 1);
  const uint8_t* blk = a.cache.base + static_cast<uint64_t>(slot >> a.cache.shift) * static_cast<uint64_t>(a.cache.page_bytes) +
                       static_cast<uint64_t>(h) * a.cache.head_bytes;
  const uint32_t w = *reinterpret_cast<const uint32_t*>(blk + Block<D>::codes(a.cache.page, kv, off) + e0 / 2);
  const uint32_t byte = blk[Block<D>::scales(a.cache.page, kv, e0 / 32, off)];
  const u32x4 b = cvt8(w, scale_of(byte));
  T* out = kv ? reinterpret_cast<T*>(a.v) + static_cast<int64_t>(t) * a.v_stride
              : reinterpret_cast<T*>(a.k) + static_cast<int64_t>(t) * a.k_stride;
  out += h * D + e0;
  float f[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) f[2 * i] = bf16_lo(b[i]), f[2 * i + 1] = bf16_hi(b[i]);
  stream8(out, f);
}

// ------------------------------------------------------------------- attention

struct AttendArgs {
  Cache cache;
  const void* q;
  void* out;
  int64_t q_stride, out_stride;
  const int32_t *q_start, *kv_len, *pages;
  int64_t pages_stride;
  int n_seq, n_tokens, Hkv, G;  // G: query heads per key/value head
  int max_rows;  // of a sequence's key/value head: max_q query tokens times G
  int causal;
  int planes, row_tiles;  // a plane: one key/value head and row tile (Hkv * row_tiles of them)
  int units;              // about the parts that a plane's cached tokens are cut into; 0: a part is a whole sequence
  int min_tiles;          // tiles of the smallest part
  int sum_shift;          // see place_of
  int join_apart;         // parts are joined by a launch of their own
  unsigned* count;        // [planes][n_seq] finished parts; zero between calls
  float* part;            // [planes][units + n_seq] partial rows
  float scale_log2;  // scale * log2(e): the softmax runs on powers of two
};

constexpr int kWaves = 4;
constexpr int kTile = 32;  // cached tokens per step: one 16x16x32 product over them

// The rows of a sequence's key/value head are its query tokens times the G
// heads that share it, token-major: row r is token r / G, head r % G.
struct Seq {
  int q0, nq;  // first query token, count
  int len;     // cached tokens that the page table row has a place for
  int first;   // tokens that query 0 sees, by the whole length (causal; below 0: the next ones see none either)
  bool overlong;  // there are more than the row has a place for
  __device__ __forceinline__ int limit(const AttendArgs& a, int row) const {
    return a.causal ? min(max(0, first + row / a.G), len) : len;
  }
};

// A sequence's numbers as they stand in memory
struct RawSeq {
  int len = 0, first = 0, end = 0;
};

__device__ __forceinline__ RawSeq raw_sequence(const AttendArgs& a, int b) {
  RawSeq r;
  if (b >= a.n_seq) return r;
  r.len = a.kv_len[b];
  r.first = a.q_start ? a.q_start[b] : b;
  r.end = a.q_start ? a.q_start[b + 1] : b + 1;
  return r;
}

__device__ __forceinline__ Seq sequence(const AttendArgs& a, RawSeq r) {
  Seq s;
  s.q0 = min(max(r.first, 0), a.n_tokens);
  s.nq = min(max(r.end, s.q0), a.n_tokens) - s.q0;
  const int whole = max(r.len, 0);
  s.len = static_cast<int>(min(static_cast<int64_t>(whole), a.pages_stride * a.cache.page));
  s.first = whole - s.nq + 1;
  s.overlong = whole > s.len;
  return s;
}

__device__ __forceinline__ uint32_t tiles_of(const AttendArgs& a, RawSeq r) {
  const int64_t len = min(static_cast<int64_t>(max(r.len, 0)), a.pages_stride * a.cache.page);
  return static_cast<uint32_t>((len + kTile - 1) / kTile);
}

// Inclusive sums over the wave's lanes (all of them active)
__device__ __forceinline__ int wave_scan(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);  // from 1, 2, 4, 8 lanes below within 16
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);  // lane 15 to the second 16, lane 47 to the last
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);  // lane 31 to the upper half
  return x;
}

// Part p of a plane: tiles [first, first + each) of sequence b, which is its
// part p - base.
struct Place {
  int b, base, each;
  Seq seq;
};

// A plane's parts are equal pieces of all its sequences' tiles, at most
// units + n_seq of them (one at least for each sequence), so that a batch of
// very different lengths keeps every workgroup about as long.  Every wave
// finds its part by itself, from the lengths on the device: a scan over 64
// sequences at a time.  b >= 0: the place of that sequence's first part instead.
__device__ __forceinline__ Place place_of(const AttendArgs& a, int p, int b, int lane) {
  const RawSeq mine = raw_sequence(a, lane);
  const uint32_t up = (1u << a.sum_shift) - 1u;  // sums in units of 2^sum_shift tiles fit 31 bits
  uint32_t total = (tiles_of(a, mine) + up) >> a.sum_shift;
  for (int i = 64 + lane; i - lane < a.n_seq; i += 64) total += (tiles_of(a, raw_sequence(a, i)) + up) >> a.sum_shift;
  total = __builtin_amdgcn_readlane(wave_scan(static_cast<int>(total)), 63);
  uint32_t each = min((total + static_cast<uint32_t>(a.units) - 1) / static_cast<uint32_t>(a.units), 1u << (30 - a.sum_shift));
  each = max(each << a.sum_shift, static_cast<uint32_t>(a.min_tiles));
  each = (each + kWaves - 1) / kWaves * kWaves;  // whole steps of a workgroup
  Place at;
  at.b = -1;
  at.base = 0;
  at.each = static_cast<int>(each);
  for (int i0 = 0; i0 < a.n_seq; i0 += 64) {
    const RawSeq r = i0 == 0 ? mine : raw_sequence(a, i0 + lane);
    const int n = i0 + lane < a.n_seq ? max(1, static_cast<int>((tiles_of(a, r) + each - 1) / each)) : 0;
    const int sum = wave_scan(n);
    const uint64_t past = __ballot(b < 0 ? at.base + sum > p : i0 + lane == b);
    if (past) {
      const int l = __builtin_ctzll(past);
      at.b = i0 + l;
      at.base += __builtin_amdgcn_readlane(sum - n, l);
      RawSeq found;
      found.len = __builtin_amdgcn_readlane(r.len, l);
      found.first = __builtin_amdgcn_readlane(r.first, l);
      found.end = __builtin_amdgcn_readlane(r.end, l);
      at.seq = sequence(a, found);
      return at;
    }
    at.base += __builtin_amdgcn_readlane(sum, 63);
  }
  return at;
}

// What a workgroup works on: rows row0 .. last of a sequence's key/value head,
// and of its tiles [begin, end), one of `parts` parts.
struct Spot {
  Seq seq;
  int b, h, rt, split, parts, row0, last, begin, end;
  size_t part;  // index of its partial rows
};

// False: nothing to do (the whole workgroup alike).  rows: rows per workgroup.
__device__ __forceinline__ bool find_spot(const AttendArgs& a, int rows, int lane, Spot& s) {
  int p = 0, each = 1 << 30;
  s.split = 0;
  if (a.units > 0) {
    const int plane = static_cast<int>(blockIdx.x) % a.planes;
    p = static_cast<int>(blockIdx.x) / a.planes;
    s.h = plane % a.Hkv, s.rt = plane / a.Hkv;
    const Place at = place_of(a, p, -1, lane);
    if (at.b < 0) return false;
    s.b = at.b, s.split = p - at.base, each = at.each;
    s.seq = at.seq;
  } else {
    // the row tiles of one sequence and head are a multiple of 8 workgroups
    // apart, which brings them to one XCD and the cached rows into its L2; the
    // rows that see most go first
    const int heads = a.n_seq * a.Hkv, step = a.row_tiles > 1 ? (heads + 7) / 8 * 8 : heads;
    const int bh = static_cast<int>(blockIdx.x) % step;
    if (bh >= heads) return false;
    s.rt = a.row_tiles - 1 - static_cast<int>(blockIdx.x) / step;
    s.b = bh / a.Hkv, s.h = bh - s.b * a.Hkv;
    s.seq = sequence(a, raw_sequence(a, s.b));
  }
  const int nrows = min(s.seq.nq * a.G, a.max_rows);
  s.row0 = s.rt * rows;
  if (s.row0 >= nrows) return false;
  s.last = min(s.row0 + rows, nrows) - 1;
  const int tiles = (s.seq.limit(a, s.last) + kTile - 1) / kTile;
  s.parts = max(1, static_cast<int>((static_cast<uint32_t>(tiles) + each - 1) / static_cast<uint32_t>(each)));
  if (s.split >= s.parts) return false;
  s.begin = s.split * each, s.end = min(tiles, s.begin + each);
  s.part = static_cast<size_t>(s.rt * a.Hkv + s.h) * (a.units + a.n_seq) + p;
  return true;
}

// Two floats (8-byte aligned) written and read at agent scope
__device__ __forceinline__ void put2(float* p, float x, float y) {
  const uint64_t v = static_cast<uint64_t>(__float_as_uint(y)) << 32 | __float_as_uint(x);
  __hip_atomic_store(reinterpret_cast<uint64_t*>(p), v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float2 get2(const float* p) {
  const uint64_t v = __hip_atomic_load(reinterpret_cast<const uint64_t*>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return make_float2(__uint_as_float(static_cast<uint32_t>(v)), __uint_as_float(static_cast<uint32_t>(v >> 32)));
}

__device__ __forceinline__ f32x4 mfma(u32x4 a, u32x4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// fp32 as NS bf16 terms: three add up to it (24 significant bits), two hold 16
// bits of it, one is the value rounded to it.
template <int NS>
__device__ __forceinline__ void split8(const float* f, u32x4* out) {
  float r[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) r[i] = f[i];
#pragma unroll
  for (int s = 0; s < NS; ++s) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t w = pack_bf16(r[2 * i], r[2 * i + 1]);
      out[s][i] = w;
      if (s + 1 < NS) {
        r[2 * i] -= bf16_lo(w);
        r[2 * i + 1] -= bf16_hi(w);
      }
    }
  }
}

// One step's share of a lane (c = lane % 16, g = lane / 16).  Keys: tokens
// kt = 8 (c/4) + c%4 and kt + 4 of the tile, elements g*D/4 .. of each (so the
// four lanes of a token read its whole row in one piece, and a lane needs one
// scale).  Values: tokens 8g .. 8g+7, elements c*D/16 .. of each.
template <int D>
struct Tile {
  static constexpr int KW = D / 32;  // words of a lane's key codes
  uint32_t k[2][KW];
  uint32_t ks[2];
  uint32_t v[8];  // D = 64: 16 bits each
  u32x2 vs;       // scale bytes of the 8 tokens
};

// Page ids of a lane's key tokens and value tokens (they differ where a tile
// spans two pages); -1: none
struct Pids {
  int k, v;
};

__device__ __forceinline__ Pids page_ids(const AttendArgs& a, const int32_t* pages, int t0, int k, int v) {
  const int ik = (t0 + k) >> a.cache.shift, iv = (t0 + v) >> a.cache.shift, room = static_cast<int>(a.pages_stride);
  Pids p;
  p.k = ik < room ? pages[ik] : -1;
  p.v = iv < room ? pages[iv] : -1;
  return p;
}

// A tile starts at a multiple of 32 tokens, so that a lane's place in a page is
// the tile's, alike for all lanes, plus its own: where a lane reads is one
// address for its own part, formed once, and a page and a tile added to it.
__device__ __forceinline__ const uint8_t* in_page(const Cache& c, const uint8_t* own, int pid, uint32_t tile_bytes) {
  return own + static_cast<uint64_t>(static_cast<uint32_t>(pid)) * c.page_bytes + tile_bytes;
}

__device__ __forceinline__ bool no_page(const Cache& c, int pid) {
  return static_cast<uint32_t>(pid) >= static_cast<uint32_t>(c.n_pages);
}

// A lane's key tokens 8 (c/4) + c%4 (and 4 on), its value tokens from 8g
__device__ __forceinline__ int key_token(int c) { return (c >> 2) * 8 + (c & 3); }

template <int D>
struct TileLane {
  const uint8_t *k, *ks, *v, *vs;

  __device__ __forceinline__ TileLane(const Cache& cache, const uint8_t* head, int c, int g) {
    const int page = cache.page, kt = key_token(c) & (page - 1), vt = (8 * g) & (page - 1);
    k = head + Block<D>::codes(page, 0, kt) + g * (D / 8);
    ks = head + Block<D>::scales(page, 0, g * (D / 4) / 32, kt);
    v = head + Block<D>::codes(page, 1, vt) + c * (D / 32);
    vs = head + Block<D>::scales(page, 1, c * (D / 16) / 32, vt);
  }
};

template <int D>
__device__ __forceinline__ void load_tile(const Cache& cache, const TileLane<D>& own, Pids pid, int t0, Tile<D>& t) {
  // a page that is none: its keys are NaN, which makes NaN of every row that
  // sees them; page 0 stands in for the loads
  const bool kbad = no_page(cache, pid.k);
  const int kp = kbad ? 0 : pid.k, vp = no_page(cache, pid.v) ? 0 : pid.v;
  const uint32_t u = static_cast<uint32_t>(t0 & (cache.page - 1));
  const uint8_t *k = in_page(cache, own.k, kp, u * (D / 2)), *ks = in_page(cache, own.ks, kp, u);
  const uint8_t *v = in_page(cache, own.v, vp, u * (D / 2)), *vs = in_page(cache, own.vs, vp, u);
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    if constexpr (D == 128) {
      const u32x4 w = *reinterpret_cast<const u32x4*>(k + 4 * i * (D / 2));
#pragma unroll
      for (int j = 0; j < 4; ++j) t.k[i][j] = w[j];
    } else {
      const u32x2 w = *reinterpret_cast<const u32x2*>(k + 4 * i * (D / 2));
      t.k[i][0] = w[0], t.k[i][1] = w[1];
    }
    const uint32_t byte = ks[4 * i];
    t.ks[i] = kbad ? static_cast<uint32_t>(kNanByte) : byte;
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    if constexpr (D == 128)
      t.v[j] = *reinterpret_cast<const uint32_t*>(v + j * (D / 2));
    else
      t.v[j] = *reinterpret_cast<const uint16_t*>(v + j * (D / 2));
  }
  t.vs = *reinterpret_cast<const u32x2*>(vs);
}

// O += V^T P^T over a tile: product n takes element c * D/16 + n of every
// lane, so a lane's codes become operands by pairing tokens (one permutation
// per pair).  frag(n, A operand) is called for n = 0 .. D/16 - 1.
template <int D, int B = 0, typename Fn>
__device__ __forceinline__ void value_frags(const uint32_t* w, const float* sc, Fn frag) {
  uint32_t x[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) x[j] = cvt2<B>(w[j], sc[j]);
  u32x4 lo, hi;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    lo[j] = __builtin_amdgcn_perm(x[2 * j + 1], x[2 * j], 0x05040100u);
    hi[j] = __builtin_amdgcn_perm(x[2 * j + 1], x[2 * j], 0x07060302u);
  }
  frag(2 * B, lo);
  frag(2 * B + 1, hi);
  __builtin_amdgcn_sched_barrier(0);  // the next elements are not converted ahead: registers
  if constexpr (B + 1 < D / 32) value_frags<D, B + 1>(w, sc, frag);
}

// The B operand of K Q^T for one row: step j covers elements g*D/4 + 8j ..
template <typename T, int D, int NS>
__device__ __forceinline__ void load_query(const AttendArgs& a, const Seq& seq, int h, int row, int g,
                                           u32x4 (&qf)[NS][D / 32]) {
  const int tok = row / a.G, hq = h * a.G + row - tok * a.G;
  const T* qp = reinterpret_cast<const T*>(a.q) + static_cast<int64_t>(seq.q0 + tok) * a.q_stride + hq * D + g * (D / 4);
#pragma unroll
  for (int j = 0; j < D / 32; ++j) {
    if constexpr (NS == 1) {
      qf[0][j] = *reinterpret_cast<const u32x4*>(qp + 8 * j);
    } else {
      float f[8];
      load8(qp + 8 * j, f);
      u32x4 terms[NS];
      split8<NS>(f, terms);
#pragma unroll
      for (int s = 0; s < NS; ++s) qf[s][j] = terms[s];
    }
  }
}

// The running maximum m over a tile's scores (masked ones -inf) too; l and o
// follow where it moves.
template <int D, int R, typename Sum>
__device__ __forceinline__ void follow_maximum(const f32x4 (&s)[R][2], float scale_log2, float (&m)[R], Sum (&l)[R],
                                               f32x4 (&o)[R][D / 16]) {
  float top[R];
  bool moves = false;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    top[r] = s[r][0][0];
#pragma unroll
    for (int k = 1; k < 8; ++k) top[r] = fmaxf(top[r], s[r][k / 4][k % 4]);
    top[r] *= scale_log2;
    moves |= top[r] > m[r] + 8.f;
  }
  // The running maximum moves only when a score passes it by 2^8: the
  // probabilities stay below 2^8, far from fp32's range, and most steps
  // neither reduce across lanes nor rescale.
  if (__any(moves)) {
#pragma unroll
    for (int r = 0; r < R; ++r) {
      top[r] = fmaxf(top[r], __shfl_xor(top[r], 16));
      top[r] = fmaxf(top[r], __shfl_xor(top[r], 32));
      const float now = top[r] > m[r] + 8.f ? top[r] : m[r];  // a row's bits do not depend on the rows beside it
      const float alpha = m[r] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m[r] - now);
      m[r] = now;
      l[r] *= alpha;
#pragma unroll
      for (int n = 0; n < D / 16; ++n) o[r][n] *= alpha;
    }
  }
}

// A tile's scores to the probabilities of the value product, relative to the
// maximum.  One term (f32x4 sums): l sums the row's as rounded, so that what the
// rounding does to all of them alike is divided out.  More: l sums this lane's
// eight as they are.
template <int R, int NP, typename Sum>
__device__ __forceinline__ void probabilities(const f32x4 (&s)[R][2], float scale_log2, const float (&m)[R],
                                              Sum (&l)[R], u32x4 (&pf)[R][NP]) {
  const u32x4 ones = u32x4{0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u};
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const float ref = m[r] == -INFINITY ? 0.f : m[r];  // nothing seen yet: every power is 0
    float p[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) p[k] = __builtin_amdgcn_exp2f(fmaf(s[r][k / 4][k % 4], scale_log2, -ref));
    if constexpr (NP > 1) l[r] += ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
    split8<NP>(p, pf[r]);
    if constexpr (NP == 1) l[r] = mfma(ones, pf[r][0], l[r]);
  }
}

template <typename T>
__device__ __forceinline__ T* out_row(const AttendArgs& a, const Seq& seq, int h, int row, int d) {
  const int tok = row / a.G, hq = h * a.G + row - tok * a.G;
  return reinterpret_cast<T*>(a.out) + static_cast<int64_t>(seq.q0 + tok) * a.out_stride + hq * d;
}

template <typename T, int N>
__device__ __forceinline__ void store_n(T* p, const float* y);

// N elements of a finished row: its sums over the sum of its probabilities
template <typename T, int N>
__device__ __forceinline__ void finish(const AttendArgs& a, const Seq& seq, int h, int row, int d, int e0, float sum,
                                       const float* y) {
  const bool empty = seq.limit(a, row) <= 0;
  const float inv = 1.f / sum;
  float v[N];
#pragma unroll
  for (int k = 0; k < N; ++k) v[k] = empty ? 0.f : (seq.overlong ? NAN : y[k] * inv);
  store_n<T, N>(out_row<T>(a, seq, h, row, d) + e0, v);
}

template <typename T, int N>
__device__ __forceinline__ void store_n(T* p, const float* y) {
  if constexpr (N == 8) {
    store8(p, y);
  } else if constexpr (N == 1 || std::is_same<T, float>::value) {
#pragma unroll
    for (int i = 0; i < N; ++i) p[i] = static_cast<T>(y[i]);
  } else {
#pragma unroll
    for (int i = 0; i < N; i += 2) reinterpret_cast<uint32_t*>(p)[i / 2] = pack_bf16(y[i], y[i + 1]);
  }
}

// Workgroups per compute unit (waves per SIMD) that the registers of a variant
// leave without spilling.
constexpr int resident(bool f32, int d, int R) {
  const int w = R == 1 ? 4 : 2;
  return f32 && d == 128 && w > 1 ? w / 2 : w;
}

// N elements of a row joined from parts, in their order: each part a maximum,
// a sum of probabilities and N sums relative to that maximum.
template <int N>
struct Joined {
  float top = -INFINITY, sum = 0.f, y[N] = {};

  // Parts first, first + step, ... below count; read(k, (maximum, sum), sums)
  // reads part k.  B of them are read before the first is used: the joins are
  // bound by the latency of these reads.
  template <int B, typename Fn>
  __device__ __forceinline__ void take(int count, int first, int step, Fn read) {
    for (int k0 = first; k0 < count; k0 += step * B) {
      float2 ml[B];
      float v[B][N];
#pragma unroll
      for (int i = 0; i < B; ++i) read(min(k0 + step * i, count - 1), ml[i], v[i]);
      float now = top;
#pragma unroll
      for (int i = 0; i < B; ++i)
        if (k0 + step * i < count) now = fmaxf(now, ml[i].x);
      const float ref = now == -INFINITY ? 0.f : now, keep = __builtin_amdgcn_exp2f(top - ref);
      top = now;
      sum *= keep;
#pragma unroll
      for (int n = 0; n < N; ++n) y[n] *= keep;
#pragma unroll
      for (int i = 0; i < B; ++i) {
        if (k0 + step * i >= count) continue;
        const float f = __builtin_amdgcn_exp2f(ml[i].x - ref);
        sum += f * ml[i].y;
#pragma unroll
        for (int n = 0; n < N; ++n) y[n] += f * v[i][n];
      }
    }
  }
};

// Few rows (decoding): 16 R rows a workgroup, its waves take the cached tiles by
// turns, one pass with the running maximum and sum.  Scores are formed as
// S^T = K Q^T and outputs as O^T = V^T P^T: a lane then holds the probabilities
// of its row for eight tokens in a row, which is the operand of the second
// product as it stands, and codes become operands in registers, keys without any
// exchange.  Codes are converted by the hardware (exactly), scales with them.
// Bound by reading the cache, with the conversions' vector work close behind:
// 131,072 tokens of 4 heads of 128, 71 MB, in 20.6 us from memory (3.5 TB/s, about
// 2.5 us of them the first loads' latency) and 18.9 where the last-level cache
// still holds a part; vector instructions issue for 0.65 of the waves' time, and a
// wave waits for loads for 0.43 of its own.  64 sequences of 128 to 8,192 tokens,
// 90 MB, 28.9 us (31 from memory), of which 4.5 joining parts and 2 writing them.
// Four waves and as many workgroups as are resident at once; with one term of a
// probability (see NP), 17.5 us: half as many workgroups 18.5, twice as many 20.7
// and a longer join, 16 waves (a quarter as many parts) 20.0; the 64 sequences
// with half as many parts 36 us, twice as many 36, not 27.  Parts of 4 tiles
// instead of 8 at least: nine short fp32 sequences 13.5 us, not 11.6.
template <typename T, int D, int R>
__global__ __launch_bounds__(64 * kWaves, resident(std::is_same<T, float>::value, D, R)) void kv4_attend_kernel(AttendArgs a) {
  constexpr int W = kWaves;
  constexpr int NS = std::is_same<T, float>::value ? 3 : 1;  // bf16 terms of a query
  // and of a probability: two lose 2^-16 of it, so that a bf16 output is off by
  // its own rounding alone (1.6e-3; with one term 2.3e-3).  One token over
  // 131,072 takes 24.0 us with two and 23.1 with one, 64 ragged sequences 27.8
  // and 26.9.  32 rows a workgroup keep one: their products and vector work bound
  // them, and two terms would make 60 us of 53 (48 sequences of 32 rows over
  // 6,000 tokens) and 93 of 78 (64 rows).
  constexpr int NP = std::is_same<T, float>::value ? 3 : (R == 1 ? 2 : 1);
  using Sum = typename std::conditional<NP == 1, f32x4, float>::type;
  constexpr int KW = D / 32, NT = D / 16;
  constexpr int kRows = 16 * R, kPad = 4;
  __shared__ float s_o[W][16][D + kPad];
  __shared__ float s_m[W][16], s_l[W][16];
  __shared__ unsigned s_done;

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 15, g = lane >> 4;
  Spot at;
  if (!find_spot(a, kRows, lane, at)) return;
  const Seq& seq = at.seq;
  const int h = at.h, row0 = at.row0, last = at.last, parts = at.parts, begin = at.begin, end = at.end;
  const int lim_min = seq.limit(a, row0), lim_max = seq.limit(a, last);

  const int32_t* pages = a.pages + static_cast<int64_t>(at.b) * a.pages_stride;
  const uint8_t* head = a.cache.base + static_cast<uint64_t>(h) * a.cache.head_bytes;
  // two steps ahead the page ids, one step ahead the codes and scales
  int tile = begin + wave;
  const TileLane<D> own(a.cache, head, c, g);
  Pids pid = page_ids(a, pages, tile * kTile, key_token(c), 8 * g);
  Tile<D> next;
  if (tile < end) load_tile<D>(a.cache, own, pid, tile * kTile, next);
  pid = page_ids(a, pages, (tile + W) * kTile, key_token(c), 8 * g);

  u32x4 qf[R][NS][KW];
  int limit[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int row = min(row0 + r * 16 + c, last);  // rows past the last repeat it and are not stored
    limit[r] = seq.limit(a, row);
    load_query<T, D, NS>(a, seq, h, row, g, qf[r]);
  }

  f32x4 o[R][NT];
  Sum l[R];
  float m[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    m[r] = -INFINITY;
    l[r] = Sum{};
#pragma unroll
    for (int n = 0; n < NT; ++n) o[r][n] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  for (; tile < end; tile += W) {
    const int t0 = tile * kTile;
    Tile<D> t = next;
    if (tile + W < end) {
      load_tile<D>(a.cache, own, pid, t0 + W * kTile, next);
      pid = page_ids(a, pages, t0 + 2 * W * kTile, key_token(c), 8 * g);
    }
    const bool masked = t0 + kTile > lim_min;
    __builtin_amdgcn_sched_barrier(0);

    // scores: lane holds tokens 8g + 4i + e of its row c
    f32x4 s[R][2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
#pragma unroll
      for (int r = 0; r < R; ++r) s[r][i] = f32x4{0.f, 0.f, 0.f, 0.f};
      const float sc = scale_of(t.ks[i]);
#pragma unroll
      for (int j = 0; j < KW; ++j) {
        const u32x4 kf = cvt8(t.k[i][j], sc);
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
          for (int n = 0; n < NS; ++n) s[r][i] = mfma(kf, qf[r][NS - 1 - n][j], s[r][i]);
      }
    }
    __builtin_amdgcn_sched_barrier(0);

    if (masked) {
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (t0 + 8 * g + 4 * i + e >= limit[r]) s[r][i][e] = -INFINITY;
    }
    follow_maximum<D, R>(s, a.scale_log2, m, l, o);
    u32x4 pf[R][NP];
    probabilities<R, NP>(s, a.scale_log2, m, l, pf);

    float sc[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) sc[j] = scale_byte(t.vs, j);
    if (masked) {
      // Zero times a value that is not finite is NaN, so none goes into the
      // product of a tile with masked places: what no row sees may hold
      // anything, and where some rows see a NaN block they get their NaN here.
      int poisoned = INT32_MAX;  // the first such token of this lane's block
#pragma unroll
      for (int j = 7; j >= 0; --j) {
        const int token = t0 + 8 * g + j;
        const bool special = ((t.vs[j / 4] >> (8 * (j % 4))) & 255u) > kMaxByte;
        if (special && token < lim_max) poisoned = token;
        if (special || token >= lim_max) {
          t.v[j] = 0u;
          sc[j] = 1.f;
        }
      }
      if (__any(poisoned != INT32_MAX)) {
        // this lane's sums are of block g (D = 128) or g / 2
        const int from = D == 128 ? 4 * g : 8 * (g >> 1);
        int first = INT32_MAX;
#pragma unroll
        for (int k = 0; k < 4; ++k) first = min(first, __shfl(poisoned, 16 * k + from));
#pragma unroll
        for (int r = 0; r < R; ++r)
          if (first < limit[r]) {
#pragma unroll
            for (int n = 0; n < NT; ++n) o[r][n] = f32x4{NAN, NAN, NAN, NAN};
          }
      }
    }
    value_frags<D>(t.v, sc, [&](int n, u32x4 vf) {
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int k = 0; k < NP; ++k) o[r][n] = mfma(vf, pf[r][NP - 1 - k], o[r][n]);
    });
  }

  // rows are divided by the head count again below: the reciprocal from above
  // would take a register through the loop
  AttendArgs again = a;
  asm volatile("" : "+s"(again.G));

  // the waves' sums join: weights 2^(m_w - max m)
  const size_t part_floats = static_cast<size_t>(kRows) * (D + 2);  // [rows][D] sums, then [rows] maximum, sum
  float* part = a.part + at.part * part_floats;
  constexpr int kPer = 16 * D / (64 * W), kThr = D / kPer;  // elements per thread, threads per row
#pragma unroll
  for (int r = 0; r < R; ++r) {
    if (r > 0) __syncthreads();
    float whole;  // the row's sum of this wave's probabilities
    if constexpr (NP == 1) {
      whole = l[r][0];
    } else {
      whole = l[r] + __shfl_xor(l[r], 16);
      whole += __shfl_xor(whole, 32);
    }
    if (g == 0) {
      s_m[wave][c] = m[r];
      s_l[wave][c] = whole;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)  // A row 4g + e is elements (4g + e) * NT + n
#pragma unroll
      for (int n = 0; n < NT; n += 4)
        *reinterpret_cast<f32x4*>(&s_o[wave][c][(4 * g + e) * NT + n]) =
            f32x4{o[r][n][e], o[r][n + 1][e], o[r][n + 2][e], o[r][n + 3][e]};
    __syncthreads();
    // a thread's elements, in pairs: one run of a finished row; of a partial row
    // pairs 2 kThr apart, so that the threads of a row write 128 bytes in a piece
    // (their 8-byte agent-scope writes are not gathered on the way)
    const int rr = threadIdx.x / kThr, tc = threadIdx.x % kThr;
    const int e0 = tc * (parts > 1 ? 2 : kPer), apart = parts > 1 ? 2 * kThr : 2;
    const int row = row0 + r * 16 + rr;
    if (row > last) continue;
    float top = s_m[0][rr];
#pragma unroll
    for (int w = 1; w < W; ++w) top = fmaxf(top, s_m[w][rr]);
    const float ref = top == -INFINITY ? 0.f : top;
    float sum = 0.f, y[kPer];
#pragma unroll
    for (int k = 0; k < kPer; ++k) y[k] = 0.f;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const float f = __builtin_amdgcn_exp2f(s_m[w][rr] - ref);
      sum += f * s_l[w][rr];
#pragma unroll
      for (int k = 0; k < kPer; k += 2) {
        const float2 v = *reinterpret_cast<const float2*>(&s_o[w][rr][e0 + k / 2 * apart]);
        y[k] += f * v.x;
        y[k + 1] += f * v.y;
      }
    }
    if (parts > 1) {
      const int ri = r * 16 + rr;
      float *to = part + ri * D + e0, *ml = part + kRows * D + 2 * ri;
#pragma unroll
      for (int k = 0; k < kPer; k += 2) {
        if (a.join_apart)
          *reinterpret_cast<float2*>(to + k / 2 * apart) = make_float2(y[k], y[k + 1]);
        else
          put2(to + k / 2 * apart, y[k], y[k + 1]);
      }
      if (tc == 0) {
        if (a.join_apart)
          *reinterpret_cast<float2*>(ml) = make_float2(top, sum);
        else
          put2(ml, top, sum);
      }
      continue;
    }
    finish<T, kPer>(again, seq, h, row, D, e0, sum, y);
  }
  if (parts == 1 || a.join_apart) return;

  // The workgroup that finishes a sequence's parts last joins them, in their
  // order.  Parts pass between XCDs, whose L2 caches do not see each other:
  // they are written and read at agent scope, past those caches, and counted
  // only when every write has arrived.  (Fences in their place write back and
  // drop whole caches: one token against 131,072 took 92 us, not 27, joined this way.)
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (threadIdx.x == 0) {
    unsigned* count = a.count + static_cast<size_t>(at.rt * a.Hkv + h) * a.n_seq + at.b;
    const unsigned before = __hip_atomic_fetch_add(count, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (before + 1 >= static_cast<unsigned>(parts)) __hip_atomic_store(count, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    s_done = before + 1;
  }
  __syncthreads();
  const unsigned done = __builtin_amdgcn_readfirstlane(s_done);
  if (done < static_cast<unsigned>(parts)) return;
  const float* all = part - static_cast<size_t>(at.split) * part_floats;
  constexpr int kCols = D / 4, kSlots = 64 * W / kCols;  // a slot of threads takes a row of a group of parts
  const int slot = threadIdx.x / kCols, col = threadIdx.x % kCols, rows = last - row0 + 1;
  const int groups = max(1, kSlots / rows);
  float* s_y = &s_o[0][0][0];  // [kSlots][D]
  float *s_sum = &s_l[0][0], *s_top = &s_m[0][0];
  static_assert(sizeof(s_o) >= sizeof(float) * kSlots * D && sizeof(s_l) >= sizeof(float) * kSlots, "join buffers");
  for (int ri = groups > 1 ? slot % rows : slot, grp = groups > 1 ? slot / rows : 0; ri < rows; ri += kSlots) {
    Joined<4> j;
    if (grp < groups)
      j.template take<8>(parts, grp, groups, [&](int k, float2& ml, float* v) {
        const float* from = all + k * part_floats;
        ml = get2(from + kRows * D + 2 * ri);
        const float2 lo = get2(from + ri * D + 4 * col), hi = get2(from + ri * D + 4 * col + 2);
        v[0] = lo.x, v[1] = lo.y, v[2] = hi.x, v[3] = hi.y;
      });
    if (groups > 1) {
      *reinterpret_cast<f32x4*>(s_y + slot * D + 4 * col) = f32x4{j.y[0], j.y[1], j.y[2], j.y[3]};
      if (col == 0) s_sum[slot] = j.sum, s_top[slot] = j.top;
      __syncthreads();
      if (slot >= rows) return;
      Joined<4> whole;
      whole.template take<1>(groups, 0, 1, [&](int k, float2& ml, float* v) {
        const int from = slot + k * rows;
        ml = make_float2(s_top[from], s_sum[from]);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = s_y[from * D + 4 * col + i];
      });
      j = whole;
    }
    // a count beyond the parts: the workspace was not zero, and nothing is known of the parts
    finish<T, 4>(again, seq, h, row0 + ri, D, 4 * col, done > static_cast<unsigned>(parts) ? NAN : j.sum, j.y);
  }
}

// Many rows (a prompt's tokens): 16 R rows a wave, 8 waves a workgroup.  The
// waves form the operands of a step's two tiles together, each its share of
// the codes, straight in the order in which lanes read them from LDS; then
// every wave multiplies them with its own rows.  One barrier a step: while one
// step is multiplied, the codes of the next ones are on their way.  A tile's
// scores are multiplied while the tile before it goes through the softmax, so
// that the matrix cores and the vector units have work at the same time; the
// keys are therefore formed two steps ahead, the values one, beside the value
// products.  2 sequences of 1,024 tokens over 8,192, 32 heads of 128, 256 us,
// 1,007 TFLOP/s (1,140 for a large library product here).  The matrix units are
// busy for 0.46 of that, other vector instructions issue for 0.36, and the two
// waves of a SIMD overlap the two only in part; a wave waits for LDS, loads and
// the barrier for 0.29 of its time.  On the way: 64 rows a workgroup in the form
// above 437 us; operands shared, tile after tile 349; scores ahead 325; wider
// loads of the codes 271; forming beside the products 258.  Without forming (wrong
// results) it is 228.
constexpr int kRowWaves = 8;

// Two tokens' codes as words of the value operands: fn(n, word) for element n
template <int D, int B = 0, typename Fn>
__device__ __forceinline__ void join_pairs(const uint32_t (&codes)[2], float s0, float s1, Fn fn) {
  const uint32_t x = cvt2<B>(codes[0], s0), y = cvt2<B>(codes[1], s1);
  fn(2 * B, __builtin_amdgcn_perm(y, x, 0x05040100u));
  fn(2 * B + 1, __builtin_amdgcn_perm(y, x, 0x07060302u));
  if constexpr (B + 1 < D / 32) join_pairs<D, B + 1>(codes, s0, s1, fn);
}

template <int D>
struct RawKeys {
  uint32_t k[D / 64];  // the lane's words of one token's codes
  uint32_t ks;
};
struct RawValues {
  uint32_t v[2];  // codes of two tokens (D = 64: 16 bits each)
  uint32_t vs;    // their scale bytes
};

template <typename T, int D, int R>
__global__ __launch_bounds__(64 * kRowWaves, 2) void kv4_attend_rows_kernel(AttendArgs a) {
  constexpr int W = kRowWaves;
  // bf16 terms of a query and of a probability.  One term of a probability is a
  // choice: bf16 outputs are then 2.3e-3 from the exact ones instead of the 1.7e-3
  // that their own rounding costs, but two terms make 347 us of the 256 above.
  constexpr int NS = std::is_same<T, float>::value ? 3 : 1;
  constexpr int KW = D / 32, NT = D / 16;
  constexpr int kRows = 16 * R * W;
  __shared__ u32x4 s_k[3][2][2 * KW][64];  // buffer, tile, (half of the tile's tokens, step over elements), lane
  __shared__ u32x4 s_v[2][2][NT][64];
  __shared__ int s_poisoned[D / 32];

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 15, g = lane >> 4;
  Spot at;
  if (!find_spot(a, kRows, lane, at)) return;
  const Seq& seq = at.seq;
  if (threadIdx.x < D / 32) s_poisoned[threadIdx.x] = INT32_MAX;
  const int lim_all = seq.limit(a, at.last);
  const int row0 = at.row0 + wave * 16 * R, last = min(row0 + 16 * R - 1, at.last);
  const bool mine = row0 <= at.last;
  const int lim_min = mine ? seq.limit(a, row0) : 0, lim_max = mine ? seq.limit(a, last) : 0;

  const int32_t* pages = a.pages + static_cast<int64_t>(at.b) * a.pages_stride;
  const uint8_t* head = a.cache.base + static_cast<uint64_t>(at.h) * a.cache.head_bytes;
  // this wave's share of a step: of tile wave / 4 the keys of half (wave / 2) % 2,
  // every second pair of their words, and the value tokens 8g + 2 (wave % 4) and
  // the next, which are one word of each operand
  const int share = wave >> 2, half = (wave >> 1) & 1, part_k = wave & 1, pair = wave & 3;
  const int kt = key_token(c) + 4 * half, vt = 8 * g + 2 * pair, kin = kt & (a.cache.page - 1), vin = vt & (a.cache.page - 1);
  const uint8_t* own_k = head + Block<D>::codes(a.cache.page, 0, kin) + g * (D / 8) + part_k * (D / 16);
  const uint8_t* own_ks = head + Block<D>::scales(a.cache.page, 0, g * (D / 4) / 32, kin);
  const uint8_t* own_v = head + Block<D>::codes(a.cache.page, 1, vin) + c * (D / 32);
  const uint8_t* own_vs = head + Block<D>::scales(a.cache.page, 1, c * (D / 16) / 32, vin);
  const auto load_keys = [&](int pid, int t0, RawKeys<D>& x) {
    const bool none = no_page(a.cache, pid);
    const uint32_t u = static_cast<uint32_t>(t0 & (a.cache.page - 1));
    const uint8_t* k = in_page(a.cache, own_k, none ? 0 : pid, u * (D / 2));
    if constexpr (D == 128) {
      const u32x2 w = *reinterpret_cast<const u32x2*>(k);
      x.k[0] = w[0], x.k[1] = w[1];
    } else {
      x.k[0] = *reinterpret_cast<const uint32_t*>(k);
    }
    const uint32_t byte = *in_page(a.cache, own_ks, none ? 0 : pid, u);
    x.ks = none ? static_cast<uint32_t>(kNanByte) : byte;
  };
  const auto load_values = [&](int pid, int t0, RawValues& x) {
    const int p = no_page(a.cache, pid) ? 0 : pid;
    const uint32_t u = static_cast<uint32_t>(t0 & (a.cache.page - 1));
    const uint8_t* v = in_page(a.cache, own_v, p, u * (D / 2));
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      if constexpr (D == 128)
        x.v[j] = *reinterpret_cast<const uint32_t*>(v + j * (D / 2));
      else
        x.v[j] = *reinterpret_cast<const uint16_t*>(v + j * (D / 2));
    }
    x.vs = *reinterpret_cast<const uint16_t*>(in_page(a.cache, own_vs, p, u));
  };
  const auto form_keys = [&](const RawKeys<D>& x, int buf) {
    const float ks = scale_of(x.ks);
#pragma unroll
    for (int j = 0; j < D / 64; ++j) s_k[buf][share][half * KW + part_k * (D / 64) + j][lane] = cvt8(x.k[j], ks);
  };
  // Values that are not finite go in as zeros, whoever sees them, and rows that
  // see one of a block's get their NaN at the end: the first such token is
  // enough to know, since a row sees all tokens up to its limit.
  int poisoned = INT32_MAX;
  const auto form_values = [&](const RawValues& x, int t0, int buf, int lim) {
    uint32_t codes[2] = {x.v[0], x.v[1]}, scales = x.vs;
    if (__any(high_byte(scales))) {
#pragma unroll
      for (int j = 1; j >= 0; --j) {
        const int token = t0 + vt + j;
        if (((scales >> (8 * j)) & 255u) <= kMaxByte) continue;
        if (token < lim) poisoned = min(poisoned, token);
        codes[j] = 0u;
        scales &= ~(128u << (8 * j));
      }
    }
    uint32_t* to = reinterpret_cast<uint32_t*>(&s_v[buf][share][0][lane]) + pair;
    join_pairs<D>(codes, scale_of(scales & 255u), scale_of(scales >> 8), [&](int n, uint32_t w) { to[n * 64 * 4] = w; });
  };

  // where this wave's share of the step at `tile` starts, and the pages there
  const auto start = [&](int tile) { return (tile + share) * kTile; };
  const auto ids = [&](int tile) { return page_ids(a, pages, start(tile), kt, vt); };
  int tile = at.begin;
  RawKeys<D> rk, rk1;
  RawValues rv;
  Pids id = ids(tile), id1 = ids(tile + 2);
  load_keys(id.k, start(tile), rk);
  load_values(id.v, start(tile), rv);
  load_keys(id1.k, start(tile + 2), rk1);
  const Pids id2 = ids(tile + 4);

  u32x4 qf[R][NS][KW];
  int limit[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int row = min(row0 + r * 16 + c, at.last);
    limit[r] = seq.limit(a, row);
    load_query<T, D, NS>(a, seq, at.h, row, g, qf[r]);
  }
  f32x4 o[R][NT], l[R];
  float m[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    m[r] = -INFINITY;
    l[r] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int n = 0; n < NT; ++n) o[r][n] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  form_keys(rk, 0);
  form_values(rv, start(tile), 0, at.begin < at.end ? lim_all : 0);
  form_keys(rk1, 1);
  load_values(id1.v, start(tile + 2), rv);
  load_keys(id2.k, start(tile + 4), rk);
  id = id2;
  id1 = ids(tile + 6);  // the next step's keys and the values behind them: read a step before they are needed
  __syncthreads();

  const auto scores = [&](int buf, int i2, f32x4 (&s)[R][2]) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
#pragma unroll
      for (int r = 0; r < R; ++r) s[r][i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < KW; ++j) {
        const u32x4 kf = s_k[buf][i2][i * KW + j][lane];
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
          for (int n = 0; n < NS; ++n) s[r][i] = mfma(kf, qf[r][NS - 1 - n][j], s[r][i]);
      }
    }
  };
  const auto hide = [&](int t0, f32x4 (&s)[R][2]) {
    if (t0 + kTile > lim_min) {
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (t0 + 8 * g + 4 * i + e >= limit[r]) s[r][i][e] = -INFINITY;
    }
  };
  // a wave has work as long as its rows see something of a tile
  const auto seen = [&](int tile) { return tile < at.end && tile * kTile < lim_max; };
  bool live = seen(tile);
  f32x4 s[R][2], s2[R][2];  // by turns: the tile that is in the softmax, and the next one's
  if (live) {
    scores(0, 0, s);
    hide(tile * kTile, s);
    follow_maximum<D, R>(s, a.scale_log2, m, l, o);
  }
  // The operands' reads stand half a tile or more before their products, so
  // that the waves, which are in step behind a barrier, do not all wait for LDS
  // at once.  kh: the first half of the keys of the scores to come.
  constexpr int QF = 2 * KW, kHalf = QF / 2, kEach = 8 * R / QF;  // kEach: powers behind each operand's products
  u32x4 kh[kHalf];
  const auto key = [&](int buf, int i2, int q) { return s_k[buf][i2][q % 2 * KW + q / 2][lane]; };  // halves by turns
  const auto step = [&](int now, int kbuf, int vbuf, int i2, int after, f32x4 (&s)[R][2], f32x4 (&ahead)[R][2],
                        const auto& form) {
    if (!live) return form();
    u32x4 kl[kHalf], vf[NT];
#pragma unroll
    for (int q = 0; q < kHalf; ++q) kl[q] = key(kbuf, 1 - i2, kHalf + q);
    float ref[R], p[R][8];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      ref[r] = m[r] == -INFINITY ? 0.f : m[r];  // nothing seen yet: every power is 0
#pragma unroll
      for (int i = 0; i < 2; ++i) ahead[r][i] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int q = 0; q < QF; ++q) {
      const u32x4 kf = q < kHalf ? kh[q] : kl[q - kHalf];
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int n = 0; n < NS; ++n) ahead[r][q % 2] = mfma(kf, qf[r][NS - 1 - n][q / 2], ahead[r][q % 2]);
#pragma unroll
      for (int x = 0; x < kEach; ++x) {
        const int at = q * kEach + x, r = at / 8, k = at % 8;
        p[r][k] = __builtin_amdgcn_exp2f(fmaf(s[r][k / 4][k % 4], a.scale_log2, -ref[r]));
        asm volatile("" : "+v"(p[r][k]));  // here, not where it is used
      }
      if (q == kHalf - 1) {
#pragma unroll
        for (int n = 0; n < NT / 2; ++n) vf[n] = s_v[vbuf][i2][n][lane];
      }
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int n = NT / 2; n < NT; ++n) vf[n] = s_v[vbuf][i2][n][lane];
    u32x4 pf[R][NS];
#pragma unroll
    for (int r = 0; r < R; ++r) split8<NS>(p[r], pf[r]);
    live = seen(now + 1);
    if (live) hide((now + 1) * kTile, ahead);
    form();  // vector work beside the products below
    const u32x4 ones = u32x4{0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u};
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int k = 0; k < NS; ++k) l[r] = mfma(ones, pf[r][NS - 1 - k], l[r]);
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      if (n == NT / 2) {
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int q = 0; q < kHalf; ++q) kh[q] = key(after, i2, q);
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int k = 0; k < NS; ++k) o[r][n] = mfma(vf[n], pf[r][NS - 1 - k], o[r][n]);
    }
    if (live) follow_maximum<D, R>(ahead, a.scale_log2, m, l, o);
  };
  int kbuf = 0, knext = 1, kfree = 2;
#pragma unroll
  for (int q = 0; q < kHalf; ++q) kh[q] = key(kbuf, 1, q);
  for (int vbuf = 0; tile < at.end; tile += 2, vbuf ^= 1) {
    // the scores to come: tile 1 of this step, then tile 0 of the next, whose tile 1 follows; behind the last step
    // what is formed and read is of no use, and of the cache all the same
    step(tile, kbuf, vbuf, 0, knext, s, s2, [&] {
      form_keys(rk, kfree);
      load_keys(id1.k, start(tile + 6), rk);
    });
    step(tile + 1, knext, vbuf, 1, knext, s2, s, [&] {
      form_values(rv, start(tile + 2), vbuf ^ 1, tile + 2 < at.end ? lim_all : 0);
      load_values(id.v, start(tile + 4), rv);
      id = id1;
      id1 = ids(tile + 8);
    });
    const int used = kbuf;
    kbuf = knext, knext = kfree, kfree = used;
    __syncthreads();
  }

  // this lane's sums are of block g (D = 128) or g / 2
  if (poisoned != INT32_MAX) atomicMin(&s_poisoned[c * (D / 16) / 32], poisoned);
  __syncthreads();
  const int first = s_poisoned[g * (D / 4) / 32];
  constexpr size_t kPartFloats = static_cast<size_t>(kRows) * (D + 2);
  float* part = a.part + at.part * kPartFloats;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int row = row0 + r * 16 + c, ri = row - at.row0;
    if (row > at.last) continue;
    const float sum = l[r][0];
#pragma unroll
    for (int e = 0; e < 4; ++e) {  // A row 4g + e is elements (4g + e) * NT + n
      const int e0 = (4 * g + e) * NT;
      float y[NT];
#pragma unroll
      for (int n = 0; n < NT; ++n) y[n] = first < limit[r] ? NAN : o[r][n][e];
      if (at.parts > 1) {
#pragma unroll
        for (int n = 0; n < NT; n += 4)
          *reinterpret_cast<f32x4*>(part + ri * D + e0 + n) = f32x4{y[n], y[n + 1], y[n + 2], y[n + 3]};
      } else {
        finish<T, NT>(a, seq, at.h, row, D, e0, sum, y);
      }
    }
    if (at.parts > 1 && g == 0) *reinterpret_cast<float2*>(part + kRows * D + 2 * ri) = make_float2(m[r], sum);
  }
}

// Joins the parts of rows.  W = 16: a workgroup of 16 waves per (row, head and
// sequence), for many parts: a wave takes every 16th, and the waves' sums join.
// W = 1: a wave per row, four rows a workgroup.  Bound by the latency of the
// reads, so a wave has several parts' in flight at once.
template <typename T, int D, int kRows, int W>
__global__ __launch_bounds__(64 * (W == 1 ? 4 : W)) void kv4_join_kernel(AttendArgs a) {
  constexpr int kPer = D / 64, kBatch = W == 1 ? 8 : 16;
  __shared__ float s_y[W][D], s_sum[W], s_m[W];
  const int heads = a.n_seq * a.Hkv;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int bh = static_cast<int>(blockIdx.x) % heads;
  const int row = W == 1 ? static_cast<int>(blockIdx.x) / heads * 4 + wave : static_cast<int>(blockIdx.x) / heads;
  const int b = bh / a.Hkv, h = bh - b * a.Hkv;
  const Place at = place_of(a, 0, b, lane);
  const Seq& seq = at.seq;
  const int nrows = min(seq.nq * a.G, a.max_rows);
  if (row >= nrows) return;
  const int rt = row / kRows, ri = row - rt * kRows;
  const int tiles = (seq.limit(a, min((rt + 1) * kRows, nrows) - 1) + kTile - 1) / kTile;
  const int parts = max(1, static_cast<int>((static_cast<uint32_t>(tiles) + at.each - 1) / static_cast<uint32_t>(at.each)));
  if (parts == 1) return;  // written whole
  constexpr size_t kStride = static_cast<size_t>(kRows) * (D + 2);
  const float* part = a.part + (static_cast<size_t>(rt * a.Hkv + h) * (a.units + a.n_seq) + at.base) * kStride;
  Joined<kPer> j;
  j.template take<kBatch>(parts, W == 1 ? 0 : wave, W, [&](int k, float2& ml, float* v) {
    const float* from = part + k * kStride;
    ml = *reinterpret_cast<const float2*>(from + kRows * D + 2 * ri);
#pragma unroll
    for (int i = 0; i < kPer; ++i) v[i] = from[ri * D + lane * kPer + i];
  });
  if constexpr (W > 1) {
    if (lane == 0) s_sum[wave] = j.sum, s_m[wave] = j.top;
#pragma unroll
    for (int k = 0; k < kPer; ++k) s_y[wave][lane * kPer + k] = j.y[k];
    __syncthreads();
    if (wave != 0) return;
    Joined<kPer> whole;
    whole.template take<W>(W, 0, 1, [&](int k, float2& ml, float* v) {
      ml = make_float2(s_m[k], s_sum[k]);
#pragma unroll
      for (int i = 0; i < kPer; ++i) v[i] = s_y[k][lane * kPer + i];
    });
    j = whole;
  }
  finish<T, kPer>(a, seq, h, row, D, lane * kPer, j.sum, j.y);
}

// ------------------------------------------------------------------ host side

bool aligned(const void* p, unsigned n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

spp_status bad(const char* why) { return spp::set_error(SPP_EINVAL, why); }

const char* desc_why(const spp_attn_desc* d) {
  if (!d) return "desc is NULL";
  if (d->n_kv_heads < 1 || d->n_heads < 1 || d->n_heads > 1024 || d->n_heads % d->n_kv_heads != 0)
    return "n_heads must be a multiple of n_kv_heads, both at least 1 and n_heads at most 1024";
  if (d->head_dim != 64 && d->head_dim != 128) return "head_dim must be 64 or 128";
  if (d->page != 16 && d->page != 32 && d->page != 64 && d->page != 128 && d->page != 256)
    return "page must be 16, 32, 64, 128 or 256";
  if (d->n_pages < 1) return "n_pages must be at least 1";
  return nullptr;
}

Cache cache_of(const spp_attn_desc* d, const void* base) {
  Cache c;
  c.base = static_cast<const uint8_t*>(base);
  c.head_bytes = static_cast<uint32_t>(d->page * (d->head_dim + d->head_dim / 16));
  c.page_bytes = c.head_bytes * static_cast<uint32_t>(d->n_kv_heads);  // at most 2^10 heads of 256 tokens: 36 MB
  c.page = d->page;
  c.shift = __builtin_ctz(static_cast<unsigned>(d->page));
  c.n_pages = d->n_pages;
  return c;
}

constexpr int64_t kMaxUnits = int64_t{1} << 30;     // so that 32-bit indices hold
constexpr int64_t kMaxHeadRows = int64_t{1} << 27;  // 16 threads each: a launch has less than 2^32

// Rows [T][heads][d] at a stride of `stride` elements
const char* rows_why(const void* p, int64_t stride, int heads, int d, int elem) {
  if (stride < static_cast<int64_t>(heads) * d) return "a row stride is smaller than its row";
  if (stride > kMaxUnits) return "a row stride is larger than 2^30 elements";
  if (!aligned16(p) || stride * elem % 16 != 0) return "rows must be 16-byte aligned, their stride a multiple of 16 bytes";
  return nullptr;
}

// Bytes from the first row's start to the last one's end
uint64_t extent(int64_t stride, int64_t T, int heads, int d, int elem) {
  return static_cast<uint64_t>((T - 1) * stride + static_cast<int64_t>(heads) * d) * static_cast<uint64_t>(elem);
}

bool overlap(const void* a, uint64_t na, const void* b, uint64_t nb) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x < y + nb && y < x + na;
}

// Whether T rows of na bytes, sa bytes apart, and T rows of nb bytes, sb apart,
// have a byte in common (a stride is at least its row).  Rows of one fused
// product lie between each other without.
bool rows_overlap(const void* a, int64_t sa, int64_t na, const void* b, int64_t sb, int64_t nb, int64_t T) {
  const int64_t span_a = (T - 1) * sa + na, span_b = (T - 1) * sb + nb;
  if (!overlap(a, static_cast<uint64_t>(span_a), b, static_cast<uint64_t>(span_b))) return false;
  const int64_t off = static_cast<int64_t>(reinterpret_cast<uintptr_t>(b) - reinterpret_cast<uintptr_t>(a));
  const auto below = [](int64_t x, int64_t y) { return x / y - (x % y < 0); };  // floor(x / y)
  // rows of a from the first that ends past row u of b to the last that starts before its end
  const auto meets = [&](int64_t u) {
    const int64_t at = off + u * sb;
    return std::max<int64_t>(0, below(at - na, sa) + 1) <= std::min<int64_t>(T - 1, below(at + nb - 1, sa));
  };
  // with one stride all of b's rows lie alike to a's: its first and last are the ones that meet the most
  if (sa == sb) return meets(0) || meets(T - 1);
  for (int64_t u = 0; u < T; ++u)
    if (meets(u)) return true;
  return false;
}

const char* dtype_why(int32_t dtype) {
  return dtype == SPP_DTYPE_F32 || dtype == SPP_DTYPE_BF16 ? nullptr : "dtype must be 0 (f32) or 1 (bf16)";
}

spp_status launched(hipError_t e) { return e == hipSuccess ? SPP_OK : spp::set_error(SPP_EHIP, hipGetErrorString(e)); }

// The launch's own status, and no other call's that may still be pending
template <typename Args>
hipError_t launch(void (*kernel)(Args), unsigned grid, unsigned threads, const Args& args, hipStream_t st) {
  void* params[] = {const_cast<Args*>(&args)};
  return hipLaunchKernel(reinterpret_cast<const void*>(kernel), dim3(grid), dim3(threads), params, 0, st);
}

#define SPP_BAD(expr)                   \
  do {                                  \
    if (const char* w_ = (expr)) return bad(w_); \
  } while (0)

template <typename T>
hipError_t launch_store(const StoreArgs& a, int d, unsigned grid, hipStream_t st) {
  return d == 128 ? launch(kv4_store_kernel<T, 128>, grid, 256, a, st) : launch(kv4_store_kernel<T, 64>, grid, 256, a, st);
}

template <typename T>
hipError_t launch_load(const LoadArgs& a, int d, unsigned grid, hipStream_t st) {
  return d == 128 ? launch(kv4_load_kernel<T, 128>, grid, 256, a, st) : launch(kv4_load_kernel<T, 64>, grid, 256, a, st);
}

// How a call's work is cut: rows per workgroup, row tiles, waves per workgroup,
// and about how many parts a plane's cached tokens make.  Goes by the caller's
// bounds alone, so that the workspace can be sized without a device.
struct Cut {
  int form;  // 0: 16 rows, 1: 32 rows, whose waves share the tokens out; 2: kv4_attend_rows_kernel
  int rows;  // rows per workgroup
  int row_tiles, planes, units;
  bool join_apart;
};

constexpr int kCUs = 256;
constexpr int kMinTiles = 2 * kWaves;  // two steps a wave
// Parts a sequence from which a launch of its own joins them: 256 parts by the
// last workgroup alone would read 1 MB in turn (131,072 tokens 51.9 us in all, 24.0
// with a launch of 5.8), while 64 sequences in about four parts each take 27.8 us
// joined by the last workgroup and 44.9 with a launch.
constexpr int kFusedParts = 32;
constexpr int kPairRows = 32, kFewRows = 208, kFewHeads = 32;

// The counters stand at the workspace's start and take the same room in every
// call, so that no call's partial rows come to lie where another one counts.
constexpr int kMaxItems = 4 * kCUs * 4;
constexpr size_t kCountBytes = kMaxItems * sizeof(unsigned);

// Rows of a wave of kv4_attend_rows_kernel, in sixteens, by the registers of fp32's three terms
constexpr int rows_r(bool f32, int d) { return f32 && d == 128 ? 1 : 2; }

// kv4_attend_rows_kernel takes 256 rows (128 for fp32 heads of 128) whether they
// are there or not, but needs fewer parts to fill the device.  Measured in us,
// 8 heads per key/value head of 128, tokens cut over the waves / rows over them:
// 48 sequences over 6,000 tokens of 64 rows each 78 / 146, of 192 rows 176 /
// 212; one sequence of 64 rows 26 / 18, of 192 rows 25 / 25; six sequences of
// 64 rows 34 / 29, of 128 rows 34 / 35; of 24 rows 20 / 16 and 26 / 25, but over
// 1,000 tokens 12.7 / 14.0.
int form_of(int64_t rows, int64_t heads) {
  if (rows <= 16) return 0;
  return rows <= kPairRows || (rows <= kFewRows && heads > kFewHeads) ? 1 : 2;
}

int group_rows(bool f32, int d, int form) { return form == 2 ? 16 * kRowWaves * rows_r(f32, d) : 16 << form; }

// Workgroups that fill the device
int fill(bool f32, int d, int form) { return form == 2 ? kCUs : kCUs * resident(f32, d, 1 << form); }

// Row tiles, over all sequences and heads, below which tokens are split
int split_below(bool f32, int d, int form) { return form == 2 ? kCUs : std::min(4 * fill(f32, d, form), kMaxItems); }

Cut cut_of(const spp_attn_desc* d, bool f32, int32_t n_seq, int32_t max_q, int32_t max_kv) {
  Cut c{};
  const int64_t rows = static_cast<int64_t>(max_q) * (d->n_heads / d->n_kv_heads);
  c.form = form_of(rows, static_cast<int64_t>(n_seq) * d->n_kv_heads);
  c.rows = group_rows(f32, d->head_dim, c.form);
  c.row_tiles = static_cast<int>((rows + c.rows - 1) / c.rows);
  c.planes = d->n_kv_heads * c.row_tiles;
  const int64_t items = static_cast<int64_t>(n_seq) * c.planes;
  const int64_t tiles = (static_cast<int64_t>(max_kv) + kTile - 1) / kTile;
  if (items == 0 || tiles <= kMinTiles || items >= split_below(f32, d->head_dim, c.form)) return c;
  c.units = std::max(1, fill(f32, d->head_dim, c.form) / c.planes - n_seq / 2);
  c.join_apart = c.form == 2 || std::min<int64_t>(c.units / n_seq, tiles / kMinTiles) >= kFusedParts;
  return c;
}

size_t part_bytes(const Cut& c, int32_t n_seq, int d) {
  return c.units > 0 ? static_cast<size_t>(c.planes) * (c.units + n_seq) * c.rows * (d + 2) * sizeof(float) : 0;
}

// Workgroups of the attention itself
int64_t attend_grid(const Cut& c, int64_t n_seq, int64_t Hkv) {
  if (c.units > 0) return (c.units + n_seq) * c.planes;
  return (c.row_tiles > 1 ? (n_seq * Hkv + 7) / 8 * 8 : n_seq * Hkv) * c.row_tiles;
}

template <typename T, int D>
hipError_t launch_attend_d(const AttendArgs& a, const Cut& c, int64_t rows, hipStream_t st) {
  constexpr bool f32 = std::is_same<T, float>::value;
  const auto run = [&](void (*kernel)(AttendArgs), void (*joining)(AttendArgs), int waves, int rows_each, int join_waves) {
    const hipError_t e = launch(kernel, static_cast<unsigned>(attend_grid(c, a.n_seq, a.Hkv)), 64u * waves, a, st);
    if (e != hipSuccess || !c.join_apart) return e;
    return launch(joining, static_cast<unsigned>(a.n_seq * a.Hkv * ((rows + rows_each - 1) / rows_each)), 64u * join_waves,
                  a, st);
  };
  constexpr int kR = rows_r(f32, D);
  if (c.form == 0) return run(kv4_attend_kernel<T, D, 1>, kv4_join_kernel<T, D, 16, 16>, kWaves, 1, 16);
  if (c.form == 1) return run(kv4_attend_kernel<T, D, 2>, kv4_join_kernel<T, D, 32, 16>, kWaves, 1, 16);
  return run(kv4_attend_rows_kernel<T, D, kR>, kv4_join_kernel<T, D, 16 * kRowWaves * kR, 1>, kRowWaves, 4, 4);
}

template <typename T>
hipError_t launch_attend(const AttendArgs& a, int d, const Cut& c, int64_t rows, hipStream_t st) {
  return d == 128 ? launch_attend_d<T, 128>(a, c, rows, st) : launch_attend_d<T, 64>(a, c, rows, st);
}

}  // namespace

extern "C" size_t spp_kv4_cache_bytes(const spp_attn_desc* desc) {
  if (const char* w = desc_why(desc)) return bad(w), 0;
  return static_cast<size_t>(cache_of(desc, nullptr).page_bytes) * static_cast<size_t>(desc->n_pages);
}

extern "C" spp_status spp_rotary_table(const int32_t* pos, int64_t pos_stride, int32_t n_axes, const int32_t* axis_of,
                                       const float* inv_freq, int32_t n_freq, int32_t T, float* table,
                                       void* hip_stream) {
  if (n_axes < 1 || n_axes > 4) return bad("n_axes must be in [1, 4]");
  if (n_freq < 8 || n_freq > kMaxFreq || n_freq % 8 != 0) return bad("n_freq must be a multiple of 8 in [8, 64]");
  if (T < 0 || static_cast<int64_t>(T) * n_freq > kMaxUnits) return bad("T must be >= 0, T * n_freq at most 2^30");
  TableArgs a{};
  for (int i = 0; axis_of && i < n_freq; ++i) {
    if (axis_of[i] < 0 || axis_of[i] >= n_axes) return bad("axis_of names an axis outside [0, n_axes)");
    a.axes[i / 16] |= static_cast<uint32_t>(axis_of[i]) << (2 * (i % 16));
  }
  if (T == 0) return SPP_OK;
  if (!pos || !inv_freq || !table) return bad("pos, inv_freq and table must not be NULL");
  if ((n_axes > 1 && pos_stride < T) || pos_stride > int64_t{1} << 40) return bad("pos_stride must be at least T");
  if (!aligned16(table) || !aligned(pos, 4) || !aligned(inv_freq, 4))
    return bad("table must be 16-byte aligned, pos and inv_freq aligned to their elements");
  a.pos = pos;
  a.pos_stride = pos_stride;
  a.inv_freq = inv_freq;
  a.table = table;
  a.F = n_freq;
  a.T = T;
  const int64_t threads = static_cast<int64_t>(T) * (n_freq / kTableFreqs);
  return launched(launch(rotary_table_kernel, static_cast<unsigned>((threads + 255) / 256), 256, a,
                         static_cast<hipStream_t>(hip_stream)));
}

extern "C" spp_status spp_kv4_store(const spp_attn_desc* desc, void* cache, int32_t dtype, const void* q,
                                    int64_t q_stride, void* q_out, int64_t q_out_stride, const void* k,
                                    int64_t k_stride, const void* v, int64_t v_stride, const float* table,
                                    int32_t n_freq, const int64_t* slots, int32_t T, void* hip_stream) {
  SPP_BAD(desc_why(desc));
  SPP_BAD(dtype_why(dtype));
  const int d = desc->head_dim, elem = dtype == SPP_DTYPE_BF16 ? 2 : 4;
  if (n_freq < 0 || n_freq % 8 != 0 || 2 * n_freq > d) return bad("n_freq must be a multiple of 8, at most head_dim / 2");
  if ((table != nullptr) != (n_freq > 0) && T > 0) return bad("table must be given iff n_freq > 0");
  if ((q != nullptr) != (q_out != nullptr)) return bad("q and q_out must be given together");
  const int Hq = q ? desc->n_heads : 0;
  if (T < 0 || static_cast<int64_t>(T) * (desc->n_heads + 2 * desc->n_kv_heads) > kMaxHeadRows)
    return bad("T must be >= 0, T * (n_heads + 2 n_kv_heads) at most 2^27");
  if (T == 0) return SPP_OK;
  if (!cache || !k || !v || !slots) return bad("cache, k, v and slots must not be NULL");
  if (!aligned16(cache) || !aligned(slots, 8)) return bad("cache must be 16-byte aligned, slots 8-byte aligned");
  if (table && !aligned16(table)) return bad("table must be 16-byte aligned");
  SPP_BAD(rows_why(k, k_stride, desc->n_kv_heads, d, elem));
  SPP_BAD(rows_why(v, v_stride, desc->n_kv_heads, d, elem));
  if (q) {
    SPP_BAD(rows_why(q, q_stride, desc->n_heads, d, elem));
    SPP_BAD(rows_why(q_out, q_out_stride, desc->n_heads, d, elem));
    const bool same = q == q_out && q_stride == q_out_stride;
    const uint64_t out_bytes = extent(q_out_stride, T, desc->n_heads, d, elem);
    if (!same && overlap(q, extent(q_stride, T, desc->n_heads, d, elem), q_out, out_bytes))
      return bad("q_out must be q with the same stride, or not overlap it");
    const int64_t kv_bytes = static_cast<int64_t>(desc->n_kv_heads) * d * elem;
    for (const auto& [rows, stride] : {std::pair{k, k_stride}, std::pair{v, v_stride}})
      if (rows_overlap(q_out, q_out_stride * elem, static_cast<int64_t>(desc->n_heads) * d * elem, rows, stride * elem,
                       kv_bytes, T))
        return bad("q_out must not overlap rows of k or v");
  }
  StoreArgs a{};
  a.cache = cache_of(desc, cache);
  a.q = q;
  a.k = k;
  a.v = v;
  a.q_out = q_out;
  a.q_stride = q_stride;
  a.q_out_stride = q_out_stride;
  a.k_stride = k_stride;
  a.v_stride = v_stride;
  a.table = table;
  a.slots = slots;
  a.Hq = Hq;
  a.Hkv = desc->n_kv_heads;
  a.F = n_freq;
  a.T = T;
  const int per = 256 / (d / 8);
  const int64_t units = static_cast<int64_t>(T) * (Hq + 2 * desc->n_kv_heads);
  const unsigned grid = static_cast<unsigned>((units + per - 1) / per);
  const hipStream_t st = static_cast<hipStream_t>(hip_stream);
  return launched(dtype == SPP_DTYPE_BF16 ? launch_store<__bf16>(a, d, grid, st) : launch_store<float>(a, d, grid, st));
}

extern "C" spp_status spp_kv4_load(const spp_attn_desc* desc, const void* cache, int32_t dtype, const int64_t* slots,
                                   int32_t T, void* k_out, int64_t k_stride, void* v_out, int64_t v_stride,
                                   void* hip_stream) {
  SPP_BAD(desc_why(desc));
  SPP_BAD(dtype_why(dtype));
  const int d = desc->head_dim, elem = dtype == SPP_DTYPE_BF16 ? 2 : 4;
  if (T < 0 || static_cast<int64_t>(T) * 2 * desc->n_kv_heads > kMaxHeadRows)
    return bad("T must be >= 0, T * 2 n_kv_heads at most 2^27");
  if (T == 0 || (!k_out && !v_out)) return SPP_OK;
  if (!cache || !slots) return bad("cache and slots must not be NULL");
  if (!aligned16(cache) || !aligned(slots, 8)) return bad("cache must be 16-byte aligned, slots 8-byte aligned");
  if (k_out) SPP_BAD(rows_why(k_out, k_stride, desc->n_kv_heads, d, elem));
  if (v_out) SPP_BAD(rows_why(v_out, v_stride, desc->n_kv_heads, d, elem));
  const int64_t row_bytes = static_cast<int64_t>(desc->n_kv_heads) * d * elem;
  if (k_out && v_out && rows_overlap(k_out, k_stride * elem, row_bytes, v_out, v_stride * elem, row_bytes, T))
    return bad("k_out must not overlap rows of v_out");
  LoadArgs a{};
  a.cache = cache_of(desc, cache);
  a.slots = slots;
  a.k = k_out;
  a.v = v_out;
  a.k_stride = k_stride;
  a.v_stride = v_stride;
  a.Hkv = desc->n_kv_heads;
  a.T = T;
  const int per = 256 / (d / 8);
  const int64_t units = static_cast<int64_t>(T) * desc->n_kv_heads * (k_out && v_out ? 2 : 1);
  const unsigned grid = static_cast<unsigned>((units + per - 1) / per);
  const hipStream_t st = static_cast<hipStream_t>(hip_stream);
  return launched(dtype == SPP_DTYPE_BF16 ? launch_load<__bf16>(a, d, grid, st) : launch_load<float>(a, d, grid, st));
}

namespace {

const char* attend_why(const spp_attn_desc* desc, int32_t n_seq, int32_t max_q, int32_t max_kv) {
  if (const char* w = desc_why(desc)) return w;
  if (n_seq < 0 || max_q < 1 || max_kv < 0) return "n_seq and max_kv must be >= 0, max_q >= 1";
  if (static_cast<int64_t>(n_seq) * max_q * desc->n_heads > kMaxUnits) return "n_seq * max_q * n_heads must be at most 2^30";
  return nullptr;
}

}  // namespace

extern "C" size_t spp_kv4_attend_workspace(const spp_attn_desc* desc, int32_t n_seq, int32_t max_q, int32_t max_kv) {
  if (const char* w = attend_why(desc, n_seq, max_q, max_kv)) return bad(w), 0;
  // bounds of cut_of over every smaller size: a part for each item, and as many as fill the device
  size_t most = 16;
  const int64_t rows = static_cast<int64_t>(max_q) * (desc->n_heads / desc->n_kv_heads);
  if ((static_cast<int64_t>(max_kv) + kTile - 1) / kTile <= kMinTiles) return most;
  for (bool f32 : {false, true})
    for (int form = 0; form <= (rows <= 16 ? 0 : (rows <= kPairRows ? 1 : 2)); ++form) {
      const int d = desc->head_dim, each = group_rows(f32, d, form);
      const int64_t row_tiles = ((form == 2 ? rows : std::min<int64_t>(rows, kFewRows)) + each - 1) / each;
      const int64_t items = std::min<int64_t>(n_seq * desc->n_kv_heads * row_tiles, split_below(f32, d, form) - 1);
      const int64_t parts = std::max<int64_t>(fill(f32, d, form), items) + items;
      most = std::max(most, kCountBytes + static_cast<size_t>(parts) * each * (d + 2) * sizeof(float));
    }
  return most;
}

extern "C" spp_status spp_kv4_attend(const spp_attn_desc* desc, const void* cache, int32_t dtype, const void* q,
                                     int64_t q_stride, const int32_t* q_start, const int32_t* kv_len,
                                     const int32_t* pages, int64_t pages_stride, int32_t n_seq, int32_t n_tokens,
                                     int32_t max_q, int32_t max_kv, int32_t causal, float scale, void* out,
                                     int64_t out_stride, void* workspace, size_t workspace_bytes, void* hip_stream) {
  SPP_BAD(attend_why(desc, n_seq, max_q, max_kv));
  SPP_BAD(dtype_why(dtype));
  const int d = desc->head_dim, elem = dtype == SPP_DTYPE_BF16 ? 2 : 4;
  if (causal != 0 && causal != 1) return bad("causal must be 0 or 1");
  if (!(scale > 0.f) || !(scale <= 1e38f)) return bad("scale must be positive, at most 1e38");
  if (n_tokens < 0 || static_cast<int64_t>(n_tokens) * desc->n_heads > kMaxUnits)
    return bad("n_tokens must be >= 0, n_tokens * n_heads at most 2^30");
  if (!q_start && n_tokens != n_seq) return bad("without q_start every sequence has one query token: n_tokens must be n_seq");
  if (n_seq == 0 || n_tokens == 0) return SPP_OK;
  if (!cache || !q || !kv_len || !pages || !out) return bad("cache, q, kv_len, pages and out must not be NULL");
  if (!aligned16(cache) || !aligned(kv_len, 4) || !aligned(pages, 4) || !aligned(q_start, 4))
    return bad("cache must be 16-byte aligned, q_start, kv_len and pages aligned to their elements");
  if (pages_stride < 1 || pages_stride > INT32_MAX || pages_stride * desc->page > INT32_MAX - 1024)
    return bad("pages_stride must be at least 1, pages_stride * page below 2^31 - 1024");
  SPP_BAD(rows_why(q, q_stride, desc->n_heads, d, elem));
  SPP_BAD(rows_why(out, out_stride, desc->n_heads, d, elem));
  const bool same = q == out && q_stride == out_stride;
  if (!same && overlap(q, extent(q_stride, n_tokens, desc->n_heads, d, elem), out,
                       extent(out_stride, n_tokens, desc->n_heads, d, elem)))
    return bad("out must be q with the same stride, or not overlap it");
  if (!workspace || !aligned16(workspace)) return bad("workspace must not be NULL, and 16-byte aligned");
  const Cut cut = cut_of(desc, dtype == SPP_DTYPE_F32, n_seq, max_q, max_kv);
  if (attend_grid(cut, n_seq, desc->n_kv_heads) >= int64_t{1} << 22)
    return bad("too many sequences, heads and query tokens for one call");
  if (cut.units > 0 && workspace_bytes < kCountBytes + part_bytes(cut, n_seq, d)) return bad("the workspace is too small");
  AttendArgs a{};
  a.cache = cache_of(desc, cache);
  a.q = q;
  a.out = out;
  a.q_stride = q_stride;
  a.out_stride = out_stride;
  a.q_start = q_start;
  a.kv_len = kv_len;
  a.pages = pages;
  a.pages_stride = pages_stride;
  a.n_seq = n_seq;
  a.n_tokens = n_tokens;
  a.Hkv = desc->n_kv_heads;
  a.G = desc->n_heads / desc->n_kv_heads;
  const int64_t rows = static_cast<int64_t>(max_q) * a.G;
  a.max_rows = static_cast<int>(rows);  // at most 2^30
  a.causal = causal;
  a.scale_log2 = scale * 1.44269504088896340736f;
  a.planes = cut.planes;
  a.row_tiles = cut.row_tiles;
  a.units = cut.units;
  a.min_tiles = kMinTiles;
  a.join_apart = cut.join_apart;
  while (n_seq >> a.sum_shift > 16) ++a.sum_shift;  // a sequence has at most 2^26 tiles
  a.count = static_cast<unsigned*>(workspace);
  a.part = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + kCountBytes);
  const hipStream_t st = static_cast<hipStream_t>(hip_stream);
  return launched(dtype == SPP_DTYPE_BF16 ? launch_attend<__bf16>(a, d, cut, rows, st) : launch_attend<float>(a, d, cut, rows, st));
}
