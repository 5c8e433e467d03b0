// Matrices in microscaled 4 bits: quantisation, products with them, and an MoE
// layer's routed experts on them.  The calls' contracts and the format are in
// spp.h.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <cstring>
#include <type_traits>

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

// A lane takes 8 elements, four lanes a block.
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
enum { kXBf16 = 0, kXCodes = 1, kXQuantBf16 = 2, kXQuantF32 = 3 };
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
  const int32_t* start;
  int M, groups;
  const int32_t* ids;             // kRowsIds: [M]
  const int32_t* pair;            // row i of a group is row pair[i] / xdiv of x (NULL: i / xdiv)
  int xdiv;
  int by_pair;                    // kRowsIds: blockIdx.y is a pair, and the first with its id takes the group
  void* out;
  int64_t out_stride;             // elements
};

// Scale bytes [at, at + 4) as one word, of `total` bytes; those past the end do
// not count.
__device__ __forceinline__ uint32_t scales4(const uint8_t* p, int64_t at, int64_t total) {
  if (total < 4) {
    uint32_t w = 0;
    for (int j = 0; j < 4; ++j)
      if (at + j < total) w |= static_cast<uint32_t>(p[at + j]) << (8 * j);
    return w;
  }
  const int64_t o = min(at, total - 4);
  uint32_t w;
  __builtin_memcpy(&w, p + o, 4);
  return w >> (8 * static_cast<int>(at - o));
}

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

// Block b of row x (or nothing): bf16 rows as four operands of 8 elements, rows
// in 4 bits as codes in v[0] with their scale byte
template <int X>
__device__ __forceinline__ void x_block(const ProductArgs& a, int64_t row, int b, bool ok, u32x4* v, uint32_t* byte) {
  *byte = kOne;
#pragma unroll
  for (int q = 0; q < 4; ++q) v[q] = u32x4{0, 0, 0, 0};
  if (!ok) return;
  const uint8_t* p = static_cast<const uint8_t*>(a.x) + row * a.x_stride;
  if constexpr (X == kXCodes) {
    v[0] = reinterpret_cast<const u32x4*>(p)[b];
    *byte = a.x_scales[row * a.nb + b];
  } else if constexpr (X == kXQuantF32) {
    float y[32];
#pragma unroll
    for (int q = 0; q < 4; ++q) load8(reinterpret_cast<const float*>(p) + 32 * b + 8 * q, y + 8 * q);
    v[0] = quantise32(y, byte);
  } else if constexpr (X == kXQuantBf16) {
    float y[32];
#pragma unroll
    for (int q = 0; q < 4; ++q) load8(reinterpret_cast<const __bf16*>(p) + 32 * b + 8 * q, y + 8 * q);
    v[0] = quantise32(y, byte);
  } else {
#pragma unroll
    for (int q = 0; q < 4; ++q) v[q] = reinterpret_cast<const u32x4*>(p)[4 * b + q];
  }
}

template <int SEL>
__device__ __forceinline__ f32x4 mfma_mx4(u32x4 w, uint32_t w_scales, u32x4 x, uint32_t x_byte, f32x4 c) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wide(w), wide(x), c, 4, 4, SEL, static_cast<int>(w_scales), 0,
                                                          static_cast<int>(x_byte));
}

__device__ __forceinline__ float swiglu(float g, float u) { return g / (1.f + expf(-g)) * u; }

// Byte s of w, or 1's
__device__ __forceinline__ uint32_t byte_or_one(uint32_t w, int s, bool ok) { return ok ? (w >> (8 * s)) & 255u : kOne; }

constexpr int kFewThreads = 256;
constexpr int kFewWaves = kFewThreads / 64;
constexpr int kStep = 4;  // blocks of a lane whose loads are in flight together

// The sums of one wave's share of K for 16 weight rows (times kTiles) and 16
// rows of x.  Lane l holds weight row and row of x l % 16; lanes 16g .. 16g+15
// of wave w own blocks (4w + g) * per and on, of both: what the matrix
// instruction sums over goes by lane and place, whatever the blocks' order in K.
template <int X, int kTiles>
__device__ __forceinline__ void few_sums(const ProductArgs& a, const int64_t* row, int64_t x_row, bool x_ok, int b0, int b1,
                                         int per, f32x4* acc) {
  for (int s0 = 0; s0 < per; s0 += kStep) {
    u32x4 w[kTiles][kStep];
    uint32_t ws[kTiles];
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
      ws[t] = scales4(a.scales, row[t] * a.nb + min(b0 + s0, a.nb - 1), a.blocks);
#pragma unroll
      for (int s = 0; s < kStep; ++s) {
        const int b = b0 + s0 + s;
        w[t][s] = reinterpret_cast<const u32x4*>(a.codes)[row[t] * a.nb + (b < b1 ? b : 0)];
      }
    }
#pragma unroll
    for (int s = 0; s < kStep; ++s) {
      const bool ok = b0 + s0 + s < b1;
      u32x4 v[4];
      uint32_t byte;
      x_block<X>(a, x_row, b0 + s0 + s, ok && x_ok, v, &byte);
#pragma unroll
      for (int t = 0; t < kTiles; ++t) {
        const uint32_t wb = byte_or_one(ws[t], s, ok);
        if constexpr (X == kXBf16) {
#pragma unroll
          for (int q = 0; q < 4; ++q) acc[t] = mfma_bf16(cvt8(w[t][s][q], scale_of(wb)), v[q], acc[t]);
        } else {
          acc[t] = mfma_mx4<0>(w[t][s], wb, v[0], byte, acc[t]);
        }
      }
    }
  }
}

// A workgroup takes 16 outputs (of both matrices for SwiGLU) of one group for
// 16 of its rows at a time; its waves share K.
template <int X, bool kSwiglu, typename Out, int kRows>
__global__ __launch_bounds__(kFewThreads) void mx4_few_kernel(ProductArgs a) {
  constexpr int kTiles = kSwiglu ? 2 : 1;
  __shared__ f32x4 s_part[kFewWaves][kTiles][64];
  __shared__ int s_row[16];
  __shared__ int s_count;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, g = lane >> 4, l16 = lane & 15;
  int group = blockIdx.y, begin = 0, count = 0;
  if constexpr (kRows == kRowsIds) {
    if (a.by_pair) {
      group = a.ids[blockIdx.y];
      if (static_cast<unsigned>(group) >= static_cast<unsigned>(a.groups)) return;
      bool earlier = false;
      for (int p = lane; p < static_cast<int>(blockIdx.y); p += 64) earlier |= a.ids[p] == group;
      if (__ballot(earlier)) return;
    }
  } else {
    count = a.M;
    if (a.start) {
      begin = min(max(a.start[group], 0), a.M);
      count = min(max(a.start[group + 1], 0), a.M) - begin;
    }
    if (count <= 0) return;
  }
  const int per = (a.nb + 4 * kFewWaves - 1) / (4 * kFewWaves);
  const int b0 = (wave * 4 + g) * per, b1 = min(b0 + per, a.nb);
  const int f0 = blockIdx.x * 16;
  int64_t row[kTiles];
#pragma unroll
  for (int t = 0; t < kTiles; ++t)
    row[t] = (static_cast<int64_t>(group) * kTiles + t) * a.N + min(f0 + l16, a.N - 1);
  for (int r0 = 0;; r0 += 16) {
    if constexpr (kRows == kRowsIds) {
      if (wave == 0) {
        int seen = 0;
        for (int p0 = 0; p0 < a.M; p0 += 64) {
          const bool mine = p0 + lane < a.M && a.ids[p0 + lane] == group;
          const uint64_t m = __ballot(mine);
          const int at = seen + __popcll(m & ((uint64_t{1} << lane) - 1)) - r0;
          if (mine && at >= 0 && at < 16) s_row[at] = p0 + lane;
          seen += __popcll(m);
        }
        if (lane == 0) s_count = seen;
      }
      __syncthreads();
      count = s_count;
      if (r0 >= count) return;
    } else {
      if (tid < 16) s_row[tid] = begin + min(r0 + tid, count - 1);
      __syncthreads();
    }
    const bool x_ok = r0 + l16 < count;
    int64_t x_row = 0;
    if (x_ok) {
      const int i = s_row[l16];
      const int p = a.pair ? a.pair[i] : i;
      x_row = p / a.xdiv;
    }
    f32x4 acc[kTiles];
#pragma unroll
    for (int t = 0; t < kTiles; ++t) acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
    few_sums<X, kTiles>(a, row, x_row, x_ok, b0, b1, per, acc);
    // outputs 4g .. 4g+3 of row l16
#pragma unroll
    for (int t = 0; t < kTiles; ++t) s_part[wave][t][l16 * 4 + g] = acc[t];
    __syncthreads();
    const int i = tid >> 4, f = f0 + (tid & 15);
    float v[kTiles];
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
      v[t] = 0.f;
      for (int w = 0; w < kFewWaves; ++w) v[t] += reinterpret_cast<const float*>(s_part[w][t])[tid];
    }
    if (r0 + i < count && f < a.N) {
      float y = v[0];
      if constexpr (kSwiglu) y = swiglu(v[0], v[1]);
      static_cast<Out*>(a.out)[s_row[i] * a.out_stride + f] = static_cast<Out>(y);
    }
    if (r0 + 16 >= count) return;
    __syncthreads();
  }
}

// ------------------------------------------------------------------ host side

const char* rows_why(const void* p, int64_t stride, int64_t row, int elem) {
  if (!p) return "a pointer to rows is NULL";
  if (stride < row || stride > int64_t{1} << 30) return "a row stride must be at least a row, at most 2^30 elements";
  if (!aligned16(p) || stride * elem % 16 != 0) return "rows must be 16-byte aligned, their stride a multiple of 16 bytes";
  return nullptr;
}

// The end of rows as bytes from their start
uint64_t span(int64_t rows, int64_t stride, int64_t row, int elem) {
  return rows < 1 ? 0 : static_cast<uint64_t>((rows - 1) * stride + row) * static_cast<uint64_t>(elem);
}

const char* matrix_why(const spp_mx4_matrix* m) {
  if (!m) return "a matrix is NULL";
  if (m->cols < 32 || m->cols > 1 << 17 || m->cols % 32 != 0) return "cols must be a multiple of 32, at most 2^17";
  if (m->rows < 0 || m->rows > INT32_MAX || m->rows * m->cols > int64_t{1} << 40)
    return "rows must be in [0, 2^31), and rows * cols at most 2^40";
  if (m->rows > 0 && (!m->codes || !m->scales)) return "codes and scales must not be NULL";
  if (!aligned16(m->codes)) return "codes must be 16-byte aligned";
  return nullptr;
}

uint64_t code_bytes(const spp_mx4_matrix& m) { return static_cast<uint64_t>(m.rows) * (m.cols / 2); }
uint64_t scale_bytes(const spp_mx4_matrix& m) { return static_cast<uint64_t>(m.rows) * (m.cols / 32); }

bool over(const spp_mx4_matrix& m, const void* p, uint64_t bytes) {
  return overlap(m.codes, code_bytes(m), p, bytes) || overlap(m.scales, scale_bytes(m), p, bytes);
}

unsigned quant_grid(int64_t words) {
  return static_cast<unsigned>(std::min<int64_t>((words + kQuantThreads - 1) / kQuantThreads, 1 << 20));
}

hipError_t launch2(void (*kernel)(ProductArgs), unsigned x, unsigned y, unsigned threads, const ProductArgs& a,
                   hipStream_t st) {
  void* params[] = {const_cast<ProductArgs*>(&a)};
  return hipLaunchKernel(reinterpret_cast<const void*>(kernel), dim3(x, y), dim3(threads), params, 0, st);
}

constexpr int kMaxM = 1 << 24;
constexpr int kMaxN = 1 << 20;

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
  if (M == 0) return nullptr;
  const int64_t N = w->rows / groups;
  if (!out || !aligned(out, dtype == SPP_DTYPE_BF16 ? 2 : 4)) return "out must not be NULL, and aligned to its elements";
  if (out_stride < N || out_stride > int64_t{1} << 30) return "out's stride must be at least a row, at most 2^30 elements";
  const uint64_t bytes = span(M, out_stride, N, dtype == SPP_DTYPE_BF16 ? 2 : 4);
  if (over(*w, out, bytes) || (start && overlap(start, static_cast<uint64_t>(groups + 1) * 4, out, bytes)))
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

unsigned tiles16(int N) { return static_cast<unsigned>((N + 15) / 16); }

template <int X>
hipError_t launch_product(const ProductArgs& a, int32_t dtype, hipStream_t st) {
  const auto kernel = dtype == SPP_DTYPE_BF16 ? mx4_few_kernel<X, false, __bf16, kRowsStart>
                                              : mx4_few_kernel<X, false, float, kRowsStart>;
  return launch2(kernel, tiles16(a.N), static_cast<unsigned>(a.groups), kFewThreads, a, st);
}

// The parts of a workspace of the experts' call
struct Space {
  size_t h, y, bytes;
};

size_t up256(size_t n) { return (n + 255) & ~size_t{255}; }

Space space_of(int64_t P, int32_t D, int32_t I) {
  Space s{};
  s.h = 0;
  s.y = up256(static_cast<size_t>(P) * I * 4);
  s.bytes = s.y + up256(static_cast<size_t>(P) * D * 4);
  return s;
}

const char* experts_why(int32_t n, int32_t D, int32_t I, int32_t T, int32_t K) {
  if (n < 1 || n > spp::kMaxExpertsTopK) return "n must be in [1, 1024]";
  if (K < 1 || K > 64) return "K must be in [1, 64]";
  if (T < 0 || static_cast<int64_t>(T) * K > kMaxM) return "T must be >= 0, and T * K at most 2^24";
  if (D < 32 || D % 32 != 0 || D > 1 << 17 || I < 32 || I % 32 != 0 || I > 1 << 17)
    return "D and I must be multiples of 32, at most 2^17";
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
  if (over(*q, x, span(q->rows, x_stride, q->cols, elem)) || overlap(q->codes, code_bytes(*q), q->scales, scale_bytes(*q)))
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
  if (over(*q, out, span(q->rows, out_stride, q->cols, elem))) return bad("out must not overlap codes or scales");
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
  const uint64_t bytes = span(M, out_stride, w->rows / groups, dtype == SPP_DTYPE_BF16 ? 2 : 4);
  if (overlap(x, span(M, x_stride, w->cols, 2), out, bytes)) return bad("out must not overlap an input");
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
  const uint64_t bytes = span(M, out_stride, w->rows / groups, dtype == SPP_DTYPE_BF16 ? 2 : 4);
  if (over(*x, out, bytes)) return bad("out must not overlap an input");
  ProductArgs a = product_of(*w, groups, start, M, out, out_stride);
  a.x = x->codes;
  a.x_stride = x->cols / 2;
  a.x_scales = static_cast<const uint8_t*>(x->scales);
  return launched(launch_product<kXCodes>(a, dtype, static_cast<hipStream_t>(hip_stream)));
}

extern "C" size_t spp_mx4_experts_workspace(int32_t n, int32_t D, int32_t I, int32_t T, int32_t K) {
  if (const char* w = experts_why(n, D, I, T, K)) return bad(w), 0;
  return std::max<size_t>(16, space_of(static_cast<int64_t>(T) * K, D, I).bytes);
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
  const uint64_t out_bytes = span(T, out_stride, D, 2), each = static_cast<uint64_t>(P) * 4;
  if (overlap(x, span(T, x_stride, D, 2), out, out_bytes) || overlap(topk, each, out, out_bytes) ||
      overlap(gates, each, out, out_bytes) || over(*gate_up, out, out_bytes) || over(*down, out, out_bytes))
    return bad("out must not overlap an input");
  if (residual) {
    SPP_BAD(rows_why(residual, residual_stride, D, 2));
    if (!(residual == out && residual_stride == out_stride) &&
        overlap(residual, span(T, residual_stride, D, 2), out, out_bytes))
      return bad("out must be residual with the same stride, or not overlap it");
  }
  const Space s = space_of(P, D, I);
  if (!workspace || !aligned16(workspace)) return bad("workspace must not be NULL, and 16-byte aligned");
  if (workspace_bytes < s.bytes) return bad("the workspace is too small");
  const hipStream_t st = static_cast<hipStream_t>(hip_stream);
  uint8_t* space = static_cast<uint8_t*>(workspace);
  const bool mx4 = act == SPP_ACT_MX4;

  ProductArgs a = product_of(*gate_up, n, nullptr, static_cast<int32_t>(P), space + s.h, I);
  a.N = I;
  a.x = x;
  a.x_stride = x_stride * 2;
  a.ids = topk;
  a.xdiv = K;
  a.by_pair = P < n;
  const unsigned groups = static_cast<unsigned>(std::min<int64_t>(P, n));
  hipError_t e = launch2(mx4 ? mx4_few_kernel<kXQuantBf16, true, float, kRowsIds>
                             : mx4_few_kernel<kXBf16, true, __bf16, kRowsIds>,
                         tiles16(I), groups, kFewThreads, a, st);
  if (e != hipSuccess) return launched(e);
  ProductArgs d = product_of(*down, n, nullptr, static_cast<int32_t>(P), space + s.y, D);
  d.x = space + s.h;
  d.x_stride = static_cast<int64_t>(I) * (mx4 ? 4 : 2);
  d.ids = topk;
  d.by_pair = P < n;
  e = launch2(mx4 ? mx4_few_kernel<kXQuantF32, false, float, kRowsIds> : mx4_few_kernel<kXBf16, false, float, kRowsIds>,
              tiles16(D), groups, kFewThreads, d, st);
  if (e != hipSuccess) return launched(e);
  spp::ExpertSum c{};
  c.rows = space + s.y;
  c.rows_stride = D;
  c.ids = topk;
  c.weights = gates;
  c.n = n;
  c.dtype = SPP_DTYPE_BF16;
  c.fp32_rows = 1;
  c.T = T;
  c.K = K;
  c.D = D;
  c.residual = residual;
  c.residual_stride = residual_stride;
  c.out = out;
  c.out_stride = out_stride;
  return launched(spp::launch_expert_combine(c, st));
}
