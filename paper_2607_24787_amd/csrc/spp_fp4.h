// What the operators on explicit device pointers share: the microscaled 4-bit
// format (codes, scales and their conversions; spp.h has the contract), wide
// loads and stores of rows, and the host side's checks and launches.
#pragma once

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

constexpr uint32_t kExpMask = 0x7f800000u;
constexpr int kNanByte = 255;
constexpr int kMinByte = 2;    // scale 2^-125: every nonzero value of a block stays a normal number
constexpr int kMaxByte = 252;  // scale 2^125: 6 * 2^125 is the largest that is finite in bf16 and fp32

__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }

// The scale byte of a block by its largest magnitude's bits: the smallest with
// no magnitude above 7 * 2^(byte - 127); an infinity or a NaN gives kNanByte.
// top = 1.m * 2^(E-127) <= 7 * 2^e = 1.75 * 2^(e+2)
__device__ __forceinline__ uint32_t byte_of(uint32_t top) {
  if (top >= kExpMask) return kNanByte;
  const int E = static_cast<int>(top >> 23);
  const int s = (top & 0x7fffffu) <= 0x600000u ? E - 2 : E - 1;
  return static_cast<uint32_t>(min(max(s, kMinByte), kMaxByte));
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

// Codes (one word) and scale byte of this lane's 8 elements of a block of 32,
// which lanes 4j .. 4j+3 hold together.
__device__ __forceinline__ uint32_t quantise8(const float* y, uint32_t* byte) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(y[i]) & 0x7fffffffu);  // ordered as the magnitudes are; NaN above infinity
  top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), 1)));
  top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), 2)));
  *byte = byte_of(top);
  if (*byte == kNanByte) return 0u;
  const float scale = scale_of(*byte);
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[0], y[1], scale, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[2], y[3], scale, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[4], y[5], scale, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[6], y[7], scale, 3);
  return w;
}

// ------------------------------------------------------------------ host side

bool aligned(const void* p, unsigned n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

spp_status bad(const char* why) { return spp::set_error(SPP_EINVAL, why); }

bool overlap(const void* a, uint64_t na, const void* b, uint64_t nb) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x < y + nb && y < x + na;
}

// `count` rows of `bytes` each, `stride` bytes apart (at least a row); an array is one row
struct Rows {
  const void* at;
  int64_t bytes, stride, count;
};

Rows array(const void* p, int64_t bytes) { return {p, bytes, bytes, 1}; }
Rows rows_from(const void* p, int64_t stride, int64_t row, int64_t count, int elem) { return {p, row * elem, stride * elem, count}; }

// Whether they have a byte in common.  Column ranges of one buffer lie between
// each other without.
bool meet(Rows a, Rows b) {
  if (!a.at || !b.at || a.count < 1 || b.count < 1 || a.bytes < 1 || b.bytes < 1) return false;
  if (a.count < b.count) std::swap(a, b);
  if (!overlap(a.at, static_cast<uint64_t>((a.count - 1) * a.stride + a.bytes), b.at,
               static_cast<uint64_t>((b.count - 1) * b.stride + b.bytes)))
    return false;
  const int64_t off = static_cast<int64_t>(reinterpret_cast<uintptr_t>(b.at) - reinterpret_cast<uintptr_t>(a.at));
  const auto below = [](int64_t x, int64_t y) { return x / y - (x % y < 0); };  // floor(x / y)
  // rows of a, before the first and behind the last too, from the first that ends past row u of b to the last that
  // starts before its end
  const auto first = [&](int64_t u) { return below(off + u * b.stride - a.bytes, a.stride) + 1; };
  const auto last = [&](int64_t u) { return below(off + u * b.stride + b.bytes - 1, a.stride); };
  if (a.stride == b.stride) {  // row u meets the rows that row 0 meets, u further on
    const int64_t f = first(0), l = last(0);
    return f <= l && std::max<int64_t>(0, -l) <= std::min<int64_t>(b.count - 1, a.count - 1 - f);
  }
  for (int64_t u = 0; u < b.count; ++u)
    if (std::max<int64_t>(0, first(u)) <= std::min<int64_t>(a.count - 1, last(u))) return true;
  return false;
}

const char* rows_why(const void* p, int64_t stride, int64_t row, int elem) {
  if (!p) return "a pointer to rows is NULL";
  if (stride < row || stride > int64_t{1} << 30) return "a row stride must be at least a row, at most 2^30 elements";
  if (!aligned16(p) || stride * elem % 16 != 0) return "rows must be 16-byte aligned, their stride a multiple of 16 bytes";
  return nullptr;
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

}  // namespace
