// The 4-bit paged cache: its elements, how the kernels convert them, the host's checks.
//
// An element is E2M1: a sign and 0, 0.5, 1, 1.5, 2, 3, 4 or 6, two to a byte, the even element low. 32 neighbouring
// elements of a head share a byte b for the scale 2^(b - 127), and b = 255 says that the block is NaN (the conversion reads
// it so). 0, 253 and 254 are not written (6 * 2^126 and 6 * 2^127 are no bf16 values) and have no meaning.
// Every other block's elements are bf16 values, so they go to the matrix cores without an error.
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "common.hpp"
#include "lilicorr.h"
#include "paged.hpp"

namespace lilicorr {

typedef float f32x4_t __attribute__((ext_vector_type(4)));

constexpr int kBlock4 = 32;          // elements that share a scale
constexpr uint32_t kLeastScale = 1;  // 2^-126
constexpr uint32_t kMostScale = 252; // 2^125
constexpr uint32_t kNanScale = 255;

// elements 2 BYTE and 2 BYTE + 1 of the eight in w, times the scale, as two bf16 (exact)
template <int BYTE>
__device__ __forceinline__ uint32_t from4(uint32_t w, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, BYTE));
}

__device__ __forceinline__ float scale_of(uint32_t b) { return __uint_as_float(b << 23); }

__device__ __forceinline__ f32x4_t mfma16(const u32x4_t& a, const u32x4_t& b, const f32x4_t& c) {
  typedef __bf16 x8 __attribute__((ext_vector_type(8)));
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(x8, a), __builtin_bit_cast(x8, b), c, 0, 0, 0);
}

// An operand of eight 16-bit query elements in bf16: exact, as one term for bf16 and as two for fp16, whose 11
// significant bits are the leading 8 and the 3 that are left.
template <typename T>
struct Query;
template <>
struct Query<Bf16> {
  static constexpr int kTerms = 1;
  static __device__ __forceinline__ void split(const u32x4_t& w, u32x4_t (&to)[1]) { to[0] = w; }
};
template <>
struct Query<F16> {
  static constexpr int kTerms = 2;
  static __device__ __forceinline__ void split(const u32x4_t& w, u32x4_t (&to)[2]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t x = w[i];
      const f32x2_t v = F16::unpack(x);
      const uint32_t hi = Bf16::pack(v[0], v[1]);
      const f32x2_t h = Bf16::unpack(hi);
      // an infinity stays in the leading term alone
      const float r0 = v[0] == h[0] ? 0.f : v[0] - h[0], r1 = v[1] == h[1] ? 0.f : v[1] - h[1];
      to[0][i] = hi;
      to[1][i] = Bf16::pack(r0, r1);
    }
  }
};

// the sum, and the largest, over the four lanes l, l ^ 16, l ^ 32, l ^ 48
__device__ __forceinline__ float quad_sum(float v) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}
__device__ __forceinline__ float quad_max(float v) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// The reference m of a row's powers 2^(x s - m), x a score and s the scale: a whole number that follows the largest score
// when that has grown by more than 2^8, and -inf before the first one. A tile in which one has grown is done again after the
// growth, so a growth has to end that whatever the score. In the difference the product x s is not rounded, and where m
// comes from it it is: up to 2^24 the two are less than two apart, from 2^28 on rounding alone can make up more
// than 2^8, for good. So from 2^24 on (`far4`) scores are multiplied and rounded first, as m was, and then s is 1.
constexpr float kRescale4 = 8.f;
constexpr float kFar4 = 0x1p24f;
__host__ __device__ inline float scaled4(float x, float s) {
#pragma clang fp contract(off)
  return x * s;
}
__host__ __device__ inline bool grown4(float x, float s, float m) {
  return fmaf(x, s, -m) > kRescale4;  // -inf - -inf is NaN and does not count
}
// (finite below, where -inf would stay -inf)
__host__ __device__ inline float reference4(float x, float s) { return floorf(fmaxf(scaled4(x, s), -__FLT_MAX__)); }
__host__ __device__ inline bool far4(float m) { return fabsf(m) >= kFar4 && m != -__builtin_inff(); }

// bits at and above n, and below it, of 32 (any n)
__device__ __forceinline__ uint32_t bits32_from(int n) { return n <= 0 ? ~0u : n >= 32 ? 0 : ~0u << n; }
__device__ __forceinline__ uint32_t bits32_below(int n) { return ~bits32_from(n); }

// Workgroup b, which runs on XCD b % 8, as an item, where `together` items in a row share cache lines: they come one after
// the other on one XCD, so that they find the lines in its L2, and what follows goes round the XCDs.
__device__ __forceinline__ int beside(int b, int items, int together) {
  const int whole = items / together / 8 * 8 * together;
  if (b >= whole) return b;
  const int q = b / 8;
  return (q / together * 8 + b % 8) * together + q % together;
}

// How many of a thread's loads of page numbers, and then of weights, the eviction has under way at a time
constexpr int loads_at_once(int slots) { return slots < 8 ? slots : 8; }

// ---- host ------------------------------------------------------------------------------------------
inline bool stride4_ok(int64_t s) { return s % 16 == 0 && s < ((int64_t)1 << 40); }

// sizes of a 4-bit cache, without its pointers
inline lilicorr_status cache4_sizes(const lilicorr_cache4& c) {
  if (c.page_size < 1 || c.heads < 1 || c.d < 1 || c.pages < 1) return LILICORR_ERR_INVALID_ARG;
  if (c.page_stride < 0 || c.token_stride < 0 || c.head_stride < 0) return LILICORR_ERR_INVALID_ARG;
  if (c.d % kBlock4 || c.d > 256 || c.page_size > 65536 || c.heads > 65535) return LILICORR_ERR_UNSUPPORTED;
  if (c.pages > 0x7fffffffll / c.page_size) return LILICORR_ERR_UNSUPPORTED;
  if (!stride4_ok(c.page_stride) || !stride4_ok(c.token_stride) || !stride4_ok(c.head_stride))
    return LILICORR_ERR_ALIGNMENT;
  return LILICORR_OK;
}

// bytes from the cache's first to behind its last code, and scale (a sixteenth of a code's offset, and d / 32)
inline size_t cache4_span(const lilicorr_cache4& c) {
  return (size_t)(c.page_stride * (c.pages - 1) + c.token_stride * (c.page_size - 1) + c.head_stride * (c.heads - 1)) +
         (size_t)c.d / 2;
}
inline size_t cache4_scales(size_t span) { return span / 16; }

// the multiplier and shift of n / P = (n * mul) >> shift for n < 2^31, mul = floor(2^shift / P) + 1 below 2^32
inline void divide_by(int P, uint32_t& mul, uint32_t& shift) {
  int bits = 0;
  while ((1 << bits) < P) ++bits;
  shift = 31 + bits;
  mul = (uint32_t)((((uint64_t)1 << shift) / P) + 1);
}

}  // namespace lilicorr
