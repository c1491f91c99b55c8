// What the paged-cache calls share: types of stored elements and the host's checks of a cache.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "common.hpp"
#include "lilicorr.h"

namespace lilicorr {

typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2_t __attribute__((ext_vector_type(2)));

// A 16-bit type of the cache: how two of its elements become floats and come from them (nearest,
// ties to even)
struct Bf16 {
  typedef __bf16 elem;
  static __device__ __forceinline__ f32x2_t unpack(uint32_t w) {
    return f32x2_t{__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)};
  }
  static __device__ __forceinline__ uint32_t pack(float a, float b) {
    typedef __bf16 pair __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2_t{a, b}), pair));
  }
  // nonzero if one of the two is infinite or NaN
  static __device__ __forceinline__ uint32_t nonfinite(uint32_t w) {
    return (uint32_t)((w & 0x7f80u) == 0x7f80u) | (uint32_t)((w & 0x7f800000u) == 0x7f800000u);
  }
};

struct F16 {
  typedef _Float16 elem;
  static __device__ __forceinline__ f32x2_t unpack(uint32_t w) {
    typedef _Float16 pair __attribute__((ext_vector_type(2)));
    return __builtin_convertvector(__builtin_bit_cast(pair, w), f32x2_t);
  }
  static __device__ __forceinline__ uint32_t pack(float a, float b) {
    typedef _Float16 pair __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2_t{a, b}), pair));
  }
  static __device__ __forceinline__ uint32_t nonfinite(uint32_t w) {
    return (uint32_t)((w & 0x7c00u) == 0x7c00u) | (uint32_t)((w & 0x7c000000u) == 0x7c000000u);
  }
};

inline bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }
inline bool aligned8(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 7u) == 0; }
// whether two stretches of memory have a byte in common
inline bool overlap(const void* a, size_t a_bytes, const void* b, size_t b_bytes) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x < y ? a_bytes > y - x && b_bytes > 0 : b_bytes > x - y && a_bytes > 0;
}
// whether one of `rows` rows, `stride` bytes apart, has a byte in common with a stretch of memory
inline bool rows_overlap(const void* a, int64_t stride, size_t row_bytes, int64_t rows, const void* b,
                         size_t b_bytes) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  // the first row that ends past the stretch's beginning
  const uint64_t first = x + row_bytes > y ? 0 : stride ? (y - x - row_bytes) / (uint64_t)stride + 1 : (uint64_t)rows;
  return first < (uint64_t)rows && x + first * (uint64_t)stride < y + b_bytes;
}
inline bool stride_ok(int64_t s) { return s >= 0 && s % 8 == 0 && s < ((int64_t)1 << 40); }

// sizes of a cache, without its pointers
inline lilicorr_status cache_sizes(const lilicorr_cache& c) {
  if (c.dtype != LILICORR_BF16 && c.dtype != LILICORR_F16) return LILICORR_ERR_INVALID_ARG;
  if (c.page_size < 1 || c.heads < 1 || c.d < 1 || c.pages < 1) return LILICORR_ERR_INVALID_ARG;
  if (c.page_stride < 0 || c.token_stride < 0 || c.head_stride < 0)
    return LILICORR_ERR_INVALID_ARG;
  if (c.d % 8 || c.d < 16 || c.d > 256 || c.page_size > 65536 || c.heads > 65535)
    return LILICORR_ERR_UNSUPPORTED;
  if (c.pages > 0x7fffffffll / c.page_size) return LILICORR_ERR_UNSUPPORTED;
  if (!stride_ok(c.page_stride) || !stride_ok(c.token_stride) || !stride_ok(c.head_stride))
    return LILICORR_ERR_ALIGNMENT;
  return LILICORR_OK;
}

}  // namespace lilicorr
