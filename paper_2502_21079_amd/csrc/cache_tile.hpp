// Building blocks of the 8-bit cache's kernels: conversions, pages.
#pragma once

#include "cache.hpp"
#include "cross_tile.hpp"

namespace adaspa {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

// Two codes (the lower or the upper two bytes of w) times a power of two, as two
// 16-bit values: e4m3 has 4 significant bits, so this is exact.
template <class T, bool UPPER>
__device__ __forceinline__ uint32_t decode2(uint32_t w, float scale) {
  if constexpr (T::kHalf) return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, scale, UPPER));
  else return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, UPPER));
}
// Eight codes.
template <class T>
__device__ __forceinline__ typename T::x8 decode8(uint32_t a, uint32_t b, float scale) {
  const u32x4 r = {decode2<T, false>(a, scale), decode2<T, true>(a, scale), decode2<T, false>(b, scale),
                   decode2<T, true>(b, scale)};
  return __builtin_bit_cast(typename T::x8, r);
}
// Four values, to the nearest code, ties to even.  |x| <= 448, or infinities and NaN,
// which get the code that stands for no number.
__device__ __forceinline__ uint32_t encode4(float a, float b, float c, float d) {
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false), true);
}
__device__ __forceinline__ void decode4(uint32_t w, float (&f)[4]) {
  const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
  f[0] = lo[0];
  f[1] = lo[1];
  f[2] = hi[0];
  f[3] = hi[1];
}
// Codes of one scale as codes of another, `by` the old over the new one.
__device__ __forceinline__ uint32_t recode4(uint32_t w, float by) {
  float f[4];
  decode4(w, f);
  return encode4(f[0] * by, f[1] * by, f[2] * by, f[3] * by);
}

// The least power of two s >= 2^-126 with amax <= 448 s (448 = 1.75 * 2^8 is the
// largest code).
__device__ __forceinline__ float scale_for(float amax) {
  const uint32_t u = __float_as_uint(amax);
  const int e = (int)(u >> 23) - 8 + ((u & 0x7FFFFFu) > 0x600000u);
  return __uint_as_float((uint32_t)(e < 1 ? 1 : e) << 23);
}

// Bytes [0, n) of a word.
__device__ __forceinline__ uint32_t first_bytes(int n) { return n >= 4 ? ~0u : (n <= 0 ? 0u : (1u << (8 * n)) - 1); }

// The page of sequence b that holds position pos, -1 if the table names none of
// the pool there.
__device__ __forceinline__ int page_at(const CachePool& c, int b, int page_index) {
  if (page_index >= c.max_pages) return -1;
  const int id = c.table[b * c.table_stride + page_index];
  return (uint32_t)id < (uint32_t)c.pages ? id : -1;
}
__device__ __forceinline__ int clamp_len(int n, int most) { return n < 0 ? 0 : (n < most ? n : most); }

}  // namespace adaspa
