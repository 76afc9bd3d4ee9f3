// Eight neighbouring elements of a row: what the kernels that pass over rows load, compute and store at a time.
#pragma once
#include "tile_loads.h"

namespace scd {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x8 __attribute__((ext_vector_type(8)));

__device__ __forceinline__ f32x8 widen(u32x4 v) { return __builtin_convertvector(__builtin_bit_cast(bf16x8, v), f32x8); }
__device__ __forceinline__ u32x4 narrow(f32x8 v) { return __builtin_bit_cast(u32x4, __builtin_convertvector(v, bf16x8)); }

// As they lie in memory, bf16 or fp32: loaded at once, widened where they are used.
template <bool F32>
struct Eight;
template <>
struct Eight<false> {
  u32x4 v;
  __device__ __forceinline__ f32x8 wide() const { return widen(v); }
};
template <>
struct Eight<true> {
  f32x4 a, b;
  __device__ __forceinline__ f32x8 wide() const { return f32x8{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w}; }
};
// piece `at` (of eight elements) of an array that is aligned to 16 bytes
template <bool F32>
__device__ __forceinline__ Eight<F32> load_eight(const void* p, int64_t at) {
  if constexpr (F32) {
    const f32x4* const q = static_cast<const f32x4*>(p) + 2 * at;
    return {q[0], q[1]};
  } else {
    return {static_cast<const u32x4*>(p)[at]};
  }
}
template <bool F32>
__device__ __forceinline__ void store_eight(void* p, int64_t at, f32x8 v) {
  if constexpr (F32) {
    f32x4* const q = static_cast<f32x4*>(p) + 2 * at;
    q[0] = f32x4{v[0], v[1], v[2], v[3]};
    q[1] = f32x4{v[4], v[5], v[6], v[7]};
  } else {
    static_cast<u32x4*>(p)[at] = narrow(v);
  }
}
// the same where the type is known at run time only (alike for all lanes)
__device__ __forceinline__ f32x8 eight_of(bool f32, const void* p, int64_t at) {
  return f32 ? load_eight<true>(p, at).wide() : load_eight<false>(p, at).wide();
}
__device__ __forceinline__ void put_eight(bool f32, void* p, int64_t at, f32x8 v) {
  if (f32) store_eight<true>(p, at, v);
  else store_eight<false>(p, at, v);
}

// ---- e4m3 numbers under a scale for each 128 --------------------------------------------------------
// scale = largest / 448, code = v / scale: the largest becomes 448, the largest finite code.  Blocks whose largest is below 448 * 2^-126
// (the scale would lose digits) count as zeros: scale 0, codes 0.  A block that holds an infinity has an infinite scale, one that holds a
// NaN a NaN for it.
constexpr float kMostE4M3 = 448.f;
struct E4M3Scale {
  float scale, inverse, rest;         // rest = 1 - scale * inverse
};
__device__ __forceinline__ E4M3Scale e4m3_scale(uint32_t largest_bits) {       // of |v|: as integers they compare alike, NaNs highest
  const float most = __uint_as_float(largest_bits);
  const bool none = most < 448.f * 1.17549435e-38f;
  const float scale = none ? 0.f : __fdiv_rn(most, kMostE4M3), inverse = none ? 0.f : __fdiv_rn(1.f, scale);
  return {scale, inverse, inverse == 0.f ? 0.f : __fmaf_rn(-scale, inverse, 1.f)};
}
// The quotient v / scale = v * inverse / (1 - rest) = v * inverse + v * inverse * rest + ..., within 2^-46 of its size before its one rounding to fp32.
// (v * inverse alone is off by up to two steps of fp32 and lands on the other side of a border of two codes where the quotient is on it: 3 of
// 10000 codes of bf16 weights.)  None of its terms leaves the normal numbers, whatever the scale.  The compiler's own division takes 2304 x 4096 rows
// 14.4 us, these three operations 12.8, one 12.5; 16384 x 1280 weights 17.6, 12.2 and 11.1.
//   Zeros and infinite scales have 0 for inverse and rest: quotients 0, and NaN for an infinity.  A quotient is at most 448.0001, which
// rounds to 448, so nothing has to be clamped.
__device__ __forceinline__ uint2 to_e4m3(f32x8 v, const E4M3Scale& s) {
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = __fmaf_rn(v[j], s.inverse, v[j] * s.inverse * s.rest);
  auto four = [&](float a, float b, float c, float d) -> uint32_t {
    const int low = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(c, d, low, true));
  };
  return make_uint2(four(v[0], v[1], v[2], v[3]), four(v[4], v[5], v[6], v[7]));
}
__device__ __forceinline__ uint32_t largest_bits(f32x8 v) {
  uint32_t m = 0u;
#pragma unroll
  for (int j = 0; j < 8; ++j) m = max(m, __float_as_uint(v[j]) & 0x7FFFFFFFu);
  return m;
}

}  // namespace
}  // namespace scd
