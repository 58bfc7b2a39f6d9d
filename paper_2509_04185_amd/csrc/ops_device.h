// Device-side helpers of the operators without a context: 16-bit element types, e4m3
// conversions, block exponents, the search for a row's sequence.  Included only by *.hip files.
#pragma once

#include "ops_internal.h"
#include "sbd_device.h"

namespace sbd {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

struct Bf16 {};  // tags of the 16-bit element types
struct Fp16 {};

// Two elements in a 32-bit word, low one first.
template <class T>
__device__ __forceinline__ f32x2 unpack2(uint32_t w) {
  if constexpr (std::is_same_v<T, Bf16>)
    return f32x2{__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)};
  else
    return __builtin_convertvector(__builtin_bit_cast(f16x2, w), f32x2);
}
template <class T>
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  if constexpr (std::is_same_v<T, Bf16>)
    return pack_bf2(a, b);
  else
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{a, b}), f16x2));
}

// 16x16x32 product of 16-bit operands, fp32 sums.
template <class T>
__device__ __forceinline__ f32x4 mfma16(i32x4 a, i32x4 b, f32x4 c) {
  if constexpr (std::is_same_v<T, Bf16>)
    return mfma16x16x32(a, b, c);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// Eight e4m3 codes as 16-bit values times s (a power of two).  In bf16 every code is exact; in
// fp16 every code times s >= 2^-15 is (the smallest code is 2^-9, the smallest fp16 2^-24).
template <class T>
__device__ __forceinline__ i32x4 widen8(i32x2 w, float s) {
  if constexpr (std::is_same_v<T, Bf16>) {
    return e4m3x8_to_bf16(w, s);
  } else {
    i32x4 o;
    o[0] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w[0], s, false));
    o[1] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w[0], s, true));
    o[2] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w[1], s, false));
    o[3] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w[1], s, true));
    return o;
  }
}

// v in [-448, 448] (infinities too); NaN stays NaN.
__device__ __forceinline__ float clamp_e4m3(float v) {
  v = v > 448.f ? 448.f : v;
  return v < -448.f ? -448.f : v;
}
// e4m3 codes of four values, nearest with ties to even, saturating (the gfx950 conversion
// rounds so; it is given values of at most 448).
__device__ __forceinline__ uint32_t to_e4m3x4(float a, float b, float c, float d) {
  int v = __builtin_amdgcn_cvt_pk_fp8_f32(clamp_e4m3(a), clamp_e4m3(b), 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(clamp_e4m3(c), clamp_e4m3(d), v, true);
}

// |v| where v is finite, else 0: infinities and NaN do not move a block's exponent.
__device__ __forceinline__ float finite_abs(float v) {
  const float a = fabsf(v);
  return a <= 3.402823466e38f ? a : 0.f;
}
// Smallest e in [-100, 100] with amax <= 448 * 2^e.  With amax = f * 2^x, f in [0.5, 1), and
// 448 = 0.875 * 2^9, that is x - 9, or one more when f > 0.875 (mantissa bits above 0x600000).
__device__ __forceinline__ int block_exponent(float amax) {
  const uint32_t u = __float_as_uint(amax);
  const int e = (int)(u >> 23) - 126 - 9 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
  return min(max(e, -100), 100);
}
// 2^e, e in [-126, 127]
__device__ __forceinline__ float pow2i(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// Largest b in [0, n) with start(b) <= idx, for a start() that rises and start(0) <= idx: 64
// probes at a time.  Every lane of the wave takes part.  Leaves
// lo and n such that b is one of lo .. lo + n, n <= 64, for the caller's own last round.  They stay
// in range whatever start() gives.
template <class F>
__device__ __forceinline__ void narrow_sequence(int& lo, int& n, int64_t idx, F&& start) {
  const int lane = threadIdx.x & 63;
  while (n > 64) {
    const int step = (n + 63) / 64;
    const int at = lane * step;
    const bool below = at < n && start(lo + at) <= idx;
    const int c = max(1, (int)__popcll(__ballot(below)));
    lo += (c - 1) * step;
    n = min(step, n - (c - 1) * step);
  }
}
}  // namespace sbd
