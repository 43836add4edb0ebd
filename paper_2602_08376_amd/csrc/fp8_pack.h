// Rounding to 8 bits with a power-of-two scale, on the device.
//
// A block's scale 2^e is the least with a <= 448 2^e for its largest finite
// magnitude a; 448 = 1.75 x 2^8, so e is a's exponent less 8, one more where
// its mantissa is above 1.75.  Dividing by it is exact, so a value is rounded
// once, by the convert to e4m3.
#pragma once

#include "fp8.h"

namespace ojbkq {

typedef uint32_t u2 __attribute__((ext_vector_type(2)));

// The largest of a value over the 16 lanes of a row of lanes, in all of them.
__device__ __forceinline__ uint32_t max16(uint32_t v) {
#define OJBKQ_ROTATE(N)                                                                        \
  {                                                                                            \
    const uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x120 + N, 0xf, 0xf,   \
                                                             true);                            \
    v = v > o ? v : o;                                                                         \
  }
  OJBKQ_ROTATE(8)
  OJBKQ_ROTATE(4)
  OJBKQ_ROTATE(2)
  OJBKQ_ROTATE(1)
#undef OJBKQ_ROTATE
  return v;
}

// ---- from float32 ----------------------------------------------------------

// |v| as an integer that grows with it; 0 for infinities and NaN.
__device__ __forceinline__ uint32_t size_key(float v) {
  const uint32_t a = __float_as_uint(v) & 0x7fffffffu;
  return a < 0x7f800000u ? a : 0u;
}
// The scale's code from the largest key of the block.
__device__ __forceinline__ uint32_t scale_code(uint32_t a) {
  const int c = (int)(a >> 23) - 8 + ((a & 0x7fffffu) > 0x600000u ? 1 : 0);
  return a == 0u ? 127u : (uint32_t)(c > 0 ? c : 0);
}
// 2^-e (codes up to 247 come from float32 values).
__device__ __forceinline__ float inverse_scale(uint32_t code) {
  return __uint_as_float((254u - code) << 23);
}
__device__ __forceinline__ float finite_or_nan(float v) {
  return __builtin_fabsf(v) <= 3.402823466e38f ? v : __builtin_nanf("");
}
// Eight values, lowest byte first.
__device__ __forceinline__ u2 to_e4m3(const float (&v)[8], float inv) {
  u2 out;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(finite_or_nan(v[4 * h]) * inv,
                                            finite_or_nan(v[4 * h + 1]) * inv, 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(finite_or_nan(v[4 * h + 2]) * inv,
                                        finite_or_nan(v[4 * h + 3]) * inv, w, true);
    out[h] = (uint32_t)w;
  }
  return out;
}

// ---- from float64 ----------------------------------------------------------

// The high word of a float64, its last bit set where anything stands below
// it: 20 mantissa bits and a sticky one, all that rounding to 4 bits needs.
__device__ __forceinline__ uint32_t sticky_high(double v) {
  const uint64_t b = __builtin_bit_cast(uint64_t, v);
  return (uint32_t)(b >> 32) | ((uint32_t)b != 0u ? 1u : 0u);
}
constexpr uint32_t kBeyondFloat = (1023u + 128u) << 20;   // 2^128 and above, infinities, NaN
__device__ __forceinline__ uint32_t size_key64(uint32_t hi) {
  const uint32_t a = hi & 0x7fffffffu;
  return a < kBeyondFloat ? a : 0u;
}
__device__ __forceinline__ uint32_t scale_code64(uint32_t a) {
  const int c = (int)(a >> 20) - (1023 - 127) - 8 + ((a & 0xfffffu) > 0xc0000u ? 1 : 0);
  return a == 0u ? 127u : (uint32_t)(c > 0 ? c : 0);
}
// The value over its scale as a float32 that rounds to e4m3 as it does: the
// exponent moved (below float32's range it is 0, far under half the smallest
// e4m3 number), the mantissa's 20 bits with the sticky one as the last.
__device__ __forceinline__ float scaled64(uint32_t hi, uint32_t code) {
  const uint32_t a = hi & 0x7fffffffu;
  const int t = (int)a - (int)((code + (1023 - 127) - 127u) << 20);
  const uint32_t f = (uint32_t)(t > 0 ? t : 0) << 3;
  return a < kBeyondFloat ? __uint_as_float((hi & 0x80000000u) | f) : __builtin_nanf("");
}
__device__ __forceinline__ u2 to_e4m3(const uint32_t (&hi)[8], uint32_t code) {
  u2 out;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(scaled64(hi[4 * h], code),
                                            scaled64(hi[4 * h + 1], code), 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(scaled64(hi[4 * h + 2], code),
                                        scaled64(hi[4 * h + 3], code), w, true);
    out[h] = (uint32_t)w;
  }
  return out;
}

// ---- eight neighbours ------------------------------------------------------

// Eight elements at any alignment; those past `left` are 0.
template <class E>
struct Eight {
  typedef E Any __attribute__((ext_vector_type(8), aligned(sizeof(E))));
  Any v;
  __device__ __forceinline__ void load(const E* p, int64_t left) {
    if (left >= 8) {
      v = *reinterpret_cast<const Any*>(p);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = i < left ? p[i] : (E)0.f;
    }
  }
  __device__ __forceinline__ void store(E* p, int64_t left) const {
    if (left >= 8) {
      *reinterpret_cast<Any*>(p) = v;
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i < left) p[i] = v[i];
    }
  }
};

}  // namespace ojbkq
