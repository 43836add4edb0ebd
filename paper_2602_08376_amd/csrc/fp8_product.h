// What the product kernels with 8-bit operands share (fp8_few.hip,
// fp8_matmul.hip).
#pragma once

#include "device.h"
#include "fp8.h"

namespace ojbkq {

typedef __bf16 b8 __attribute__((ext_vector_type(8)));
typedef __bf16 b2 __attribute__((ext_vector_type(2)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef float v4 __attribute__((ext_vector_type(4)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));
typedef uint32_t u2v __attribute__((ext_vector_type(2)));

// 4 bytes per lane straight to LDS, lane i's at lds + 4 i (load_to_lds16_at's
// narrow form).
__device__ __forceinline__ void load_to_lds4_at(const void* src, const void* lds) {
  const uint32_t a = __builtin_amdgcn_readfirstlane(lds_address(lds));
  asm volatile("s_nop 0\n\tglobal_load_lds_dword %0, off" : : "v"(src), "{m0}"(a) : "memory");
}
// All but the youngest N of the wave's loads have arrived.
template <int N>
__device__ __forceinline__ void wait_loads() {
  static_assert(N < 64, "six bits");
  asm volatile("s_waitcnt vmcnt(%0)" : : "n"(N) : "memory");
}

// 2^(code - 127) (code 0: 2^-127, the one below float32's normal range).
__device__ __forceinline__ float from_e8m0(uint32_t code) {
  const uint32_t b = code << 23;
  return __uint_as_float(b > (1u << 22) ? b : 1u << 22);
}

// A weight scale as a power of two, which goes to the weights in bf16 or in the
// matrix instruction (exactly), and the rest, with which a block's sums are
// multiplied: these then lie in the result's own range, whatever the scales.
// (The rest is 1 to 2; below it for 0 and numbers under float32's normal range,
// whose power is the range's least; all of an infinity or a NaN.)
struct SplitScale {
  float power, rest;
};
__device__ __forceinline__ SplitScale split_scale(float s) {
  const uint32_t b = __float_as_uint(s), e = b & 0x7f800000u;
  if (e == 0u) return {0x1p-126f, s * 0x1p126f};
  if (e == 0x7f800000u) return {1.f, s};
  return {__uint_as_float(e), __uint_as_float((b & 0x807fffffu) | 0x3f800000u)};
}

// Eight e4m3 values times a power of two, exactly, in bf16 (whose 8 mantissa
// bits and float32 exponents hold them).
__device__ __forceinline__ b8 to_bf16(uint32_t lo, uint32_t hi, float scale) {
  b8 out;
#pragma unroll
  for (int h = 0; h < 4; ++h) {
    const uint32_t w = h < 2 ? lo : hi;
    const b2 p = (h & 1) ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, true)
                         : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, false);
    out[2 * h] = p.x;
    out[2 * h + 1] = p.y;
  }
  return out;
}

// Code c (a constant after unrolling) of 32 that fill BITS words.
template <int BITS>
__device__ __forceinline__ uint32_t code_of(const uint32_t (&w)[BITS], int c) {
  const int b = c * BITS, lo = b >> 5, sh = b & 31;
  uint32_t q = w[lo] >> sh;
  if (sh + BITS > 32) q = __builtin_amdgcn_alignbit(w[lo + 1 < BITS ? lo + 1 : lo], w[lo], sh);
  return q & ((1u << BITS) - 1u);
}
// A zero point, the nearest whole number of the codes' range.
template <int BITS>
__device__ __forceinline__ float whole_zero(float z) {
  return fminf(fmaxf(__builtin_rintf(z), 0.f), (float)((1 << BITS) - 1));
}

// The bytes of a word that belong to features below m, the word starting at k.
__device__ __forceinline__ uint32_t features_below(uint32_t w, int64_t k, int64_t m) {
  const int64_t left = m - k;
  return left >= 4 ? w : left <= 0 ? 0u : w & ((1u << (8 * (int)left)) - 1u);
}

__device__ __forceinline__ void store_y(const Product8Args& a, int64_t j, int64_t t, float v) {
  const int64_t at = a.tokens_first ? t * a.ldy + j : j * a.ldy + t;
  if (a.ytype == 0) static_cast<float*>(a.Y)[at] = v;
  else if (a.ytype == 1) static_cast<_Float16*>(a.Y)[at] = (_Float16)v;
  else static_cast<__bf16*>(a.Y)[at] = (__bf16)v;
}

}  // namespace ojbkq
