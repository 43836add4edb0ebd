// 8-bit floating point arrays (ojbkq_fp8.h): the launches behind the entry
// points and what their kernels share.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace ojbkq {

constexpr int kFp8Block = 128;   // features to a scale

// Element types of the arrays that are not in 8 bits, in the order of
// OJBKQ_F32, OJBKQ_F16, OJBKQ_BF16.
template <int TYPE> struct Number { typedef float type; };
template <> struct Number<1> { typedef _Float16 type; };
template <> struct Number<2> { typedef __bf16 type; };

struct Quantize8Args {
  const void* X;
  int64_t rows, m, ldx;
  uint8_t* X8;
  int64_t ld8;
  uint8_t* scales;
  int64_t lds;
};
hipError_t launch_quantize_fp8(const Quantize8Args& a, int xtype, bool features_first,
                               int block_rows, hipStream_t stream);

struct Norm8Args {
  const void* x;
  int64_t T, m, ldx;
  const void* r_in;   // null: no residual
  void* r_out;
  int64_t ldr;
  const float* gain;  // null: 1
  double eps;
  uint8_t* X8;
  int64_t ld8;
  uint8_t* scales;
  int64_t lds;
};
hipError_t launch_rmsnorm_fp8(const Norm8Args& a, int xtype, int rtype, hipStream_t stream);

}  // namespace ojbkq
