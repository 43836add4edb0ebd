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

// Y = W X^T of 8-bit weights, or of packed codes, with 8-bit activations.
struct Product8Args {
  int64_t n, m, T;
  const uint8_t* W8;      // [n, m] e4m3, row stride ldw; or null:
  int64_t ldw;
  const uint32_t* P;      // packed codes, wpr words to a row,
  int64_t wpr;
  const float* Z;         // with zero points laid out as the scales
  const void* ws;         // scale of row j, block b of 128 features:
  int64_t ws_ld;          //   ws[(j >> ws_shift) * ws_ld + b / ws_div]
  int ws_shift, ws_e8m0;  //   e8m0 bytes or float32
  uint32_t ws_div;
  const uint8_t* X8;      // [T, m] e4m3, row stride ldx, scales xs, row stride lds
  int64_t ldx;
  const uint8_t* xs;
  int64_t lds;
  void* Y;                // type ytype, tokens_first [T, n] or [n, T], row stride ldy
  int64_t ldy;
  int ytype, tokens_first;
};
// One pass over the weights or codes for every 16 or 32 tokens (fp8_few.hip).
hipError_t launch_product_few8(const Product8Args& a, int bits, hipStream_t stream);
// The product in the kernel that its sizes ask for (fp8_matmul.hip); bits = 0:
// of W8, otherwise of packed codes, with product8_workspace_bytes(n, m, T)
// bytes of workspace.
hipError_t launch_product8(const Product8Args& a, int bits, void* workspace, hipStream_t stream);
size_t product8_workspace_bytes(int64_t n, int64_t m, int64_t T);

}  // namespace ojbkq
