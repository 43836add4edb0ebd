/*
 * ojbkq_fp8.h -- C ABI of the 8-bit floating point side of the library: the
 * activations of a linear layer in 8 bits, and the layer's product with them.
 *
 * A layer quantized by the calls of ojbkq.h is applied as W_hat = S (Q - Z)
 * (the Q, S, Z data model of Sec. 3.2) to activations in 16 bits
 * (ojbkq_dequant_matmul).  The calls here bring the activations to 8 bits --
 * by themselves, or as the output of the norm in front of the layer -- and
 * multiply them with such a layer, or with weights that are 8-bit floating
 * point numbers themselves.
 *
 * Number formats (those of the OCP 8-bit and microscaling specifications)
 *   e4m3  sign, 4 exponent bits, 3 mantissa bits; largest 448, smallest
 *         2^-9; no infinity, one NaN (0x7f, 0xff).
 *   e8m0  a power of two 2^(code - 127) in a byte (code 255, NaN, is never
 *         written).
 *   A scale that is a power of two costs a floating point format nothing
 *   (multiplying by it is exact).
 *
 * An 8-bit array is [rows, m] e4m3 values, features contiguous, row stride ld
 * (bytes), with one e8m0 scale for each block of `block_rows` rows (1 or 128)
 * x 128 features: [ceil(rows / block_rows), G], G = ceil(m / 128), row stride
 * lds (bytes).  It stands for value x scale.  The values are 16-byte aligned,
 * ld is a multiple of 16 and at least m rounded up to 16; the scales are 4-byte
 * aligned, lds is a multiple of 4 and at least G rounded up to 4.  Every row
 * (the last one too) is readable up to these roundings; what stands there is
 * not used.
 *
 * Conventions otherwise as in ojbkq.h: device pointers owned by the caller, no
 * device memory allocated, argument errors (OJBKQ_EINVAL) before anything is
 * enqueued, messages through ojbkq_last_error().  Every call is asynchronous
 * on `stream`, which must belong to the current device, and can be captured
 * into a HIP graph.  Results depend only on the inputs, and outputs must not
 * overlap inputs except where a call says so.
 */
#ifndef OJBKQ_FP8_H
#define OJBKQ_FP8_H

#include "ojbkq.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Features to a scale. */
#define OJBKQ_FP8_BLOCK 128

/* Types of the arrays that are not in 8 bits. */
enum { OJBKQ_F32 = 0, OJBKQ_F16 = 1, OJBKQ_BF16 = 2 };

/* Types of the scales of 8-bit weights. */
enum { OJBKQ_SCALE_F32 = 0, OJBKQ_SCALE_E8M0 = 1 };

/* X brought to 8 bits.  With a the largest finite magnitude of a block, its
 * scale is 2^e with the least e >= -127 for which a <= 448 2^e (2^0 where a =
 * 0), and its values are e4m3(x 2^-e), to nearest even.  Infinities and NaN
 * become NaN and leave the others alone.
 *   X: type xtype (OJBKQ_F32, _F16, _BF16).  features_first = 0: [rows, m],
 *   row stride ldx >= m (elements).  features_first = 1: [m, rows], row stride
 *   ldx >= rows, i.e. X as ojbkq_dequant_matmul and ojbkq_quantize_layer take
 *   it, with `rows` tokens; block_rows must be 1 then.
 *   X8, scales: the 8-bit array [rows, m]; bytes m .. of a row up to m rounded
 *   up to 16 are zeroed.
 *   rows >= 1, 1 <= m <= 2^20, rows <= 2^24, block_rows 1 or 128.           */
int ojbkq_quantize_fp8(const void* X, int32_t xtype, int64_t rows, int64_t m, int64_t ldx,
                       int32_t features_first, int32_t block_rows, uint8_t* X8, int64_t ld8,
                       uint8_t* scales, int64_t lds, void* stream);

/* Root-mean-square norm of a residual stream, its output in 8 bits:
 *     h = x + residual_in (a float32 sum; h = x where residual_in is NULL),
 *     residual_out = h rounded to rtype,
 *     y = h gain / sqrt(mean(h^2) + eps)   (the mean over the token's features),
 *   and y is brought to 8 bits as by ojbkq_quantize_fp8 with block_rows = 1.
 *   Norm and rounding to 8 bits are those of float64: h gain is exact there, it
 *   is divided by the root once, and y is not rounded in between (one that lies
 *   on a border of e4m3 goes to the even side); a y beyond float32's range counts
 *   as infinite.  A token whose h holds a NaN or an infinity comes out as NaN,
 *   and so does one of zeros with eps = 0 (0 / 0).  A token's results do not go
 *   by the other tokens or by how many they are.
 *   x [T, m] type xtype, row stride ldx; residual_in, residual_out [T, m] type
 *   rtype, row stride ldr (elements), both or neither given.  residual_out may be
 *   residual_in (an update in place), or x where their rows and the size of their
 *   elements agree, and must not overlap either otherwise.  gain [m] float32
 *   (NULL: 1).  eps >= 0, finite.
 *   X8, scales as above.  T >= 1, 1 <= m <= 2^20, T <= 2^24.                */
int ojbkq_rmsnorm_fp8(const void* x, int32_t xtype, int64_t T, int64_t m, int64_t ldx,
                      const void* residual_in, void* residual_out, int32_t rtype, int64_t ldr,
                      const float* gain, double eps, uint8_t* X8, int64_t ld8, uint8_t* scales,
                      int64_t lds, void* stream);

/* The product of 8-bit weights with 8-bit activations:
 *     Y[j][t] = sum over blocks g of  sw[j / r][g] sx[t][g] sum_i W8[j][i] X8[t][i],
 *   i over the features of block g and r = w_block_rows (1 or 128).
 *   W8 [n, m] e4m3, row stride ldw; w_scales [ceil(n / r), ceil(m / 128)],
 *   row stride ldws (elements), any OJBKQ_SCALE_F32 or OJBKQ_SCALE_E8M0: with
 *   e8m0 ones an 8-bit array as above (ojbkq_quantize_fp8 of W).
 *   X8 [T, m] with scales x_scales: an 8-bit array of block_rows = 1.
 *   Y: type ytype; tokens_first = 0: [n, T], row stride ldy >= T, as
 *   ojbkq_dequant_matmul gives it; tokens_first = 1: [T, n], ldy >= n.
 *   Results are rounded to ytype once.  OJBKQ_F32: products enter exactly and
 *   are summed in float32.  In 16 bits, the matrix cores' 8-bit products serve
 *   sizes beyond a few tokens: they add eight neighbouring products after
 *   cutting each, towards zero, to 13 bits below the largest's leading one, and
 *   sums of these in float32.  Root mean square of that, relative to the
 *   results': 1.5e-5 for Gaussian operands, 7e-5 to 8e-5 for activations with
 *   log-normal channel scales and outlier channels, where rounding to 16 bits
 *   costs 2.1e-4 (float16; both together 2.2e-4) or 1.66e-3 (bfloat16; no more
 *   together); for operands of one sign it is a bias towards zero (3e-6 for
 *   magnitudes of Gaussian numbers).  So a token's last bits differ between a
 *   call with a few tokens and one with many.
 *   Weights and activations (value times scale) are taken as float32's normal
 *   numbers: a magnitude below 2^-126 may count as 0, one from 2^128 on as
 *   infinite.
 *   A NaN in a token or a channel comes out in all it meets; so does an
 *   infinite scale, and an e8m0 scale of code 255 makes all it meets infinite or
 *   NaN.  n, T in [1, 2^24], m in [1, 2^20].                                */
int ojbkq_matmul_fp8(const uint8_t* W8, int64_t ldw, const void* w_scales, int32_t w_scale_type,
                     int32_t w_block_rows, int64_t ldws, int64_t n, int64_t m, const uint8_t* X8,
                     int64_t ldx, const uint8_t* x_scales, int64_t ldxs, int64_t T, void* Y,
                     int32_t ytype, int32_t tokens_first, int64_t ldy, void* stream);

/* The product of a layer as this library quantizes it (packed, scales, zeros,
 * bits and group as in ojbkq_dequant_matmul, without a permutation) with 8-bit
 * activations:
 *     Y[j][t] = sum over groups g of  s[j][g] sum_i (q[j][i] - z[j][g]) X[t][i],
 *   X[t][i] = X8[t][i] sx[t][i / 128].  A code less its zero point is a whole
 *   number of at most 15 and enters the products exactly; no weight is rounded.
 *   bits in [1, 4]; group a multiple of 128, or one group (group <= 0 or >= m).
 *   zeros are whole numbers in 0 .. 2^bits - 1, as the quantize calls return
 *   them (any other is taken as the nearest of these).
 *   X8, x_scales, Y, ytype, tokens_first, ldy as in ojbkq_matmul_fp8.
 *   workspace: ojbkq_dequant_matmul_fp8_workspace_bytes(n, m, T) bytes, 16-byte
 *   aligned (NULL where that is 0), untouched until the product has run:
 *   ENOSPACE for fewer, EINVAL for a NULL or misaligned one.
 * ojbkq_dequant_matmul_fp8_workspace_bytes: host-only; 0 for sizes that need
 *   none, and for those that the product rejects.                           */
size_t ojbkq_dequant_matmul_fp8_workspace_bytes(int64_t n, int64_t m, int64_t T);
int ojbkq_dequant_matmul_fp8(const uint32_t* packed, const float* scales, const float* zeros,
                             int64_t n, int64_t m, int32_t bits, int32_t group, const uint8_t* X8,
                             int64_t ldx, const uint8_t* x_scales, int64_t ldxs, int64_t T,
                             void* Y, int32_t ytype, int32_t tokens_first, int64_t ldy,
                             void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* OJBKQ_FP8_H */
