// C ABI of the 8-bit floating point side (declared in include/ojbkq_fp8.h):
// argument checks.
#include "ojbkq_fp8.h"

#include <cmath>

#include "api_error.h"
#include "fp8.h"
#include "kernels.h"

namespace {

using ojbkq::fail;

constexpr int64_t kMaxRows = (int64_t)1 << 24, kMaxFeatures = (int64_t)1 << 20;
constexpr int64_t kMaxStride = (int64_t)1 << 40;   // keeps every offset inside 64 bits

bool type_ok(int32_t t) { return t == OJBKQ_F32 || t == OJBKQ_F16 || t == OJBKQ_BF16; }
bool misaligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a != 0; }
size_t size_of(int32_t t) { return t == OJBKQ_F32 ? 4 : 2; }

// An 8-bit array [rows, m] and its scales.
int check_fp8(const char* name, const void* X8, int64_t ld8, const void* scales, int64_t lds,
              int64_t m) {
  const std::string n(name);
  if (!X8 || !scales) return fail(OJBKQ_EINVAL, n + " and its scales are required");
  const int64_t G = (m + OJBKQ_FP8_BLOCK - 1) / OJBKQ_FP8_BLOCK;
  if (ld8 % 16 != 0 || ld8 < (m + 15) / 16 * 16 || ld8 > kMaxStride)
    return fail(OJBKQ_EINVAL, n + ": the row stride must be a multiple of 16 and hold m");
  if (lds % 4 != 0 || lds < (G + 3) / 4 * 4 || lds > kMaxStride)
    return fail(OJBKQ_EINVAL, n + ": the scales' row stride must be a multiple of 4 and hold ceil(m / 128)");
  if (misaligned(X8, 16) || misaligned(scales, 4))
    return fail(OJBKQ_EINVAL, n + " must be 16-byte aligned and its scales 4-byte aligned");
  return OJBKQ_OK;
}

bool product_sizes_ok(int64_t n, int64_t m, int64_t T) {
  return n >= 1 && m >= 1 && T >= 1 && n <= kMaxRows && T <= kMaxRows && m <= kMaxFeatures;
}

// What both products share: sizes, activations, result.
int check_product(int64_t n, int64_t m, int64_t T, const uint8_t* X8, int64_t ldx,
                  const uint8_t* x_scales, int64_t ldxs, const void* Y, int32_t ytype,
                  int32_t tokens_first, int64_t ldy) {
  if (!Y) return fail(OJBKQ_EINVAL, "Y is required");
  if (!product_sizes_ok(n, m, T))
    return fail(OJBKQ_EINVAL, "n and T must be in [1, 2^24] and m in [1, 2^20]");
  if (!type_ok(ytype)) return fail(OJBKQ_EINVAL, "ytype must be OJBKQ_F32, OJBKQ_F16 or OJBKQ_BF16");
  if (tokens_first != 0 && tokens_first != 1) return fail(OJBKQ_EINVAL, "tokens_first must be 0 or 1");
  if (ldy < (tokens_first ? n : T) || ldy > kMaxStride)
    return fail(OJBKQ_EINVAL, "ldy must be at least the length of Y's rows");
  if (misaligned(Y, size_of(ytype))) return fail(OJBKQ_EINVAL, "Y must be aligned to its type");
  return check_fp8("X8", X8, ldx, x_scales, ldxs, m);
}

}  // namespace

extern "C" {

int ojbkq_quantize_fp8(const void* X, int32_t xtype, int64_t rows, int64_t m, int64_t ldx,
                       int32_t features_first, int32_t block_rows, uint8_t* X8, int64_t ld8,
                       uint8_t* scales, int64_t lds, void* stream) {
  ojbkq::clear_error();
  if (!X) return fail(OJBKQ_EINVAL, "X is required");
  if (!type_ok(xtype)) return fail(OJBKQ_EINVAL, "xtype must be OJBKQ_F32, OJBKQ_F16 or OJBKQ_BF16");
  if (rows < 1 || m < 1 || rows > kMaxRows || m > kMaxFeatures)
    return fail(OJBKQ_EINVAL, "rows must be in [1, 2^24] and m in [1, 2^20]");
  if (features_first != 0 && features_first != 1)
    return fail(OJBKQ_EINVAL, "features_first must be 0 or 1");
  if (block_rows != 1 && (block_rows != 128 || features_first))
    return fail(OJBKQ_EINVAL, "block_rows must be 1, or 128 with the features contiguous");
  if (ldx < (features_first ? rows : m) || ldx > kMaxStride)
    return fail(OJBKQ_EINVAL, "ldx must be at least the length of X's rows");
  if (misaligned(X, size_of(xtype))) return fail(OJBKQ_EINVAL, "X must be aligned to its type");
  if (int rc = check_fp8("X8", X8, ld8, scales, lds, m)) return rc;
  const ojbkq::Quantize8Args a{X, rows, m, ldx, X8, ld8, scales, lds};
  OJBKQ_HIP(ojbkq::launch_quantize_fp8(a, xtype, features_first != 0, block_rows,
                                       static_cast<hipStream_t>(stream)),
            "quantize to 8 bits");
  return OJBKQ_OK;
}

int ojbkq_rmsnorm_fp8(const void* x, int32_t xtype, int64_t T, int64_t m, int64_t ldx,
                      const void* residual_in, void* residual_out, int32_t rtype, int64_t ldr,
                      const float* gain, double eps, uint8_t* X8, int64_t ld8, uint8_t* scales,
                      int64_t lds, void* stream) {
  ojbkq::clear_error();
  if (!x) return fail(OJBKQ_EINVAL, "x is required");
  if (!type_ok(xtype)) return fail(OJBKQ_EINVAL, "xtype must be OJBKQ_F32, OJBKQ_F16 or OJBKQ_BF16");
  if (T < 1 || m < 1 || T > kMaxRows || m > kMaxFeatures)
    return fail(OJBKQ_EINVAL, "T must be in [1, 2^24] and m in [1, 2^20]");
  if (ldx < m || ldx > kMaxStride) return fail(OJBKQ_EINVAL, "ldx must be >= m");
  if ((residual_in == nullptr) != (residual_out == nullptr))
    return fail(OJBKQ_EINVAL, "residual_in and residual_out go together");
  if (residual_in) {
    if (!type_ok(rtype)) return fail(OJBKQ_EINVAL, "rtype must be OJBKQ_F32, OJBKQ_F16 or OJBKQ_BF16");
    if (ldr < m || ldr > kMaxStride) return fail(OJBKQ_EINVAL, "ldr must be >= m");
    if (misaligned(residual_in, size_of(rtype)) || misaligned(residual_out, size_of(rtype)))
      return fail(OJBKQ_EINVAL, "the residual must be aligned to its type");
  }
  if (misaligned(x, size_of(xtype))) return fail(OJBKQ_EINVAL, "x must be aligned to its type");
  if (misaligned(gain, 4)) return fail(OJBKQ_EINVAL, "gain must be aligned to its type");
  if (!(eps >= 0.0) || !std::isfinite(eps)) return fail(OJBKQ_EINVAL, "eps must be finite and >= 0");
  if (int rc = check_fp8("X8", X8, ld8, scales, lds, m)) return rc;
  const ojbkq::Norm8Args a{x, T, m, ldx, residual_in, residual_out, ldr, gain, eps, X8, ld8, scales, lds};
  OJBKQ_HIP(ojbkq::launch_rmsnorm_fp8(a, xtype, rtype, static_cast<hipStream_t>(stream)),
            "rms norm to 8 bits");
  return OJBKQ_OK;
}

int ojbkq_matmul_fp8(const uint8_t* W8, int64_t ldw, const void* w_scales, int32_t w_scale_type,
                     int32_t w_block_rows, int64_t ldws, int64_t n, int64_t m, const uint8_t* X8,
                     int64_t ldx, const uint8_t* x_scales, int64_t ldxs, int64_t T, void* Y,
                     int32_t ytype, int32_t tokens_first, int64_t ldy, void* stream) {
  ojbkq::clear_error();
  if (int rc = check_product(n, m, T, X8, ldx, x_scales, ldxs, Y, ytype, tokens_first, ldy)) return rc;
  if (w_scale_type != OJBKQ_SCALE_F32 && w_scale_type != OJBKQ_SCALE_E8M0)
    return fail(OJBKQ_EINVAL, "w_scale_type must be OJBKQ_SCALE_F32 or OJBKQ_SCALE_E8M0");
  if (w_block_rows != 1 && w_block_rows != 128) return fail(OJBKQ_EINVAL, "w_block_rows must be 1 or 128");
  const bool e8m0 = w_scale_type == OJBKQ_SCALE_E8M0;
  const int64_t G = (m + OJBKQ_FP8_BLOCK - 1) / OJBKQ_FP8_BLOCK;
  if (int rc = check_fp8("W8", W8, ldw, w_scales, e8m0 ? ldws : (G + 3) / 4 * 4, m)) return rc;
  if (!e8m0 && (ldws < G || ldws > kMaxStride)) return fail(OJBKQ_EINVAL, "ldws must be >= ceil(m / 128)");
  ojbkq::Product8Args a{};
  a.n = n; a.m = m; a.T = T;
  a.W8 = W8; a.ldw = ldw;
  a.ws = w_scales; a.ws_ld = ldws; a.ws_shift = w_block_rows == 128 ? 7 : 0; a.ws_e8m0 = e8m0; a.ws_div = 1;
  a.X8 = X8; a.ldx = ldx; a.xs = x_scales; a.lds = ldxs;
  a.Y = Y; a.ldy = ldy; a.ytype = ytype; a.tokens_first = tokens_first;
  OJBKQ_HIP(ojbkq::launch_product8(a, 0, nullptr, static_cast<hipStream_t>(stream)), "8-bit product");
  return OJBKQ_OK;
}

size_t ojbkq_dequant_matmul_fp8_workspace_bytes(int64_t n, int64_t m, int64_t T) {
  return product_sizes_ok(n, m, T) ? ojbkq::product8_workspace_bytes(n, m, T) : 0;
}

int ojbkq_dequant_matmul_fp8(const uint32_t* packed, const float* scales, const float* zeros,
                             int64_t n, int64_t m, int32_t bits, int32_t group, const uint8_t* X8,
                             int64_t ldx, const uint8_t* x_scales, int64_t ldxs, int64_t T,
                             void* Y, int32_t ytype, int32_t tokens_first, int64_t ldy,
                             void* workspace, size_t workspace_bytes, void* stream) {
  ojbkq::clear_error();
  if (!packed || !scales || !zeros) return fail(OJBKQ_EINVAL, "packed, scales and zeros are required");
  if (misaligned(packed, 4) || misaligned(scales, 4) || misaligned(zeros, 4))
    return fail(OJBKQ_EINVAL, "packed, scales and zeros must be aligned to their types");
  if (int rc = check_product(n, m, T, X8, ldx, x_scales, ldxs, Y, ytype, tokens_first, ldy)) return rc;
  if (bits < 1 || bits > 4)
    return fail(OJBKQ_EINVAL, "bits must be in [1, 4]: longer codes are not exact in 8-bit floating point");
  const int64_t g = (group <= 0 || group >= m) ? m : group;
  if (g != m && g % OJBKQ_FP8_BLOCK != 0)
    return fail(OJBKQ_EINVAL, "the group must be a multiple of 128 (or the whole column)");
  const size_t need = ojbkq::product8_workspace_bytes(n, m, T);
  if (need) {
    if (!workspace) return fail(OJBKQ_EINVAL, "this product needs a workspace");
    if (workspace_bytes < need)
      return fail(OJBKQ_ENOSPACE, "workspace smaller than ojbkq_dequant_matmul_fp8_workspace_bytes");
    if (misaligned(workspace, 16)) return fail(OJBKQ_EINVAL, "the workspace must be 16-byte aligned");
  }
  ojbkq::Product8Args a{};
  a.n = n; a.m = m; a.T = T;
  a.P = packed; a.wpr = ojbkq::packed_words(m, bits); a.Z = zeros;
  a.ws = scales; a.ws_ld = (m + g - 1) / g; a.ws_shift = 0; a.ws_e8m0 = 0;
  a.ws_div = (uint32_t)((g + OJBKQ_FP8_BLOCK - 1) / OJBKQ_FP8_BLOCK);
  a.X8 = X8; a.ldx = ldx; a.xs = x_scales; a.lds = ldxs;
  a.Y = Y; a.ldy = ldy; a.ytype = ytype; a.tokens_first = tokens_first;
  OJBKQ_HIP(ojbkq::launch_product8(a, bits, workspace, static_cast<hipStream_t>(stream)),
            "product of codes with 8-bit activations");
  return OJBKQ_OK;
}

}  // extern "C"
