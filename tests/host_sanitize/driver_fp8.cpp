// Drives the entry points of the 8-bit side (ojbkq_fp8.h) against the stub
// runtime: valid calls over types, sizes from one to the largest, strides and
// layouts, and the workspace's errors.  Every launch on the way is held against
// the device's limits (`__wrap_hipLaunchKernel`, put in front of the stub's by
// the linker).  Buffers are addresses only: no kernel runs.  Test
// infrastructure.
#include <hip/hip_runtime_api.h>

#include <cstdint>
#include <cstdio>
#include <cstdlib>

#include "ojbkq_fp8.h"

namespace {

int g_checks = 0, g_launches = 0;

void expect(int got, int want, const char* what) {
  ++g_checks;
  if (got != want) {
    std::fprintf(stderr, "FAIL %s: status %d, expected %d (%s)\n", what, got, want, ojbkq_last_error());
    std::exit(1);
  }
}

void* at(uintptr_t p) { return reinterpret_cast<void*>(p); }
uint8_t* bytes(uintptr_t p) { return reinterpret_cast<uint8_t*>(p); }
constexpr uintptr_t A = 4096;
int64_t up(int64_t v, int64_t s) { return (v + s - 1) / s * s; }

// a call that has to be accepted and to launch something
void runs(int got, const char* what) {
  expect(got, OJBKQ_OK, what);
  if (g_launches == 0) {
    std::fprintf(stderr, "FAIL %s: nothing launched\n", what);
    std::exit(1);
  }
  g_launches = 0;
}

}  // namespace

extern "C" hipError_t __real_hipLaunchKernel(const void* f, dim3 grid, dim3 block, void** args,
                                             size_t shmem, hipStream_t stream);
extern "C" hipError_t __wrap_hipLaunchKernel(const void* f, dim3 grid, dim3 block, void** args,
                                             size_t shmem, hipStream_t stream) {
  ++g_launches;
  const uint64_t x = (uint64_t)grid.x * block.x;
  if (!grid.x || !grid.y || !grid.z || grid.y > 65535 || grid.z > 65535 || x >> 32 ||
      block.x * block.y * block.z > 1024 || !block.x || shmem > 160 * 1024) {
    std::fprintf(stderr, "FAIL: a launch of %u x %u x %u groups of %u threads\n", grid.x, grid.y, grid.z, block.x);
    std::exit(1);
  }
  return __real_hipLaunchKernel(f, grid, block, args, shmem, stream);
}

int main() {
  const int64_t most = (int64_t)1 << 24, features = (int64_t)1 << 20;
  const int64_t rows[] = {1, 2, 4, 63, 64, 65, 128, 129, 1000, 65535, 65537, (int64_t)65535 * 128 + 1, most - 1, most};
  const int64_t ms[] = {1, 127, 128, 129, 2048, 2049, 4097, 8192, 8193, 32768, 32769, features - 1, features};
  for (int type = 0; type < 3; ++type)
    for (int64_t r : rows)
      for (int64_t m : ms) {
        const int64_t ld8 = up(m, 16), lds = up(up(m, 128) / 128, 4);
        for (int pad = 0; pad < 2; ++pad) {
          runs(ojbkq_quantize_fp8(at(A), type, r, m, m + pad, 0, 1, bytes(A), ld8 + 16 * pad, bytes(A), lds + 4 * pad, nullptr),
               "quantize rows");
          runs(ojbkq_quantize_fp8(at(A), type, r, m, m + pad, 0, 128, bytes(A), ld8, bytes(A), lds, nullptr),
               "quantize blocks");
          runs(ojbkq_quantize_fp8(at(A), type, r, m, r + pad, 1, 1, bytes(A), ld8, bytes(A), lds, nullptr),
               "quantize features first");
        }
        for (int res = -1; res < 3; ++res)
          runs(ojbkq_rmsnorm_fp8(at(A), type, r, m, m, res < 0 ? nullptr : at(A), res < 0 ? nullptr : at(A),
                                 res < 0 ? 0 : res, m + 3, nullptr, 1e-5, bytes(A), ld8, bytes(A), lds, nullptr), "norm");
      }
  const int64_t ns[] = {1, 31, 4097, 14336, 300000}, Ts[] = {1, 16, 17, 33, 300, 4097, 100000, most};
  for (int type = 0; type < 3; ++type)
    for (int64_t n : ns)
      for (int64_t T : Ts)
        for (int64_t m : {(int64_t)1, (int64_t)128, (int64_t)11009, features}) {
          if (n * T >> 38) continue;   // no memory holds the result
          const int64_t G = up(m, 128) / 128, ld = up(m, 16), lds = up(G, 4);
          for (int first = 0; first < 2; ++first)
            for (int e8m0 = 0; e8m0 < 2; ++e8m0)
              for (int64_t more : {(int64_t)0, (int64_t)1 << 23}) {
                const int64_t ldw = up(ld + (first ? more : 0), 16), ldx = up(ld + (first ? 0 : more), 16);
                runs(ojbkq_matmul_fp8(bytes(A), ldw, at(A), e8m0, first ? 1 : 128, lds, n, m, bytes(A), ldx, bytes(A),
                                      lds, T, at(A), type, first, first ? n : T, nullptr), "product");
              }
          const size_t need = ojbkq_dequant_matmul_fp8_workspace_bytes(n, m, T);
          auto codes = [&](int bits, int group, uintptr_t ws, size_t size) {
            return ojbkq_dequant_matmul_fp8(static_cast<uint32_t*>(at(A)), static_cast<float*>(at(A)),
                                            static_cast<float*>(at(A)), n, m, bits, group, bytes(A), ld, bytes(A), lds, T,
                                            at(A), type, 0, T, at(ws), size, nullptr);
          };
          for (int bits = 1; bits <= 4; ++bits)
            for (int group : {0, 128, 384}) runs(codes(bits, group, A, need), "codes");
          if (need) {
            expect(codes(4, 128, 0, need), OJBKQ_EINVAL, "no workspace");
            expect(codes(4, 128, A, need - 1), OJBKQ_ENOSPACE, "a small workspace");
            expect(codes(4, 128, A + 8, need), OJBKQ_EINVAL, "a misaligned workspace");
          } else {
            runs(codes(4, 128, 0, 0), "no workspace needed");
          }
        }
  for (int64_t bad : {(int64_t)0, (int64_t)-1, most + 1, INT64_MAX, INT64_MIN}) {
    expect((int)ojbkq_dequant_matmul_fp8_workspace_bytes(bad, 128, 4096), 0, "workspace of no channels");
    expect((int)ojbkq_dequant_matmul_fp8_workspace_bytes(4096, bad, 4096), 0, "workspace of no features");
    expect((int)ojbkq_dequant_matmul_fp8_workspace_bytes(4096, 128, bad), 0, "workspace of no tokens");
  }
  expect(ojbkq_quantize_fp8(nullptr, 0, 1, 1, 1, 0, 1, bytes(A), 16, bytes(A), 4, nullptr), OJBKQ_EINVAL, "no X");
  expect(ojbkq_rmsnorm_fp8(nullptr, 0, 1, 1, 1, nullptr, nullptr, 0, 1, nullptr, 0.0, bytes(A), 16, bytes(A), 4, nullptr),
         OJBKQ_EINVAL, "no x");
  std::printf("8-bit host driver: %d checks passed\n", g_checks);
  return 0;
}
