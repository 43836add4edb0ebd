// Products with 8-bit activations: the kernel for the sizes at hand.
#include "fp8_product.h"

namespace ojbkq {

size_t product8_workspace_bytes(int64_t, int64_t, int64_t) { return 0; }

hipError_t launch_product8(const Product8Args& a, int bits, void*, hipStream_t stream) {
  return launch_product_few8(a, bits, stream);
}

}  // namespace ojbkq
