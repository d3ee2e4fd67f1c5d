// The products of 32-bit matrices.
#include "ffproduct.cuh"

namespace abcd {

abcd_status launch_32(abcd_ctx* ctx, int epi, int shape, const ProductArgs& a) {
  return launch_any<true>(ctx, epi, shape, a);
}

}  // namespace abcd
