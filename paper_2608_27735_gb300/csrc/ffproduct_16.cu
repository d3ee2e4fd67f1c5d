// The gated feed-forward layer's products of 16-bit matrices.
#include "ffproduct.cuh"

namespace abcd {

abcd_status launch_16(abcd_ctx* ctx, int epi, int shape, const ProductArgs& a) {
  return launch_any<false>(ctx, epi, shape, a);
}

}  // namespace abcd
