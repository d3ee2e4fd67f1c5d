// The products of 16-bit matrices.
#include "ffproduct.cuh"

namespace abcd {

abcd_status launch_16(abcd_ctx* ctx, int epi, int shape, const ProductArgs& a) {
  if (epi == kDown8) return launch_product<2, 256, kDown8, false>(ctx, a);   // planned so
  return launch_any<false>(ctx, epi, shape, a);
}

}  // namespace abcd
