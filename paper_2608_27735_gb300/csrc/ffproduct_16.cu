// The products of 16-bit matrices.
#include "ffproduct.cuh"

namespace abcd {

abcd_status launch_16(abcd_ctx* ctx, int epi, int shape, const ProductArgs& a) {
  if (epi == kDown8) return launch_product<2, 256, kDown8, false>(ctx, a);   // planned so
  if (shape == 0 && a.job[0].n % 8 != 0) {
    if (epi == kUp) return launch_product<2, 256, kUp, false, true>(ctx, a);
    if (epi == kLinear) return launch_product<2, 256, kLinear, false, true>(ctx, a);
  }
  return launch_any<false>(ctx, epi, shape, a);
}

}  // namespace abcd
