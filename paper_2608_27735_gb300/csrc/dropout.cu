// Dropout from a counter-based generator: y = residual + (kept ? x s : 0), s = 65536 / (65536 - t).
// Element e (row * cols + column) is kept where the 16-bit number e % 8 of block offset + e / 8 of
// Philox4x32-10 is at least t, so that the mask is never stored: the backward pass is the same
// kernel on dy.  One thread takes a block of eight elements.
#include <cmath>

#include "network.cuh"

namespace abcd {
namespace {

struct DropArgs {
  const void* x;
  const void* res;
  void* y;
  long long n;                        // elements
  long long cols;
  long long sx, sr, sy;               // row strides
  unsigned long long offset;
  unsigned key0, key1;
  unsigned t;
  float scale;
};

// Ten rounds of Philox4x32 (Salmon et al., 2011): two 32 x 32 bit products a round, the key moved on
// by the paper's two Weyl constants.
__device__ __forceinline__ uint4 philox(unsigned long long block, unsigned k0, unsigned k1) {
  uint4 c = make_uint4((unsigned)block, (unsigned)(block >> 32), 0u, 0u);
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const unsigned long long p0 = (unsigned long long)c.x * 0xD2511F53u;
    const unsigned long long p1 = (unsigned long long)c.z * 0xCD9E8D57u;
    c = make_uint4((unsigned)(p1 >> 32) ^ c.y ^ k0, (unsigned)p1, (unsigned)(p0 >> 32) ^ c.w ^ k1, (unsigned)p0);
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return c;
}

template <typename T>
__global__ void __launch_bounds__(256) dropout_kernel(const __grid_constant__ DropArgs a) {
  pdl_wait();
  const long long groups = (a.n + 7) / 8;
  const T* x = (const T*)a.x;
  const T* res = (const T*)a.res;
  T* y = (T*)a.y;
  for (long long g = blockIdx.x * 256LL + threadIdx.x; g < groups; g += gridDim.x * 256LL) {
    const uint4 w = philox(a.offset + (unsigned long long)g, a.key0, a.key1);
    const unsigned word[4] = {w.x, w.y, w.z, w.w};
    long long row = 8 * g / a.cols, col = 8 * g - row * a.cols;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if (8 * g + j < a.n) {
        const unsigned u = j & 1 ? word[j / 2] >> 16 : word[j / 2] & 0xffffu;
        float v = u >= a.t ? to_f32(x[row * a.sx + col]) * a.scale : 0.f;
        if (res) v += to_f32(res[row * a.sr + col]);
        y[row * a.sy + col] = from_f32<T>(v);
        if (++col == a.cols) {
          col = 0;
          ++row;
        }
      }
    }
  }
}

abcd_status drop(abcd_ctx* ctx, const char* what, const abcd_matrix* x, double p,
                 unsigned long long seed, unsigned long long offset, const abcd_matrix* res,
                 const abcd_matrix* y) {
  if (!ctx) return ABCD_ERR_INVALID_ARG;
  if (!matrix_ok(x) || !matrix_ok(y) || !same_form(x, y))
    return fail(ctx, ABCD_ERR_INVALID_ARG, "%s: bad matrices", what);
  if (res && (!matrix_ok(res) || !same_form(x, res)))
    return fail(ctx, ABCD_ERR_INVALID_ARG, "%s: bad residual", what);
  if (!(p >= 0.0 && p <= 1.0)) return fail(ctx, ABCD_ERR_INVALID_ARG, "%s: p must be in [0, 1]", what);
  if (x->rows == 0) return ABCD_OK;
  DropArgs a;
  a.x = x->data;
  a.res = res ? res->data : nullptr;
  a.y = y->data;
  a.n = x->rows * x->cols;
  a.cols = x->cols;
  a.sx = x->stride;
  a.sr = res ? res->stride : 0;
  a.sy = y->stride;
  a.offset = offset;
  a.key0 = (unsigned)seed;
  a.key1 = (unsigned)(seed >> 32);
  a.t = (unsigned)std::floor(p * 65536.0 + 0.5);
  a.scale = a.t < 65536u ? (float)(65536.0 / (double)(65536u - a.t)) : 0.f;
  const long long blocks = std::min<long long>((a.n + 2047) / 2048, 16LL * ctx->num_sms);
  return with_type(x->dtype, [&](auto v) {
    return check_launch(ctx, "dropout_kernel",
                        launch_pdl(dropout_kernel<decltype(v)>, dim3((unsigned)blocks), dim3(256), 0,
                                   ctx->stream, a));
  });
}

}  // namespace
}  // namespace abcd

using namespace abcd;

extern "C" abcd_status abcd_dropout(abcd_ctx* ctx, const abcd_matrix* x, double p,
                                    unsigned long long seed, unsigned long long offset,
                                    const abcd_matrix* residual, const abcd_matrix* y) {
  return drop(ctx, "abcd_dropout", x, p, seed, offset, residual, y);
}

extern "C" abcd_status abcd_dropout_backward(abcd_ctx* ctx, const abcd_matrix* dy, double p,
                                             unsigned long long seed, unsigned long long offset,
                                             const abcd_matrix* dx) {
  return drop(ctx, "abcd_dropout_backward", dy, p, seed, offset, nullptr, dx);
}
