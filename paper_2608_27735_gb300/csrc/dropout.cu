// Dropout from a counter-based generator: y = residual + (kept ? x s : 0), s = 65536 / (65536 - t).
// Element e (row * cols + column) is kept where the 16-bit number e % 8 of block offset + e / 8 of
// Philox4x32-10 is at least t, so that the mask is never stored: the backward pass is the same
// kernel on dy.  One thread takes a block of eight elements.
#include <algorithm>
#include <cmath>

#include "network.cuh"

namespace abcd {
namespace {

struct DropArgs {
  const void* x;
  const void* res;
  void* y;
  long long n;                        // elements
  long long rows;
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

// Drops or scales a block's eight elements by its words w.
__device__ __forceinline__ void drop8(float (&v)[8], const uint4& w, unsigned t, float scale) {
  const unsigned word[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const unsigned u = j & 1 ? word[j / 2] >> 16 : word[j / 2] & 0xffffu;
    v[j] = u >= t ? v[j] * scale : 0.f;
  }
}

// Rows of a multiple of eight elements on 16-byte boundaries (or matrices without gaps, taken as one
// row): a block is one 16-byte access of 16-bit elements, two of 32 bits.
template <typename T>
__global__ void __launch_bounds__(256) dropout_vec_kernel(const __grid_constant__ DropArgs a) {
  pdl_wait();
  using P = Pack<T, 16 / sizeof(T)>;
  constexpr int N = 8 / (16 / sizeof(T));
  const unsigned per_row = (unsigned)(a.cols / 8);
  const long long groups = a.n / 8, step = gridDim.x * 256LL;
  for (long long g = blockIdx.x * 256LL + threadIdx.x; g < groups; g += step) {
    long long row = 0, col = 8 * g;
    if (a.rows > 1) {
      row = groups < (1LL << 32) ? (unsigned)g / per_row : g / per_row;
      col = 8 * (g - row * per_row);
    }
    P px[N], pr[N];
#pragma unroll
    for (int q = 0; q < N; ++q) {
      px[q] = reinterpret_cast<const P*>((const T*)a.x + row * a.sx + col)[q];
      if (a.res) pr[q] = reinterpret_cast<const P*>((const T*)a.res + row * a.sr + col)[q];
    }
    const uint4 w = philox(a.offset + (unsigned long long)g, a.key0, a.key1);
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = to_f32(px[j * N / 8].v[j % (8 / N)]);
    drop8(v, w, a.t, a.scale);
    if (a.res) {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] += to_f32(pr[j * N / 8].v[j % (8 / N)]);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) px[j * N / 8].v[j % (8 / N)] = from_f32<T>(v[j]);
#pragma unroll
    for (int q = 0; q < N; ++q) reinterpret_cast<P*>((T*)a.y + row * a.sy + col)[q] = px[q];
  }
  // matrices without gaps: the last, short block
  if (a.n & 7 && blockIdx.x == 0 && threadIdx.x == 0) {
    const uint4 w = philox(a.offset + (unsigned long long)groups, a.key0, a.key1);
    const int left = (int)(a.n & 7);
    float v[8] = {};
    for (int j = 0; j < left; ++j) v[j] = to_f32(((const T*)a.x)[8 * groups + j]);
    drop8(v, w, a.t, a.scale);
    for (int j = 0; j < left; ++j) {
      if (a.res) v[j] += to_f32(((const T*)a.res)[8 * groups + j]);
      ((T*)a.y)[8 * groups + j] = from_f32<T>(v[j]);
    }
  }
}

// Rows of any length and stride: element by element.
template <typename T>
__global__ void __launch_bounds__(256) dropout_kernel(const __grid_constant__ DropArgs a) {
  pdl_wait();
  const long long groups = (a.n + 7) / 8, step = gridDim.x * 256LL;
  for (long long g = blockIdx.x * 256LL + threadIdx.x; g < groups; g += step) {
    const uint4 w = philox(a.offset + (unsigned long long)g, a.key0, a.key1);
    const long long row0 = a.n < (1LL << 32) ? (unsigned)(8 * g) / (unsigned)a.cols : 8 * g / a.cols;
    const int col0 = (int)(8 * g - row0 * a.cols), left = (int)min(8LL, a.n - 8 * g);
    float v[8];
    long long row = row0;
    int col = col0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      v[j] = j < left ? to_f32(((const T*)a.x)[row * a.sx + col]) : 0.f;
      if (++col == (int)a.cols) { col = 0; ++row; }
    }
    drop8(v, w, a.t, a.scale);
    if (a.res) {
      row = row0;
      col = col0;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if (j < left) v[j] += to_f32(((const T*)a.res)[row * a.sr + col]);
        if (++col == (int)a.cols) { col = 0; ++row; }
      }
    }
    row = row0;
    col = col0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if (j < left) ((T*)a.y)[row * a.sy + col] = from_f32<T>(v[j]);
      if (++col == (int)a.cols) { col = 0; ++row; }
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
  a.rows = x->rows;
  a.cols = x->cols;
  a.sx = x->stride;
  a.sr = res ? res->stride : 0;
  a.sy = y->stride;
  a.offset = offset;
  a.key0 = (unsigned)seed;
  a.key1 = (unsigned)(seed >> 32);
  a.t = (unsigned)std::floor(p * 65536.0 + 0.5);
  a.scale = a.t < 65536u ? (float)(65536.0 / (double)(65536u - a.t)) : 0.f;
  // by vectors go rows in eights on 16-byte boundaries; without gaps the rows are one
  const bool flat = x->stride == x->cols && y->stride == x->cols && (!res || res->stride == x->cols);
  const auto fits = [&](const abcd_matrix* m) {
    return ((uintptr_t)m->data & 15) == 0 && (flat || (x->cols % 8 == 0 && rows_aligned(m, 16)));
  };
  const bool vec = fits(x) && fits(y) && (!res || fits(res));
  if (vec && flat) {
    a.rows = 1;
    a.cols = a.n;
  }
  const long long blocks = std::min<long long>((a.n + 2047) / 2048, 8LL * ctx->num_sms);
  return with_type(x->dtype, [&](auto v) {
    using T = decltype(v);
    return check_launch(ctx, "dropout_kernel",
                        launch_pdl(vec ? dropout_vec_kernel<T> : dropout_kernel<T>, dim3((unsigned)blocks),
                                   dim3(256), 0, ctx->stream, a));
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
