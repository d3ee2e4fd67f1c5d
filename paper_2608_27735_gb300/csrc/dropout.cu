// Dropout from a counter-based generator: y = residual + (kept ? x s : 0), s = 65536 / (65536 - t).
// Element e (row * cols + column) is kept where the 16-bit number e % 8 of block offset + e / 8 of
// Philox4x32-10 is at least t, so that the mask is never stored: the backward pass is the same
// kernel on dy.
// Bound by HBM, and not far from it by the generator's arithmetic: 100,000 x 1,024 bf16 with a residual
// 98 us (6.3 TB/s), without one 79 us (5.2 TB/s), half of whose instruction slots are taken.  Element by
// element, with the rows' divisions for each, both took 264 us.
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
  unsigned inverse;                   // floor(2^17 / cols) + 1 where there are fewer than 256 columns
  unsigned long long offset;
  unsigned key[10][2];                // of the generator's rounds
  unsigned t;
  float scale;
};

// Ten rounds of Philox4x32 (Salmon et al., 2011): two 32 x 32 bit products a round; the rounds' keys
// come with the arguments.
__device__ __forceinline__ uint4 philox(unsigned long long block, const DropArgs& a) {
  uint4 c = make_uint4((unsigned)block, (unsigned)(block >> 32), 0u, 0u);
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const unsigned long long p0 = (unsigned long long)c.x * 0xD2511F53u;
    const unsigned long long p1 = (unsigned long long)c.z * 0xCD9E8D57u;
    c = make_uint4((unsigned)(p1 >> 32) ^ c.y ^ a.key[r][0], (unsigned)p1, (unsigned)(p0 >> 32) ^ c.w ^ a.key[r][1], (unsigned)p0);
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
// row): a block is one 16-byte access of 16-bit elements, two of 32 bits.  The next block's are on
// their way while the generator works on this one's.
template <typename T, bool RES>
__global__ void __launch_bounds__(256) dropout_vec_kernel(const __grid_constant__ DropArgs a) {
  pdl_wait();
  using P = Pack<T, 16 / sizeof(T)>;
  constexpr int N = sizeof(T) / 2;                      // accesses of a block
  const unsigned per_row = (unsigned)(a.cols / 8);
  const long long groups = a.n / 8, step = gridDim.x * 256LL;
  struct Block { P x[N], res[N]; long long y; } now, next;
  auto load = [&](long long g, Block& to) {
    if (g >= groups) return;
    long long row = 0, col = 8 * g;
    if (a.rows > 1) {
      row = groups < (1LL << 32) ? (unsigned)g / per_row : g / per_row;
      col = 8 * (g - row * per_row);
    }
    to.y = row * a.sy + col;
#pragma unroll
    for (int q = 0; q < N; ++q) {
      to.x[q] = reinterpret_cast<const P*>((const T*)a.x + row * a.sx + col)[q];
      if (RES) to.res[q] = reinterpret_cast<const P*>((const T*)a.res + row * a.sr + col)[q];
    }
  };
  long long g = blockIdx.x * 256LL + threadIdx.x;
  load(g, now);
  for (; g < groups; g += step) {
    load(g + step, next);
    const uint4 w = philox(a.offset + (unsigned long long)g, a);
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = to_f32(now.x[j * N / 8].v[j % (8 / N)]);
    drop8(v, w, a.t, a.scale);
    if (RES) {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] += to_f32(now.res[j * N / 8].v[j % (8 / N)]);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) now.x[j * N / 8].v[j % (8 / N)] = from_f32<T>(v[j]);
#pragma unroll
    for (int q = 0; q < N; ++q) reinterpret_cast<P*>((T*)a.y + now.y)[q] = now.x[q];
    now = next;
  }
  // matrices without gaps: the last, short block
  if (a.n & 7 && blockIdx.x == 0 && threadIdx.x == 0) {
    const uint4 w = philox(a.offset + (unsigned long long)groups, a);
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

// Rows of any other length and start: a warp takes 32 consecutive blocks, each lane makes one block's
// eight bits of the mask, and the lanes then take consecutive elements, 32 at a time, and the bits from
// the lanes that made them.  An element lies fewer than 256 columns past the span's first, so in its row
// or the next where these are longer; else at / cols = floor(at (floor(2^17 / cols) + 1) / 2^17), since
// at < 511 and the product's excess over at 2^17 / cols is at most at < 2^17 / cols.
// Bound by instructions, most of them addresses, which are therefore one product past the span's own:
// 100,001 x 999 fp32 with a residual, rows 1,000 apart, 195 us (6.2 TB/s); with a division and two
// products of 64 bits each 283, and with registers for five CTAs per SM instead of four 222.  Rows of 16
// bits take as long for half the bytes: 100,001 x 999 bf16 167 us without and 206 with a residual, 1,000,000
// x 59 fp16 with rows 64 apart 109 and 136 (2.2 and 2.6 TB/s).
template <typename T, bool RES>
__global__ void __launch_bounds__(256, 4) dropout_kernel(const __grid_constant__ DropArgs a) {
  pdl_wait();
  const int lane = threadIdx.x & 31;
  const long long spans = (a.n + 255) / 256, step = gridDim.x * 8LL;
  const unsigned cols = (unsigned)a.cols;
  // elements between a row's end and the next row
  const unsigned gap_x = (unsigned)(a.sx - a.cols), gap_r = (unsigned)(a.sr - a.cols), gap_y = (unsigned)(a.sy - a.cols);
  for (long long s = blockIdx.x * 8LL + threadIdx.x / 32; s < spans; s += step) {
    const long long e0 = 256 * s;
    const int left = (int)min(256LL, a.n - e0) - lane;
    const long long row0 = a.n < (1LL << 32) ? (unsigned)e0 / cols : e0 / cols;
    const unsigned at = (unsigned)(e0 - row0 * cols) + lane;
    const T* px = (const T*)a.x + row0 * a.sx + at;
    const T* pr = (const T*)a.res + row0 * a.sr + at;
    T* py = (T*)a.y + row0 * a.sy + at;
    T x[8], res[8];
    unsigned over[8];                   // rows past row0
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      over[k] = cols < 256 ? (at + 32 * k) * a.inverse >> 17 : at + 32 * k >= cols;
      if (32 * k < left) {
        x[k] = px[(unsigned long long)over[k] * gap_x + 32 * k];
        if (RES) res[k] = pr[(unsigned long long)over[k] * gap_r + 32 * k];
      }
    }
    const uint4 w = philox(a.offset + (unsigned long long)(32 * s + lane), a);
    const unsigned word[4] = {w.x, w.y, w.z, w.w};
    unsigned mask = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) mask |= ((j & 1 ? word[j / 2] >> 16 : word[j / 2] & 0xffffu) >= a.t ? 1u : 0u) << j;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const unsigned bits = __shfl_sync(~0u, mask, 4 * k + lane / 8);
      if (32 * k < left) {
        float v = bits >> (lane & 7) & 1 ? to_f32(x[k]) * a.scale : 0.f;
        if (RES) v += to_f32(res[k]);
        py[(unsigned long long)over[k] * gap_y + 32 * k] = from_f32<T>(v);
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
  a.rows = x->rows;
  a.cols = x->cols;
  a.inverse = x->cols < 256 ? (1u << 17) / (unsigned)x->cols + 1 : 0;
  a.sx = x->stride;
  a.sr = res ? res->stride : 0;
  a.sy = y->stride;
  a.offset = offset;
  for (int r = 0; r < 10; ++r) {        // moved on by the paper's two Weyl constants
    a.key[r][0] = (unsigned)seed + (unsigned)r * 0x9E3779B9u;
    a.key[r][1] = (unsigned)(seed >> 32) + (unsigned)r * 0xBB67AE85u;
  }
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
  return with_type(x->dtype, [&](auto v) {
    using T = decltype(v);
    const long long blocks = std::min<long long>((a.n + 2047) / 2048, 8LL * ctx->num_sms);
    auto* kernel = vec ? (res ? dropout_vec_kernel<T, true> : dropout_vec_kernel<T, false>) : (res ? dropout_kernel<T, true> : dropout_kernel<T, false>);
    return check_launch(ctx, "dropout_kernel", launch_pdl(kernel, dim3((unsigned)blocks), dim3(256), 0, ctx->stream, a));
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
