// Layer norm over the rows of a matrix, forward and backward.
//   y = (x - mean) rstd w + b,   rstd = 1 / sqrt(mean((x - mean)^2) + eps)
//   g = dy w, xh = (x - mean) rstd:  dx = rstd (g - mean(g) - xh mean(g xh)),
//   dw = sum_rows dy xh,  db = sum_rows dy.
// The variance is taken from the deviations (a second pass over the row), not from the difference
// of two moments.  The sums over the rows are taken in a fixed order: each CTA adds its rows' terms,
// a second kernel adds the CTAs'.
#include <algorithm>

#include "network.cuh"

namespace abcd {
namespace {

struct NormArgs {
  const void* x;
  const void* dy;
  const void* w;
  const void* b;
  void* y;                            // forward: y; backward: dx
  const void* res;                    // backward: added to dx, or NULL
  float* mean;
  float* rstd;
  float* part;                        // [grid][2][cols] sums of a CTA's rows
  long long rows;
  int cols;
  long long sx, sdy, sy, sres;
  float eps;
};

constexpr int kNormThreads = 256;

// Sum over the CTA's threads, in every thread.
__device__ __forceinline__ float cta_sum(float v, float* red) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) red[threadIdx.x / 32] = v;
  __syncthreads();
  v = 0.f;
#pragma unroll
  for (int k = 0; k < kNormThreads / 32; ++k) v += red[k];
  return v;
}

// One CTA per row.
template <typename T, typename W>
__global__ void __launch_bounds__(kNormThreads) norm_fwd_kernel(const __grid_constant__ NormArgs a) {
  pdl_wait();
  __shared__ float red[kNormThreads / 32];
  for (long long r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const T* x = (const T*)a.x + r * a.sx;
    T* y = (T*)a.y + r * a.sy;
    float s = 0.f;
    for (int c = threadIdx.x; c < a.cols; c += kNormThreads) s += to_f32(x[c]);
    const float mean = cta_sum(s, red) / (float)a.cols;
    float q = 0.f;
    for (int c = threadIdx.x; c < a.cols; c += kNormThreads) {
      const float d = to_f32(x[c]) - mean;
      q += d * d;
    }
    const float rstd = rsqrtf(cta_sum(q, red) / (float)a.cols + a.eps);
    for (int c = threadIdx.x; c < a.cols; c += kNormThreads) {
      const float w = a.w ? to_f32(((const W*)a.w)[c]) : 1.f, b = a.b ? to_f32(((const W*)a.b)[c]) : 0.f;
      y[c] = from_f32<T>((to_f32(x[c]) - mean) * rstd * w + b);
    }
    if (a.mean && threadIdx.x == 0) {
      a.mean[r] = mean;
      a.rstd[r] = rstd;
    }
  }
}

template <typename T, typename W>
__global__ void __launch_bounds__(kNormThreads) norm_bwd_kernel(const __grid_constant__ NormArgs a) {
  pdl_wait();
  __shared__ float red[kNormThreads / 32];
  float* pw = a.part + (long long)blockIdx.x * 2 * a.cols;
  float* pb = pw + a.cols;
  for (int c = threadIdx.x; c < a.cols; c += kNormThreads) pw[c] = pb[c] = 0.f;
  for (long long r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const T* x = (const T*)a.x + r * a.sx;
    const T* dy = (const T*)a.dy + r * a.sdy;
    T* dx = (T*)a.y + r * a.sy;
    const float mean = a.mean[r], rstd = a.rstd[r];
    float s1 = 0.f, s2 = 0.f;
    for (int c = threadIdx.x; c < a.cols; c += kNormThreads) {
      const float d = to_f32(dy[c]), xh = (to_f32(x[c]) - mean) * rstd;
      const float g = a.w ? d * to_f32(((const W*)a.w)[c]) : d;
      s1 += g;
      s2 += g * xh;
      pw[c] += d * xh;
      pb[c] += d;
    }
    s1 = cta_sum(s1, red) / (float)a.cols;
    s2 = cta_sum(s2, red) / (float)a.cols;
    if (a.y)
      for (int c = threadIdx.x; c < a.cols; c += kNormThreads) {
        const float d = to_f32(dy[c]), xh = (to_f32(x[c]) - mean) * rstd;
        const float g = a.w ? d * to_f32(((const W*)a.w)[c]) : d;
        const float res = a.res ? to_f32(((const T*)a.res)[r * a.sres + c]) : 0.f;
        dx[c] = from_f32<T>(rstd * (g - s1 - xh * s2) + res);
      }
  }
}

// dw and db from the CTAs' sums, in the order of the CTAs: one thread per column.
template <typename W>
__global__ void __launch_bounds__(128) norm_sum_kernel(const float* part, int ctas, int cols, W* dw, W* db) {
  pdl_wait();
  const int c = blockIdx.x * 128 + threadIdx.x;
  if (c >= cols) return;
  float w = 0.f, b = 0.f;
  for (int k = 0; k < ctas; ++k) {
    w += part[(long long)k * 2 * cols + c];
    b += part[(long long)k * 2 * cols + cols + c];
  }
  if (dw) dw[c] = from_f32<W>(w);
  if (db) db[c] = from_f32<W>(b);
}

// Calls f(T(), W()) with the matrices' type and the weights'.
template <typename F> abcd_status with_types(int dtype, int wtype, F&& f) {
  return with_type(dtype, [&](auto t) {
    return wtype == ABCD_F32 ? f(t, float()) : f(t, decltype(t)());
  });
}

bool weights_ok(const abcd_matrix* x, int wtype, const void* a, const void* b) {
  return (wtype == ABCD_F32 || wtype == x->dtype) &&
         (((uintptr_t)a | (uintptr_t)b) & (elem_size(wtype) - 1)) == 0;
}

}  // namespace

int norm_bwd_ctas(int num_sms) { return 2 * num_sms; }

}  // namespace abcd

using namespace abcd;

extern "C" abcd_status abcd_layer_norm(abcd_ctx* ctx, const abcd_matrix* x, const void* weight,
                                       const void* bias, int weight_dtype, float eps,
                                       const abcd_matrix* y, float* mean, float* rstd) {
  if (!ctx) return ABCD_ERR_INVALID_ARG;
  if (!matrix_ok(x) || !matrix_ok(y) || !same_form(x, y))
    return fail(ctx, ABCD_ERR_INVALID_ARG, "abcd_layer_norm: bad matrices");
  if (!weights_ok(x, weight_dtype, weight, bias))
    return fail(ctx, ABCD_ERR_INVALID_ARG, "abcd_layer_norm: bad weight or bias");
  if (!(eps >= 0.f && eps < 1e30f) || (mean == nullptr) != (rstd == nullptr))
    return fail(ctx, ABCD_ERR_INVALID_ARG, "abcd_layer_norm: bad eps or statistics");
  if (x->rows == 0) return ABCD_OK;
  const NormArgs a{x->data, nullptr, weight, bias, y->data, nullptr, mean, rstd, nullptr, x->rows,
                   (int)x->cols, x->stride, 0, y->stride, 0, eps};
  const unsigned grid = (unsigned)std::min<long long>(x->rows, 16LL * ctx->num_sms);
  return with_types(x->dtype, weight_dtype, [&](auto t, auto w) {
    return check_launch(ctx, "norm_fwd_kernel",
                        launch_pdl(norm_fwd_kernel<decltype(t), decltype(w)>, dim3(grid),
                                   dim3(kNormThreads), 0, ctx->stream, a));
  });
}

extern "C" abcd_status abcd_layer_norm_backward(abcd_ctx* ctx, const abcd_matrix* dy,
                                                const abcd_matrix* x, const void* weight,
                                                int weight_dtype, const float* mean,
                                                const float* rstd, const abcd_matrix* d_residual,
                                                const abcd_matrix* dx, void* dweight, void* dbias) {
  if (!ctx) return ABCD_ERR_INVALID_ARG;
  if (!matrix_ok(x) || !matrix_ok(dy) || !same_form(x, dy) ||
      (dx && (!matrix_ok(dx) || !same_form(x, dx))) ||
      (d_residual && (!dx || !matrix_ok(d_residual) || !same_form(x, d_residual))))
    return fail(ctx, ABCD_ERR_INVALID_ARG, "abcd_layer_norm_backward: bad matrices");
  if (!weights_ok(x, weight_dtype, weight, nullptr) || !weights_ok(x, weight_dtype, dweight, dbias))
    return fail(ctx, ABCD_ERR_INVALID_ARG, "abcd_layer_norm_backward: bad weight or gradients");
  if (x->rows > 0 && (!mean || !rstd))
    return fail(ctx, ABCD_ERR_INVALID_ARG, "abcd_layer_norm_backward: no statistics");
  const int ctas = (int)std::min<long long>(x->rows, norm_bwd_ctas(std::min(ctx->num_sms, kNetSms)));
  float* part = (float*)(ctx->net_base + kNetHeader);
  const size_t need = kNetHeader + (size_t)ctas * 2 * (size_t)x->cols * sizeof(float);
  if (need > ctx->net_bytes)
    return fail(ctx, ABCD_ERR_WORKSPACE, "abcd_layer_norm_backward: the network workspace has %zu bytes, needs %zu", ctx->net_bytes, need);
  const NormArgs a{x->data, dy->data, weight, nullptr, dx ? dx->data : nullptr,
                   d_residual ? d_residual->data : nullptr, (float*)mean, (float*)rstd,
                   part, x->rows, (int)x->cols, x->stride, dy->stride,
                   dx ? dx->stride : 0, d_residual ? d_residual->stride : 0, 0.f};
  return with_types(x->dtype, weight_dtype, [&](auto t, auto w) {
    abcd_status st = ABCD_OK;
    if (ctas > 0)
      st = check_launch(ctx, "norm_bwd_kernel",
                        launch_pdl(norm_bwd_kernel<decltype(t), decltype(w)>, dim3(ctas),
                                   dim3(kNormThreads), 0, ctx->stream, a));
    if (st != ABCD_OK || (!dweight && !dbias)) return st;
    return check_launch(ctx, "norm_sum_kernel",
                        launch_pdl(norm_sum_kernel<decltype(w)>, dim3((unsigned)((x->cols + 127) / 128)),
                                   dim3(128), 0, ctx->stream, (const float*)part, ctas,
                                   (int)x->cols, (decltype(w)*)dweight, (decltype(w)*)dbias));
  });
}
