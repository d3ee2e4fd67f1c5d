// The end of a block and the start of the next, forward and backward:
//   y = x + s gate after(f), n = before(y)
// with norms after and before of their own kind, xh = (x - mean) rstd, result xh w + b (an RMS norm's mean
// is 0).  With A = s gate w_after and C = s gate b_after: y = x + (A fh + C).  Backward, from dy and dn:
//   g2 = dn w_before, g = dy + r2 (g2 - mean(g2) - yh mean(g2 yh)), dx = g,
//   u = A g, df = r1 (u - mean(u) - fh mean(u fh))       (an RMS norm has no mean(g2), mean(u))
//   dw_before = sum dn yh, db_before = sum dn, and with S1 = sum g, S2 = sum g fh over the rows
//   dw_after = s gate S2, db_after = s gate S1, dgate = s (w_after S2 + b_after S1).
// Backward, y is made again from x and f: as many bytes as reading y, but in 32 bits, so that yh is the
// forward pass's own.
#include <algorithm>

#include "rows.cuh"

namespace abcd {
namespace {

enum { kNone = -1 };                  // beside ABCD_LAYER_NORM and ABCD_RMS_NORM: no norm

struct CloseArgs {
  const void* x;
  const void* f;
  const void* dy;
  const void* dn;
  void* y;                            // backward: dx
  void* n;                            // backward: df
  long long sx, sf, sdy, sdn, sy, sn;
  const void* gate;
  const void* w[2];                   // of after, before
  const void* b[2];
  int kind[2];
  float eps[2];
  float* mean[2];
  float* rstd[2];
  float scale;
  int wide_w;                         // the vectors are fp32 whatever the matrices' type
  long long rows;
  int cols;
  float* part;                        // [grid][4][cols]: S1, S2, sum dn, sum dn yh of a CTA's rows
};

struct Stat { float mean, rstd; };    // of a row under a norm

// Rows too long for registers: one CTA per row, read again for each use (from L2), element by element.
constexpr int kLongThreads = 1024;

// Statistics of the row whose values are at(c): each thread takes its columns.
template <typename F>
__device__ __forceinline__ Stat long_stat(int kind, float eps, int cols, float2 (*red)[32], F&& at) {
  float s = 0.f, q = 0.f, e = 0.f;
  if (kind == ABCD_RMS_NORM) {
    for (int c = threadIdx.x; c < cols; c += kLongThreads) {
      const float v = at(c);
      q += v * v;
    }
    row_sum2<kLongThreads>(q, e, red, 1);
    __syncthreads();
    return Stat{0.f, rsqrtf(q / (float)cols + eps)};
  }
  for (int c = threadIdx.x; c < cols; c += kLongThreads) s += at(c);
  row_sum2<kLongThreads>(s, q, red, 0);
  const float about = s / (float)cols;
  q = 0.f;
  for (int c = threadIdx.x; c < cols; c += kLongThreads) {
    const float d = at(c) - about;
    q += d * d;
    e += d;
  }
  row_sum2<kLongThreads>(q, e, red, 1);
  __syncthreads();
  e /= (float)cols;
  return Stat{about + e, rstd_of(q / (float)cols, e, eps)};
}

template <typename T>
__device__ __forceinline__ float weight_at(const void* w, int wide, int c, float none) {
  float v[1];
  load_weight<T, 1>(v, w, wide, c, 1, none);
  return v[0];
}
// A and C of a column.
template <typename T> __device__ __forceinline__ float2 factors_at(const CloseArgs& a, int c) {
  const float g = a.scale * weight_at<T>(a.gate, a.wide_w, c, 1.f);
  return make_float2(g * weight_at<T>(a.w[0], a.wide_w, c, 1.f), g * weight_at<T>(a.b[0], a.wide_w, c, 0.f));
}
// y of an element: the forward pass's and the backward pass's, bit for bit.
__device__ __forceinline__ float close_value(float x, float fh, float A, float C) { return __fadd_rn(x, __fmaf_rn(A, fh, C)); }

template <typename T>
__global__ void __launch_bounds__(kLongThreads) close_fwd_long_kernel(const __grid_constant__ CloseArgs a) {
  pdl_wait();
  __shared__ float2 red[2][32];
  for (long long r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const T* x = (const T*)a.x + r * a.sx;
    const T* f = (const T*)a.f + r * a.sf;
    T* y = (T*)a.y + r * a.sy;
    T* n = (T*)a.n + r * a.sn;
    Stat first{0.f, 1.f}, second{0.f, 1.f};
    if (a.kind[0] != kNone) first = long_stat(a.kind[0], a.eps[0], a.cols, red, [&](int c) { return to_f32(f[c]); });
    auto value = [&](int c) {
      const float2 k = factors_at<T>(a, c);
      return close_value(to_f32(x[c]), (to_f32(f[c]) - first.mean) * first.rstd, k.x, k.y);
    };
    if (a.kind[1] != kNone) second = long_stat(a.kind[1], a.eps[1], a.cols, red, value);
    for (int c = threadIdx.x; c < a.cols; c += kLongThreads) {
      const float v = value(c);
      if (a.kind[1] != kNone)
        n[c] = from_f32<T>((v - second.mean) * second.rstd * weight_at<T>(a.w[1], a.wide_w, c, 1.f) + weight_at<T>(a.b[1], a.wide_w, c, 0.f));
      y[c] = from_f32<T>(v);
    }
    if (threadIdx.x == 0) {
      const Stat s[2] = {first, second};
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        if (a.mean[k]) a.mean[k][r] = s[k].mean;
        if (a.rstd[k]) a.rstd[k][r] = s[k].rstd;
      }
    }
  }
}

// The statistics that the forward pass left of a row.
__device__ __forceinline__ Stat stat_of(const CloseArgs& a, int k, long long r) {
  if (a.kind[k] == kNone) return Stat{0.f, 1.f};
  return Stat{a.kind[k] == ABCD_LAYER_NORM ? a.mean[k][r] : 0.f, a.rstd[k][r]};
}

template <typename T>
__global__ void __launch_bounds__(kLongThreads) close_bwd_long_kernel(const __grid_constant__ CloseArgs a) {
  pdl_wait();
  __shared__ float2 red[2][32];
  float* part = a.part + (long long)blockIdx.x * 4 * a.cols;
  for (int c = threadIdx.x; c < 4 * a.cols; c += kLongThreads) part[c] = 0.f;
  __syncthreads();
  const float inv = 1.f / (float)a.cols;
  for (long long r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const T* x = (const T*)a.x + r * a.sx;
    const T* f = (const T*)a.f + r * a.sf;
    const T* dy = (const T*)a.dy + r * a.sdy;
    const T* dn = (const T*)a.dn + r * a.sdn;
    T* dx = (T*)a.y + r * a.sy;
    T* df = (T*)a.n + r * a.sn;
    const Stat first = stat_of(a, 0, r), second = stat_of(a, 1, r);
    struct Value { float fh, yh, g2, dn; float2 k; };
    auto value = [&](int c) {
      Value v;
      v.k = factors_at<T>(a, c);
      v.fh = (to_f32(f[c]) - first.mean) * first.rstd;
      v.yh = (close_value(to_f32(x[c]), v.fh, v.k.x, v.k.y) - second.mean) * second.rstd;
      v.dn = a.dn ? to_f32(dn[c]) : 0.f;
      v.g2 = v.dn * weight_at<T>(a.w[1], a.wide_w, c, 1.f);
      return v;
    };
    float s1 = 0.f, s2 = 0.f, t1 = 0.f, t2 = 0.f;
    if (a.dn) {
      for (int c = threadIdx.x; c < a.cols; c += kLongThreads) {
        const Value v = value(c);
        s1 += v.g2;
        s2 += v.g2 * v.yh;
        part[2 * (long long)a.cols + c] += v.dn;
        part[3 * (long long)a.cols + c] += v.dn * v.yh;
      }
      row_sum2<kLongThreads>(s1, s2, red, 0);
      s1 *= a.kind[1] == ABCD_LAYER_NORM ? inv : 0.f;
      s2 *= inv;
    }
    auto gradient = [&](int c, const Value& v) {
      return (a.dy ? to_f32(dy[c]) : 0.f) + (a.dn ? second.rstd * (v.g2 - s1 - v.yh * s2) : 0.f);
    };
    for (int c = threadIdx.x; c < a.cols; c += kLongThreads) {
      const Value v = value(c);
      const float g = gradient(c, v), u = v.k.x * g;
      t1 += u;
      t2 += u * v.fh;
      part[c] += g;
      part[a.cols + (long long)c] += g * v.fh;
    }
    if (a.kind[0] != kNone) {
      row_sum2<kLongThreads>(t1, t2, red, 1);
      t1 *= a.kind[0] == ABCD_LAYER_NORM ? inv : 0.f;
      t2 *= inv;
    } else {
      t1 = t2 = 0.f;
      __syncthreads();
    }
    for (int c = threadIdx.x; c < a.cols; c += kLongThreads) {
      const Value v = value(c);
      const float g = gradient(c, v);
      if (a.n) df[c] = from_f32<T>(first.rstd * (v.k.x * g - t1 - v.fh * t2));
      if (a.y) dx[c] = from_f32<T>(g);
    }
    __syncthreads();
  }
}

struct CloseSums {
  const float* part;
  int ctas, cols, wide_w;
  float scale;
  const void* gate;
  const void* w;
  const void* b;
  void* to[5];                        // dgate, dafter_weight, dafter_bias, dbefore_weight, dbefore_bias
};

// The vectors' gradients from the CTAs' sums: eight columns a CTA, whose lanes are the four sums of each;
// 32 runs of consecutive CTAs are added side by side and then in their order.
template <typename T>
__global__ void __launch_bounds__(1024) close_sum_kernel(const __grid_constant__ CloseSums a) {
  pdl_wait();
  __shared__ float run[32][33];
  const int lane = threadIdx.x & 31, k = threadIdx.x / 32, which = lane / 8, c = blockIdx.x * 8 + lane % 8;
  float s = 0.f;
  if (c < a.cols) {
    const float* p = a.part + (long long)which * a.cols + c;
    const int q1 = (int)((long long)a.ctas * (k + 1) / 32);
#pragma unroll 4
    for (int q = (int)((long long)a.ctas * k / 32); q < q1; ++q) s += p[(long long)q * 4 * a.cols];
  }
  run[k][lane] = s;
  __syncthreads();
  if (k) return;
  s = 0.f;
#pragma unroll
  for (int q = 0; q < 32; ++q) s += run[q][lane];
  const float s1 = __shfl_sync(~0u, s, lane % 8), s2 = __shfl_sync(~0u, s, 8 + lane % 8);
  if (c >= a.cols) return;
  auto put = [&](int i, float v) {
    if (!a.to[i]) return;
    if (a.wide_w) ((float*)a.to[i])[c] = v;
    else ((T*)a.to[i])[c] = from_f32<T>(v);
  };
  const float g = a.scale * weight_at<T>(a.gate, a.wide_w, c, 1.f);
  if (which == 0) put(2, g * s1);
  else if (which == 1) put(1, g * s2);
  else if (which == 2) put(4, s);
  else put(3, s);
  if (which == 0) put(0, a.scale * (weight_at<T>(a.w, a.wide_w, c, 1.f) * s2 + weight_at<T>(a.b, a.wide_w, c, 0.f) * s1));
}

constexpr int kCloseCtasPerSm = 2;    // backward, with sums in the workspace

bool vector_ok(const void* p, int dtype) { return ((uintptr_t)p & (elem_size(dtype) - 1)) == 0; }

// Whether a norm's description fits a call (`stats`: the statistics are needed).
bool norm_ok(const abcd_norm* q, int dtype, bool stats, long long rows) {
  if (!q) return true;
  if ((q->kind != ABCD_LAYER_NORM && q->kind != ABCD_RMS_NORM) || !vector_ok(q->weight, dtype) || !vector_ok(q->bias, dtype) ||
      !(q->eps >= 0.f && q->eps < 1e30f) || !vector_ok(q->mean, ABCD_F32) || !vector_ok(q->rstd, ABCD_F32))
    return false;
  if (q->kind == ABCD_RMS_NORM ? q->mean != nullptr : (q->mean == nullptr) != (q->rstd == nullptr)) return false;
  return !stats || rows == 0 || q->rstd;
}

// Whether a result may lie where an operand does: in the same elements, or nowhere near.
bool same_or_apart(const abcd_matrix* result, const abcd_matrix* operand) {
  if (!result || !operand || !overlap(result, operand)) return true;
  return result->data == operand->data && (result->stride == operand->stride || result->rows == 1);
}

void take_norm(CloseArgs& a, int k, const abcd_norm* q) {
  a.kind[k] = q ? q->kind : kNone;
  if (!q) return;
  a.w[k] = q->weight;
  a.b[k] = q->bias;
  a.eps[k] = q->eps;
  a.mean[k] = q->mean;
  a.rstd[k] = q->rstd;
}

}  // namespace
}  // namespace abcd

using namespace abcd;

extern "C" abcd_status abcd_residual_norm_workspace_size(long long rows, long long cols, size_t* bytes) {
  if (!bytes || rows < 0 || rows > kMaxNetRows || cols < 1 || cols > kMaxNetCols) return ABCD_ERR_INVALID_ARG;
  *bytes = kNetHeader + (size_t)std::min<long long>(kCloseCtasPerSm * kNetSms, rows) * 4 * (size_t)cols * sizeof(float);
  return ABCD_OK;
}

extern "C" abcd_status abcd_residual_norm(abcd_ctx* ctx, const abcd_matrix* x, const abcd_matrix* f,
                                          const abcd_norm* after, const abcd_norm* before, const void* gate,
                                          int weight_dtype, float scale, const abcd_matrix* y, const abcd_matrix* n) {
  const char* what = "abcd_residual_norm";
  if (!ctx) return ABCD_ERR_INVALID_ARG;
  if (!matrix_ok(x) || !matrix_ok(f) || !matrix_ok(y) || !same_form(x, f) || !same_form(x, y) ||
      (n && (!matrix_ok(n) || !same_form(x, n))) || (n == nullptr) != (before == nullptr))
    return fail(ctx, ABCD_ERR_INVALID_ARG, "%s: bad matrices", what);
  if ((weight_dtype != ABCD_F32 && weight_dtype != x->dtype) || !vector_ok(gate, weight_dtype) ||
      !norm_ok(after, weight_dtype, false, x->rows) || !norm_ok(before, weight_dtype, false, x->rows))
    return fail(ctx, ABCD_ERR_INVALID_ARG, "%s: bad norm or gate", what);
  if (!(scale > -3e38f && scale < 3e38f)) return fail(ctx, ABCD_ERR_INVALID_ARG, "%s: scale must be finite", what);
  if (!same_or_apart(y, x) || !same_or_apart(y, f) || !same_or_apart(n, x) || !same_or_apart(n, f) || (n && overlap(y, n)))
    return fail(ctx, ABCD_ERR_INVALID_ARG, "%s: an output overlaps an operand or the other output", what);
  if (x->rows == 0) return ABCD_OK;
  CloseArgs a{};
  a.x = x->data; a.f = f->data; a.y = y->data; a.n = n ? n->data : nullptr;
  a.sx = x->stride; a.sf = f->stride; a.sy = y->stride; a.sn = n ? n->stride : 0;
  a.gate = gate;
  take_norm(a, 0, after);
  take_norm(a, 1, before);
  a.scale = scale;
  a.wide_w = weight_dtype == ABCD_F32;
  a.rows = x->rows;
  a.cols = (int)x->cols;
  return with_type(x->dtype, [&](auto t) {
    using T = decltype(t);
    const unsigned grid = (unsigned)std::min<long long>(x->rows, 2LL * ctx->num_sms);
    return check_launch(ctx, "close_fwd_long_kernel", launch_pdl(close_fwd_long_kernel<T>, dim3(grid), dim3(kLongThreads), 0, ctx->stream, a));
  });
}

extern "C" abcd_status abcd_residual_norm_backward(abcd_ctx* ctx, const abcd_matrix* dy, const abcd_matrix* dn,
                                                   const abcd_matrix* x, const abcd_matrix* f, const abcd_norm* after,
                                                   const abcd_norm* before, const void* gate, int weight_dtype, float scale,
                                                   const abcd_matrix* dx, const abcd_matrix* df, void* dgate,
                                                   void* dafter_weight, void* dafter_bias, void* dbefore_weight,
                                                   void* dbefore_bias) {
  const char* what = "abcd_residual_norm_backward";
  if (!ctx) return ABCD_ERR_INVALID_ARG;
  const auto fits = [&](const abcd_matrix* m) { return matrix_ok(m) && same_form(x, m); };
  if (!matrix_ok(x) || !fits(f) || (dy && !fits(dy)) || (dn && !fits(dn)) || (dx && !fits(dx)) || (df && !fits(df)) ||
      (dn == nullptr) != (before == nullptr) || (!dy && !dn))
    return fail(ctx, ABCD_ERR_INVALID_ARG, "%s: bad matrices", what);
  if ((weight_dtype != ABCD_F32 && weight_dtype != x->dtype) || !vector_ok(gate, weight_dtype) ||
      !norm_ok(after, weight_dtype, true, x->rows) || !norm_ok(before, weight_dtype, true, x->rows))
    return fail(ctx, ABCD_ERR_INVALID_ARG, "%s: bad norm, statistics or gate", what);
  void* const to[5] = {dgate, dafter_weight, dafter_bias, dbefore_weight, dbefore_bias};
  for (const void* p : to)
    if (!vector_ok(p, weight_dtype)) return fail(ctx, ABCD_ERR_INVALID_ARG, "%s: bad gradients", what);
  if ((!after && (dafter_weight || dafter_bias)) || (!before && (dbefore_weight || dbefore_bias)))
    return fail(ctx, ABCD_ERR_INVALID_ARG, "%s: gradients of a norm that is not there", what);
  if (!(scale > -3e38f && scale < 3e38f)) return fail(ctx, ABCD_ERR_INVALID_ARG, "%s: scale must be finite", what);
  bool apart = !dx || !df || !overlap(dx, df);
  for (const abcd_matrix* out : {dx, df})
    for (const abcd_matrix* in : {dy, dn, x, f}) apart = apart && same_or_apart(out, in);
  if (!apart) return fail(ctx, ABCD_ERR_INVALID_ARG, "%s: a gradient overlaps an operand or the other gradient", what);
  CloseArgs a{};
  a.x = x->data; a.f = f->data; a.dy = dy ? dy->data : nullptr; a.dn = dn ? dn->data : nullptr;
  a.y = dx ? dx->data : nullptr; a.n = df ? df->data : nullptr;
  a.sx = x->stride; a.sf = f->stride; a.sdy = dy ? dy->stride : 0; a.sdn = dn ? dn->stride : 0;
  a.sy = dx ? dx->stride : 0; a.sn = df ? df->stride : 0;
  a.gate = gate;
  take_norm(a, 0, after);
  take_norm(a, 1, before);
  a.scale = scale;
  a.wide_w = weight_dtype == ABCD_F32;
  a.rows = x->rows;
  a.cols = (int)x->cols;
  a.part = (float*)(ctx->net_base + kNetHeader);
  const int ctas = (int)std::min<long long>(x->rows, (long long)kCloseCtasPerSm * std::min(ctx->num_sms, kNetSms));
  const size_t need = kNetHeader + (size_t)ctas * 4 * (size_t)x->cols * sizeof(float);
  if (need > ctx->net_bytes)
    return fail(ctx, ABCD_ERR_WORKSPACE, "%s: the network workspace has %zu bytes, needs %zu", what, ctx->net_bytes, need);
  return with_type(x->dtype, [&](auto t) {
    using T = decltype(t);
    if (ctas > 0) {
      const abcd_status st = check_launch(ctx, "close_bwd_long_kernel", launch_pdl(close_bwd_long_kernel<T>, dim3(ctas), dim3(kLongThreads), 0, ctx->stream, a));
      if (st != ABCD_OK) return st;
    }
    if (std::all_of(to, to + 5, [](void* p) { return !p; })) return ABCD_OK;
    CloseSums s{a.part, ctas, a.cols, a.wide_w, scale, gate, a.w[0], a.b[0], {}};
    std::copy(to, to + 5, s.to);
    return check_launch(ctx, "close_sum_kernel", launch_pdl(close_sum_kernel<T>, dim3((unsigned)((a.cols + 7) / 8)), dim3(1024), 0, ctx->stream, s));
  });
}
