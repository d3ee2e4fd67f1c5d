// Gated feed-forward layer, forward and backward:
//   G = x Wg^T, U = x Wu^T, H = act(G) U, y = H Wd^T
//   dH = dy Wd, dU = dH act(G), dG = dH U act'(G), dx = dG Wg + dU Wu,
//   dWg = dG^T x, dWu = dU^T x, dWd = dy^T H.
// Both projections, the activation and their product are one kernel, and so are dH and what becomes
// of it.
#include <algorithm>

#include "network.cuh"

namespace abcd {
namespace {

// element (i, k) at p[i * si + k * sk]
struct Operand {
  const void* p;
  long long si, sk;
};

struct ProductArgs {
  Operand a[2], b[2];
  int pairs;                 // products that are added up (of kUp: the two that are gated)
  long long m, n, k;
  void* c;
  long long sc;
  const void* gate;          // kDown: the saved projections
  const void* up;
  void* gate_out;            // kUp: G and U, or NULL; kDown: dG and dU (row stride sc)
  void* up_out;
  long long sg, su, sgo, suo;
  int act;
};

enum { kPlain, kUp, kDown };
constexpr int kTile64 = 64, kStep = 16;

__device__ __forceinline__ float act_value(float z, int act) {
  if (act == ABCD_SILU) return z / (1.f + __expf(-z));
  if (act == ABCD_GELU) return z * (0.5f * (1.f + erff(z * 0.70710678f)));
  return fmaxf(z, 0.f);
}

__device__ __forceinline__ float act_slope(float z, int act) {
  if (act == ABCD_SILU) {
    const float s = 1.f / (1.f + __expf(-z));
    return s * (1.f + z * (1.f - s));
  }
  if (act == ABCD_GELU) return 0.5f * (1.f + erff(z * 0.70710678f)) + z * 0.39894228f * __expf(-0.5f * z * z);
  return z > 0.f ? 1.f : 0.f;
}

// 64 x 64 outputs per CTA, 4 x 4 per thread.
template <typename T, int MODE>
__global__ void __launch_bounds__(256) product_kernel(const __grid_constant__ ProductArgs a) {
  pdl_wait();
  __shared__ float sa[kStep][kTile64 + 1], sb[2][kStep][kTile64 + 1];
  const long long m0 = (long long)blockIdx.y * kTile64, n0 = (long long)blockIdx.x * kTile64;
  const int tm = threadIdx.x / 16, tn = threadIdx.x % 16;
  float acc[2][4][4] = {};
  for (int pair = 0; pair < (MODE == kUp ? 1 : a.pairs); ++pair)
    for (long long k0 = 0; k0 < a.k; k0 += kStep) {
      for (int q = threadIdx.x; q < kTile64 * kStep; q += 256) {
        const int i = q / kStep, k = q % kStep;
        const bool in = k0 + k < a.k;
        sa[k][i] = in && m0 + i < a.m ? to_f32(((const T*)a.a[pair].p)[(m0 + i) * a.a[pair].si + (k0 + k) * a.a[pair].sk]) : 0.f;
        for (int s = 0; s < (MODE == kUp ? 2 : 1); ++s) {
          const Operand& b = a.b[MODE == kUp ? s : pair];
          sb[s][k][i] = in && n0 + i < a.n ? to_f32(((const T*)b.p)[(n0 + i) * b.si + (k0 + k) * b.sk]) : 0.f;
        }
      }
      __syncthreads();
#pragma unroll
      for (int k = 0; k < kStep; ++k)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int s = 0; s < (MODE == kUp ? 2 : 1); ++s)
              acc[s][i][j] += sa[k][tm * 4 + i] * sb[s][k][tn * 4 + j];
      __syncthreads();
    }
  for (int i = 0; i < 4; ++i)
    for (int j = 0; j < 4; ++j) {
      const long long m = m0 + tm * 4 + i, n = n0 + tn * 4 + j;
      if (m >= a.m || n >= a.n) continue;
      T* c = (T*)a.c + m * a.sc + n;
      if (MODE == kPlain) *c = from_f32<T>(acc[0][i][j]);
      if (MODE == kUp) {
        *c = from_f32<T>(act_value(acc[0][i][j], a.act) * acc[1][i][j]);
        if (a.gate_out) {
          ((T*)a.gate_out)[m * a.sgo + n] = from_f32<T>(acc[0][i][j]);
          ((T*)a.up_out)[m * a.suo + n] = from_f32<T>(acc[1][i][j]);
        }
      }
      if (MODE == kDown) {
        const float z = to_f32(((const T*)a.gate)[m * a.sg + n]), u = to_f32(((const T*)a.up)[m * a.su + n]);
        const float h = act_value(z, a.act);
        *c = from_f32<T>(h * u);
        ((T*)a.gate_out)[m * a.sgo + n] = from_f32<T>(acc[0][i][j] * u * act_slope(z, a.act));
        ((T*)a.up_out)[m * a.suo + n] = from_f32<T>(acc[0][i][j] * h);
      }
    }
}

template <int MODE>
abcd_status product(abcd_ctx* ctx, int dtype, const ProductArgs& a) {
  const dim3 grid((unsigned)((a.n + kTile64 - 1) / kTile64), (unsigned)((a.m + kTile64 - 1) / kTile64));
  return with_type(dtype, [&](auto t) {
    return check_launch(ctx, "product_kernel",
                        launch_pdl(product_kernel<decltype(t), MODE>, grid, dim3(256), 0, ctx->stream, a));
  });
}

Operand rows_of(const abcd_matrix* m) { return Operand{m->data, m->stride, 1}; }
Operand cols_of(const abcd_matrix* m) { return Operand{m->data, 1, m->stride}; }

// The scratch of one call: the hidden matrix, dG and dU.
size_t ff_scratch(long long rows, long long ff, int dtype) {
  return 3 * net_align((size_t)rows * (size_t)ff * elem_size(dtype));
}

bool shape_is(const abcd_matrix* m, int dtype, long long rows, long long cols) {
  return matrix_ok(m) && m->dtype == dtype && m->rows == rows && m->cols == cols;
}

}  // namespace

int norm_bwd_ctas(int num_sms);   // layernorm.cu

}  // namespace abcd

using namespace abcd;

extern "C" abcd_status abcd_network_workspace_size(long long rows, long long cols, long long ff,
                                                   int dtype, size_t* bytes) {
  if (!bytes || rows < 0 || rows > kMaxNetRows || cols < 1 || cols > kMaxNetCols || ff < 0 ||
      ff > kMaxNetCols || !dtype_ok(dtype))
    return ABCD_ERR_INVALID_ARG;
  int sms = 0;
  if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, 0) != cudaSuccess) sms = 160;
  *bytes = std::max((size_t)norm_bwd_ctas(sms) * 2 * (size_t)cols * sizeof(float),
                    ff_scratch(rows, ff, dtype));
  return ABCD_OK;
}

extern "C" abcd_status abcd_set_network_workspace(abcd_ctx* ctx, void* ptr, size_t bytes) {
  if (!ctx) return ABCD_ERR_INVALID_ARG;
  if (!ptr || ((uintptr_t)ptr & 255))
    return fail(ctx, ABCD_ERR_INVALID_ARG, "the network workspace must be a 256-byte aligned device pointer");
  ctx->net_base = (char*)ptr;
  ctx->net_bytes = bytes;
  return ABCD_OK;
}

extern "C" abcd_status abcd_gated_ff(abcd_ctx* ctx, const abcd_matrix* x, const abcd_matrix* w_gate,
                                     const abcd_matrix* w_up, const abcd_matrix* w_down,
                                     int activation, const abcd_matrix* y, const abcd_matrix* gate,
                                     const abcd_matrix* up) {
  if (!ctx) return ABCD_ERR_INVALID_ARG;
  if (!matrix_ok(x) || !matrix_ok(w_gate)) return fail(ctx, ABCD_ERR_INVALID_ARG, "abcd_gated_ff: bad x or w_gate");
  const long long m = x->rows, d = x->cols, f = w_gate->rows;
  if (f < 1 || f > kMaxNetCols || !shape_is(w_gate, x->dtype, f, d) || !shape_is(w_up, x->dtype, f, d) ||
      !shape_is(w_down, x->dtype, d, f))
    return fail(ctx, ABCD_ERR_INVALID_ARG, "abcd_gated_ff: the weights do not fit x");
  if (!shape_is(y, x->dtype, m, d) || (gate == nullptr) != (up == nullptr) ||
      (gate && (!shape_is(gate, x->dtype, m, f) || !shape_is(up, x->dtype, m, f))))
    return fail(ctx, ABCD_ERR_INVALID_ARG, "abcd_gated_ff: the outputs do not fit x and the weights");
  if (activation < ABCD_SILU || activation > ABCD_RELU)
    return fail(ctx, ABCD_ERR_INVALID_ARG, "abcd_gated_ff: unknown activation");
  if (m == 0) return ABCD_OK;
  const size_t need = ff_scratch(m, f, x->dtype);
  if (need > ctx->net_bytes)
    return fail(ctx, ABCD_ERR_WORKSPACE, "abcd_gated_ff: the network workspace has %zu bytes, needs %zu", ctx->net_bytes, need);
  const abcd_matrix h{ctx->net_base, m, f, f, x->dtype};
  ProductArgs a{};
  a.a[0] = rows_of(x);
  a.b[0] = rows_of(w_gate);
  a.b[1] = rows_of(w_up);
  a.m = m; a.n = f; a.k = d;
  a.c = h.data; a.sc = f;
  a.act = activation;
  if (gate) {
    a.gate_out = gate->data; a.sgo = gate->stride;
    a.up_out = up->data; a.suo = up->stride;
  }
  abcd_status st = product<kUp>(ctx, x->dtype, a);
  if (st != ABCD_OK) return st;
  ProductArgs b{};
  b.a[0] = rows_of(&h);
  b.b[0] = rows_of(w_down);
  b.pairs = 1;
  b.m = m; b.n = d; b.k = f;
  b.c = y->data; b.sc = y->stride;
  return product<kPlain>(ctx, x->dtype, b);
}

extern "C" abcd_status abcd_gated_ff_backward(abcd_ctx* ctx, const abcd_matrix* dy,
                                              const abcd_matrix* x, const abcd_matrix* w_gate,
                                              const abcd_matrix* w_up, const abcd_matrix* w_down,
                                              int activation, const abcd_matrix* gate,
                                              const abcd_matrix* up, const abcd_matrix* dx,
                                              const abcd_matrix* dw_gate, const abcd_matrix* dw_up,
                                              const abcd_matrix* dw_down) {
  const char* what = "abcd_gated_ff_backward";
  if (!ctx) return ABCD_ERR_INVALID_ARG;
  if (!matrix_ok(x) || !matrix_ok(w_gate)) return fail(ctx, ABCD_ERR_INVALID_ARG, "%s: bad x or w_gate", what);
  const long long m = x->rows, d = x->cols, f = w_gate->rows;
  const int t = x->dtype;
  if (f < 1 || f > kMaxNetCols || !shape_is(w_gate, t, f, d) || !shape_is(w_up, t, f, d) || !shape_is(w_down, t, d, f))
    return fail(ctx, ABCD_ERR_INVALID_ARG, "%s: the weights do not fit x", what);
  if (!shape_is(dy, t, m, d) || !shape_is(gate, t, m, f) || !shape_is(up, t, m, f))
    return fail(ctx, ABCD_ERR_INVALID_ARG, "%s: dy, gate or up do not fit x and the weights", what);
  if ((dx && !shape_is(dx, t, m, d)) || (dw_gate && !shape_is(dw_gate, t, f, d)) ||
      (dw_up && !shape_is(dw_up, t, f, d)) || (dw_down && !shape_is(dw_down, t, d, f)))
    return fail(ctx, ABCD_ERR_INVALID_ARG, "%s: the gradients do not fit x and the weights", what);
  if (activation < ABCD_SILU || activation > ABCD_RELU)
    return fail(ctx, ABCD_ERR_INVALID_ARG, "%s: unknown activation", what);
  const size_t need = ff_scratch(m, f, t);
  if (need > ctx->net_bytes)
    return fail(ctx, ABCD_ERR_WORKSPACE, "%s: the network workspace has %zu bytes, needs %zu", what, ctx->net_bytes, need);
  const size_t one = need / 3;
  const abcd_matrix h{ctx->net_base, m, f, f, t}, dg{ctx->net_base + one, m, f, f, t},
      du{ctx->net_base + 2 * one, m, f, f, t};
  abcd_status st = ABCD_OK;
  if (m > 0) {
    ProductArgs a{};
    a.a[0] = rows_of(dy);
    a.b[0] = cols_of(w_down);
    a.pairs = 1;
    a.m = m; a.n = f; a.k = d;
    a.c = h.data; a.sc = f;
    a.gate = gate->data; a.sg = gate->stride;
    a.up = up->data; a.su = up->stride;
    a.gate_out = dg.data; a.sgo = f;
    a.up_out = du.data; a.suo = f;
    a.act = activation;
    st = product<kDown>(ctx, t, a);
    if (st != ABCD_OK) return st;
    if (dx) {
      ProductArgs b{};
      b.a[0] = rows_of(&dg); b.a[1] = rows_of(&du);
      b.b[0] = cols_of(w_gate); b.b[1] = cols_of(w_up);
      b.pairs = 2;
      b.m = m; b.n = d; b.k = f;
      b.c = dx->data; b.sc = dx->stride;
      if ((st = product<kPlain>(ctx, t, b)) != ABCD_OK) return st;
    }
  }
  const abcd_matrix* left[3] = {&dg, &du, dy};
  const abcd_matrix* right[3] = {x, x, &h};
  const abcd_matrix* out[3] = {dw_gate, dw_up, dw_down};
  for (int k = 0; k < 3; ++k) {
    if (!out[k]) continue;
    ProductArgs b{};
    b.a[0] = cols_of(left[k]);
    b.b[0] = cols_of(right[k]);
    b.pairs = 1;
    b.m = out[k]->rows; b.n = out[k]->cols; b.k = m;
    b.c = out[k]->data; b.sc = out[k]->stride;
    if ((st = product<kPlain>(ctx, t, b)) != ABCD_OK) return st;
  }
  return ABCD_OK;
}
