// The gated feed-forward layer's forward pass for up to kFewRows tokens: two kernels without tensor
// cores.
//
// What bounds it: the weights' bytes, each read once, and the calls' latency; with so few rows a
// tile of the tensor cores' products is nearly empty, and its staging costs more than the sums.
// Layout: a warp per hidden unit (both of its weight rows) and then per output column (one row); a
// lane takes every 32nd piece of 16 bytes of a row, multiplies it with the tokens' elements from
// shared memory into 32-bit sums, and the warp adds its lanes'.  The second kernel may start while
// the first runs: it reads its weight row, which the first does not write, before it waits for the
// hidden matrix.  Weight rows that do not start on 16-byte boundaries go element by element.
#include <algorithm>

#include "ffproduct.cuh"

namespace abcd {
namespace {

struct FewArgs {
  const void* x;                      // [rows][k]: the tokens, or the hidden matrix
  const void* w[2];                   // [n][k]: gate and up, or down
  void* y;                            // [rows][n]
  void* saved[2];                     // gate and up, or NULL
  int rows, k, n, act;
  int x_vec;                          // whether x's rows start on 16-byte boundaries
  long long sx, sw[2], sy, ssaved[2];
};

constexpr int kFewThreads = 256;
constexpr int kFewChunk = 8192;       // elements of the tokens in shared memory at a time

// ROWS: tokens that the registers take (1, 2, 4 or 8).
template <typename T, int MATS, int ROWS, bool VEC>
__global__ void __launch_bounds__(kFewThreads) few_kernel(const __grid_constant__ FewArgs a) {
  constexpr int V = VEC ? 16 / sizeof(T) : 1;
  using P = Pack<T, V>;
  __shared__ alignas(16) T xs[ROWS][kFewChunk / ROWS];
  constexpr int CHUNK = kFewChunk / ROWS;
  constexpr int kFlight = MATS == 2 ? 4 : 16;          // a lane's pieces of a weight row in flight at once
  const int lane = threadIdx.x & 31;
  const int unit = blockIdx.x * (kFewThreads / 32) + threadIdx.x / 32;
  const bool in = unit < a.n;
  const T* w[MATS];
#pragma unroll
  for (int q = 0; q < MATS; ++q) w[q] = (const T*)a.w[q] + (long long)(in ? unit : 0) * a.sw[q];
  float s[MATS][ROWS] = {};
  P piece[MATS][kFlight];
  auto fetch = [&](int k0, int end) {                  // the lane's pieces from element k0 on
#pragma unroll
    for (int f = 0; f < kFlight; ++f) {
      const int k = k0 + (f * 32 + lane) * V;
      if (!in || k >= end) continue;
#pragma unroll
      for (int q = 0; q < MATS; ++q) {
        if (k + V <= end) {
          piece[q][f] = *reinterpret_cast<const P*>(w[q] + k);
        } else {
#pragma unroll
          for (int e = 0; e < V; ++e) piece[q][f].v[e] = k + e < end ? w[q][k + e] : from_f32<T>(0.f);
        }
      }
    }
  };
  // up: the grids before this one wrote the weights, perhaps, and down's grid may start from here on;
  // down: its weights are not the grid before's, whose own wait has seen the ones before that end
  if (MATS == 2) pdl_prologue();
  fetch(0, min(a.k, CHUNK));
  if (MATS == 1) pdl_wait();
  for (int c0 = 0; c0 < a.k; c0 += CHUNK) {
    const int end = min(a.k, c0 + CHUNK);
    __syncthreads();
    const int n = min(CHUNK, (end - c0 + 32 * V - 1) / (32 * V) * 32 * V);     // whole turns of the warps
#pragma unroll
    for (int r = 0; r < ROWS; ++r)
#pragma unroll 4
      for (int k = threadIdx.x * V; k < n; k += kFewThreads * V) {
        const T* x = (const T*)a.x + r * a.sx + c0 + k;
        const int left = r < a.rows ? end - c0 - k : 0;
        P xv;
        if (VEC && a.x_vec && left >= V) {
          xv = *reinterpret_cast<const P*>(x);
        } else {
#pragma unroll
          for (int e = 0; e < V; ++e) xv.v[e] = e < left ? x[e] : from_f32<T>(0.f);
        }
        *reinterpret_cast<P*>(&xs[r][k]) = xv;
      }
    __syncthreads();
    for (int k0 = c0; k0 < end; k0 += 32 * V * kFlight) {
      if (k0 > 0) fetch(k0, end);
#pragma unroll
      for (int f = 0; f < kFlight; ++f) {
        const int k = k0 + (f * 32 + lane) * V;
        if (!in || k >= end) continue;
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
          const P xv = *reinterpret_cast<const P*>(&xs[r][k - c0]);
#pragma unroll
          for (int q = 0; q < MATS; ++q)
#pragma unroll
            for (int e = 0; e < V; ++e) s[q][r] += to_f32(piece[q][f].v[e]) * to_f32(xv.v[e]);
        }
      }
    }
  }
#pragma unroll
  for (int q = 0; q < MATS; ++q)
#pragma unroll
    for (int r = 0; r < ROWS; ++r)
#pragma unroll
      for (int o = 16; o; o >>= 1) s[q][r] += __shfl_xor_sync(~0u, s[q][r], o);
  // lane r writes token r
#pragma unroll
  for (int r = 0; r < ROWS; ++r) {
    if (lane != r || r >= a.rows || !in) continue;
    float v[1] = {s[0][r]};
    if (MATS == 2) {
      const float u = s[MATS - 1][r];
      if (a.saved[0]) {
        ((T*)a.saved[0])[r * a.ssaved[0] + unit] = from_f32<T>(v[0]);
        ((T*)a.saved[1])[r * a.ssaved[1] + unit] = from_f32<T>(u);
      }
      act_values(v, a.act);
      v[0] *= u;
    }
    ((T*)a.y)[r * a.sy + unit] = from_f32<T>(v[0]);
  }
}

template <typename T, int MATS>
cudaError_t launch_few(abcd_ctx* ctx, const FewArgs& a, bool vec) {
  const dim3 grid((unsigned)((a.n + kFewThreads / 32 - 1) / (kFewThreads / 32))), block(kFewThreads);
  auto go = [&](auto* kernel) { return launch_pdl(kernel, grid, block, 0, ctx->stream, a); };
  if (vec) {
    if (a.rows == 1) return go(few_kernel<T, MATS, 1, true>);
    if (a.rows == 2) return go(few_kernel<T, MATS, 2, true>);
    if (a.rows <= 4) return go(few_kernel<T, MATS, 4, true>);
    return go(few_kernel<T, MATS, 8, true>);
  }
  if (a.rows == 1) return go(few_kernel<T, MATS, 1, false>);
  if (a.rows <= 4) return go(few_kernel<T, MATS, 4, false>);
  return go(few_kernel<T, MATS, 8, false>);
}

}  // namespace

// The layer's forward pass for few tokens; the arguments have been checked, hidden is scratch of
// rows x ff (in eights) elements of the matrices' type.
abcd_status few_tokens(abcd_ctx* ctx, const abcd_matrix* x, const abcd_matrix* w_gate, const abcd_matrix* w_up,
                       const abcd_matrix* w_down, int activation, const abcd_matrix* y, const abcd_matrix* gate,
                       const abcd_matrix* up, void* hidden) {
  const long long ff = w_gate->rows;
  FewArgs a{};
  a.x = x->data;
  a.w[0] = w_gate->data;
  a.w[1] = w_up->data;
  a.y = hidden;
  a.rows = (int)x->rows;
  a.k = (int)x->cols;
  a.n = (int)ff;
  a.act = activation;
  a.x_vec = rows_aligned(x, 16);
  a.sx = x->stride;
  a.sw[0] = w_gate->stride;
  a.sw[1] = w_up->stride;
  const long long pitch = (ff + 7) / 8 * 8;
  a.sy = pitch;
  if (gate) {
    a.saved[0] = gate->data;
    a.saved[1] = up->data;
    a.ssaved[0] = gate->stride;
    a.ssaved[1] = up->stride;
  }
  FewArgs b{};
  b.x = hidden;
  b.w[0] = w_down->data;
  b.y = y->data;
  b.rows = a.rows;
  b.k = (int)ff;
  b.n = (int)x->cols;
  b.x_vec = 1;
  b.sx = pitch;
  b.sw[0] = w_down->stride;
  b.sy = y->stride;
  return with_type(x->dtype, [&](auto t) {
    using T = decltype(t);
    const abcd_status st = check_launch(ctx, "few_kernel", launch_few<T, 2>(ctx, a, rows_aligned(w_gate, 16) && rows_aligned(w_up, 16)));
    if (st != ABCD_OK) return st;
    return check_launch(ctx, "few_kernel", launch_few<T, 1>(ctx, b, rows_aligned(w_down, 16)));
  });
}

}  // namespace abcd
