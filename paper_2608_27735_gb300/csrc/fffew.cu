// The gated feed-forward layer's forward pass for up to kFewRows tokens: two kernels without tensor
// cores.
//
// What bounds it: the weights' bytes, each read once, and latency; with so few rows a tile of the
// tensor cores' products is nearly empty, and its staging costs more than the sums.  Layout: one, two,
// four or eight warps per hidden unit (both of its weight rows) and then per output column (one row),
// so that a lane has about four pieces of 16 bytes of a row in flight; it multiplies them with the
// tokens' (from L1) into 32-bit sums, and the lanes' and warps' are added in a fixed order.  The second
// kernel may start while the first runs: it asks for its weight row, which the first does not write,
// before it waits for the hidden matrix.  1 x 1,024 x 4,096 bf16 takes 6.1 and 4.4 us with its weights
// in L2; the call is then the host's time.  Two tokens take 8.9 us, four
// 13.8, eight 21.7: each lane converts and multiplies every weight once per token.  Nine take 25.7 on the
// tensor cores, of which 3 join the splits.  Weight rows that are not whole pieces on 16-byte boundaries go
// element by element: 1, 4 and 8 tokens of 1,025 x 4,097 bf16 take 15, 29 and 50 us.
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
  int share;                          // warps of a unit
  long long sx, sw[2], sy, ssaved[2];
};

constexpr int kFewWarps = 8;          // of a CTA
constexpr int kFlight = 4;            // a lane's pieces of a weight row that are in flight at once

// ROWS: tokens that the registers take (1, 2, 4 or 8); VEC: pieces of 16 bytes, else of one element.
template <typename T, int MATS, int ROWS, bool VEC>
__global__ void __launch_bounds__(32 * kFewWarps) few_kernel(const __grid_constant__ FewArgs a) {
  constexpr int V = VEC ? 16 / sizeof(T) : 1;
  using P = Pack<T, V>;
  __shared__ float parts[kFewWarps][MATS][ROWS];
  const int lane = threadIdx.x & 31, warp = threadIdx.x / 32;
  const int unit = blockIdx.x * (kFewWarps / a.share) + warp / a.share, part = warp % a.share;
  const bool in = unit < a.n;
  const int first = (part * 32 + lane) * V, step = 32 * V * a.share;
  const T* w[MATS];
#pragma unroll
  for (int q = 0; q < MATS; ++q) w[q] = (const T*)a.w[q] + (long long)(in ? unit : 0) * a.sw[q];
  const int end = in ? a.k : 0;
  float s[MATS][ROWS] = {};
  P piece[MATS][kFlight];
  auto fetch = [&](int k0) {
#pragma unroll
    for (int f = 0; f < kFlight; ++f)
#pragma unroll
      for (int q = 0; q < MATS; ++q)
        if (k0 + f * step < end) piece[q][f] = *reinterpret_cast<const P*>(w[q] + k0 + f * step);
  };
  // up: the grids before this one may have written the weights, and down's grid may start from here on;
  // down: its weights are not the grid before's, and that grid's own wait has seen the ones before end
  if (MATS == 2) pdl_prologue();
  fetch(first);
  if (MATS == 1) pdl_wait();
  for (int k0 = first; k0 < end; k0 += kFlight * step) {
    if (k0 > first) fetch(k0);
#pragma unroll
    for (int f = 0; f < kFlight; ++f) {
      const int k = k0 + f * step;
      if (k >= end) break;
#pragma unroll
      for (int r = 0; r < ROWS; ++r) {
        P x;
        const T* from = (const T*)a.x + (r < a.rows ? r : 0) * a.sx + k;
        if (a.x_vec) {
          x = *reinterpret_cast<const P*>(from);
        } else {
#pragma unroll
          for (int e = 0; e < V; ++e) x.v[e] = from[e];
        }
#pragma unroll
        for (int q = 0; q < MATS; ++q)
#pragma unroll
          for (int e = 0; e < V; ++e) s[q][r] += to_f32(piece[q][f].v[e]) * to_f32(x.v[e]);
      }
    }
  }
#pragma unroll
  for (int q = 0; q < MATS; ++q)
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
#pragma unroll
      for (int o = 16; o; o >>= 1) s[q][r] += __shfl_xor_sync(~0u, s[q][r], o);
      if (lane == 0) parts[warp][q][r] = s[q][r];
    }
  if (a.share > 1) __syncthreads();
  else __syncwarp();
  // lane r of a unit's first warp finishes token r
  if (part || lane >= a.rows || !in) return;
  float v[1] = {0.f}, u = 0.f;
  for (int p = 0; p < a.share; ++p) {
    v[0] += parts[warp + p][0][lane];
    if (MATS == 2) u += parts[warp + p][MATS - 1][lane];
  }
  if (MATS == 2) {
    if (a.saved[0]) {
      ((T*)a.saved[0])[lane * a.ssaved[0] + unit] = from_f32<T>(v[0]);
      ((T*)a.saved[1])[lane * a.ssaved[1] + unit] = from_f32<T>(u);
    }
    act_values<sizeof(T) == 4>(v, a.act);
    v[0] *= u;
  }
  ((T*)a.y)[lane * a.sy + unit] = from_f32<T>(v[0]);
}

template <typename T, int MATS>
cudaError_t launch_few(abcd_ctx* ctx, FewArgs a, bool aligned) {
  constexpr int V = 16 / sizeof(T);
  const bool vec = aligned && a.k % V == 0;
  a.share = 1;
  while (a.share < kFewWarps && a.k > 32 * (vec ? V : 1) * kFlight * a.share) a.share *= 2;
  const int units = kFewWarps / a.share;
  const dim3 grid((unsigned)((a.n + units - 1) / units)), block(32 * kFewWarps);
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
