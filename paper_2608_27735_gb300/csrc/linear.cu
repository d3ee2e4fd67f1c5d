// Linear layer, forward and backward:
//   z = x W^T + b, y = residual + act(z);   dz = dy act'(z), dx = dz W, dW = dz^T x, db = sum of dz's rows.
// Forward is one product whose epilogue does the rest (ffproduct.cuh, kLinear); up to eight tokens go
// without tensor cores (fffew.cu).  Backward, one pass over dy and z leaves dz as an operand (rounded once to
// the matrices' type, in 32 bits as three terms) and its columns' sums, and both products are one launch.
// 16,384 x 4,096 x 4,096 bf16: forward with residual and z 332 us (1,660 TFLOP/s), the pass over dy and z 67 (6.0
// TB/s), both products 600 (1,830).  100,000 x 256 x 256 bf16: 49 us (5.2 TB/s; six rounds of tiles for 5.1) and 72.
// 20,000 x 59 x 256 fp32 with gelu: 29 and 44 us, two launches (operands, product) and five (operands, dz, dbias, products,
// their parts); the forward product is three rounds of the smallest tile, whose epilogue spills (104 bytes at the 96
// registers that two CTAs an SM leave).
#include "products.cuh"

namespace abcd {

abcd_status few_linear(abcd_ctx* ctx, const abcd_matrix* x, const abcd_matrix* weight, const void* bias, int bias_dtype,
                       int activation, const abcd_matrix* residual, const abcd_matrix* y, const abcd_matrix* z);   // fffew.cu

namespace {

constexpr long long kFewTokens = 8;   // tokens up to which the forward pass goes without tensor cores

struct SlopeArgs {
  const void* dy;
  const void* z;                      // NULL: no activation
  unsigned short* dst;                // dz as an operand, or NULL
  float* part;                        // [grid.y][cols] sums of a CTA's rows, or NULL
  long long rows, sdy, sz, pitch, plane;
  int cols, act, lanes;               // lanes: threads of a row, a power of two, eight columns each
  int vec;                            // rows of dy and z start on 16-byte boundaries
};

template <typename T>
__device__ __forceinline__ void load8(float (&v)[8], const T* p, int left, bool vec) {
  if (vec && left >= 8) {
    constexpr int N = sizeof(T) / 2, V = 16 / sizeof(T);
    using P = Pack<T, V>;
#pragma unroll
    for (int q = 0; q < N; ++q) {
      const P x = reinterpret_cast<const P*>(p)[q];
#pragma unroll
      for (int e = 0; e < V; ++e) v[q * V + e] = to_f32(x.v[e]);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = e < left ? to_f32(p[e]) : 0.f;
  }
}

// dz of eight columns a thread; a CTA takes `lanes` x 8 columns of 256 / lanes rows at a time.
template <typename T>
__global__ void __launch_bounds__(256) slope_kernel(const __grid_constant__ SlopeArgs a) {
  pdl_wait();
  constexpr bool F32 = sizeof(T) == 4;
  __shared__ float sums[256 * 9];
  const int lane = threadIdx.x % a.lanes, group = threadIdx.x / a.lanes, groups = 256 / a.lanes;
  const int c = (blockIdx.x * a.lanes + lane) * 8, left = a.cols - c;
  float db[8] = {};
  if (left > 0)
    for (long long r = (long long)blockIdx.y * groups + group; r < a.rows; r += (long long)gridDim.y * groups) {
      float d[8];
      load8(d, (const T*)a.dy + r * a.sdy + c, left, a.vec);
      if (a.z) {
        float z[8], s[8];
        load8(z, (const T*)a.z + r * a.sz + c, left, a.vec);
        act_slopes<F32, 8, true>(z, s, a.act);
#pragma unroll
        for (int e = 0; e < 8; ++e) d[e] *= s[e];
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) db[e] += d[e];
      if (!a.dst) continue;
      unsigned short* dst = a.dst + r * a.pitch + c;
      if constexpr (F32) {
#pragma unroll
        for (int t = 0; t < 3; ++t) {
          unsigned w[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) w[j] = take_terms(d[2 * j], d[2 * j + 1]);
          *reinterpret_cast<uint4*>(dst + t * a.plane) = make_uint4(w[0], w[1], w[2], w[3]);
        }
      } else {
        Pack<T, 8> q;
#pragma unroll
        for (int e = 0; e < 8; ++e) q.v[e] = from_f32<T>(d[e]);
        *reinterpret_cast<Pack<T, 8>*>(dst) = q;
      }
    }
  if (!a.part) return;
#pragma unroll
  for (int e = 0; e < 8; ++e) sums[threadIdx.x * 9 + e] = db[e];
  __syncthreads();
  // a thread adds a column's groups in their order
  for (int i = threadIdx.x; i < a.lanes * 8; i += 256) {
    const int col = blockIdx.x * a.lanes * 8 + i;
    if (col >= a.cols) break;
    float s = 0.f;
    for (int g = 0; g < groups; ++g) s += sums[(g * a.lanes + i / 8) * 9 + i % 8];
    a.part[(long long)blockIdx.y * a.cols + col] = s;
  }
}

// A bias's gradient from the CTAs' sums: eight columns a CTA, 128 runs of consecutive parts added side by
// side and then in their order (a warp's four in pairs, the warps' one after another).  With 32 columns
// and 32 runs, which are few CTAs and a chain of twenty loads, 256 columns of 640 parts took 5.4 us.
template <typename W>
__global__ void __launch_bounds__(1024) bias_sum_kernel(const float* part, int parts, int cols, W* out) {
  pdl_wait();
  __shared__ float run[32][9];
  const int lane = threadIdx.x % 8, k = threadIdx.x / 8, c = blockIdx.x * 8 + lane;
  float s = 0.f;
  if (c < cols) {
    const int q1 = parts * (k + 1) / 128;
#pragma unroll 5
    for (int q = parts * k / 128; q < q1; ++q) s += part[(long long)q * cols + c];
  }
  s += __shfl_xor_sync(~0u, s, 8);
  s += __shfl_xor_sync(~0u, s, 16);
  if ((threadIdx.x & 31) < 8) run[threadIdx.x / 32][lane] = s;
  __syncthreads();
  if (k || c >= cols) return;
  s = 0.f;
#pragma unroll
  for (int q = 0; q < 32; ++q) s += run[q][lane];
  out[c] = from_f32<W>(s);
}

constexpr int kSlopeCtas = 4 * kNetSms;   // parts of the bias's gradient at most

// A vector as a matrix of one row, for overlap().
abcd_matrix row_of(const void* p, long long n, int dtype) { return abcd_matrix{const_cast<void*>(p), p ? 1LL : 0LL, n, n, dtype}; }

bool bias_ok(const void* bias, int dtype, const abcd_matrix* x) {
  return !bias || ((dtype == ABCD_F32 || dtype == x->dtype) && ((uintptr_t)bias & (elem_size(dtype) - 1)) == 0);
}

}  // namespace
}  // namespace abcd

using namespace abcd;

extern "C" abcd_status abcd_linear_workspace_size(long long rows, long long cols, long long out, int dtype, size_t* bytes) {
  if (!bytes || rows < 0 || rows > kMaxNetRows || cols < 1 || cols > kMaxNetCols || out < 1 || out > kMaxNetCols || !dtype_ok(dtype))
    return ABCD_ERR_INVALID_ARG;
  Scratch s{nullptr};
  s.take(kPartBytes);
  s.take((size_t)kSlopeCtas * (size_t)out * 4);
  s.operand(rows, out, dtype);            // dz
  s.operand(rows, cols, dtype);           // x
  s.operand(out, cols, dtype);            // weight
  *bytes = s.at;
  return ABCD_OK;
}

extern "C" abcd_status abcd_linear(abcd_ctx* ctx, const abcd_matrix* x, const abcd_matrix* weight, const void* bias,
                                   int bias_dtype, int activation, const abcd_matrix* residual, const abcd_matrix* y,
                                   const abcd_matrix* z) {
  const char* what = "abcd_linear";
  if (!ctx) return ABCD_ERR_INVALID_ARG;
  if (!matrix_ok(x) || !matrix_ok(weight)) return fail(ctx, ABCD_ERR_INVALID_ARG, "%s: bad x or weight", what);
  const long long m = x->rows, d = x->cols, n = weight->rows;
  const int t = x->dtype;
  if (n < 1 || n > kMaxNetCols || !shape_is(weight, t, n, d) || !bias_ok(bias, bias_dtype, x))
    return fail(ctx, ABCD_ERR_INVALID_ARG, "%s: the weight or the bias does not fit x", what);
  if (!shape_is(y, t, m, n) || (z && !shape_is(z, t, m, n)) || (residual && !shape_is(residual, t, m, n)))
    return fail(ctx, ABCD_ERR_INVALID_ARG, "%s: the outputs or the residual do not fit x and the weight", what);
  if (activation < ABCD_SILU || activation > ABCD_NO_ACTIVATION)
    return fail(ctx, ABCD_ERR_INVALID_ARG, "%s: unknown activation", what);
  if (m == 0) return ABCD_OK;
  const abcd_matrix b = row_of(bias, n, bias_dtype);
  const bool on_residual = residual && overlap(residual, y) && !(residual->data == y->data && (residual->stride == y->stride || m == 1));
  if (on_residual || same_place({y, z}, {x, weight, &b}) || (z && residual && overlap(z, residual)))
    return fail(ctx, ABCD_ERR_INVALID_ARG, "%s: an output overlaps an operand or the other output", what);
  if (m <= kFewTokens) return few_linear(ctx, x, weight, bias, bias_dtype, activation, residual, y, z);
  Scratch need{nullptr};
  need.take(kPartBytes);
  if (needs_pack(x)) need.operand(m, d, t);
  if (needs_pack(weight)) need.operand(n, d, t);
  abcd_status st = room(ctx, what, need.at);
  if (st != ABCD_OK) return st;
  Scratch s{ctx->net_base};
  s.take(kPartBytes);
  Operands in{s};
  const Operand ox = in.add(x), ow = in.add(weight);
  if ((st = in.pack(ctx, t)) != ABCD_OK) return st;
  const Job job{ox, {ow}, 1, false, false, m, n, d, 1, {out_of(y), residual ? out_of(residual) : Out{}}};
  Hidden hid{};
  hid.act = activation;
  hid.bias = bias;
  hid.wide_bias = bias_dtype == ABCD_F32;
  if (z) hid.out[0] = out_of(z);
  if (residual) hid.saved[0] = out_of(residual);
  // what TMA moves, where rows allow it
  if (!needs_pack(y)) hid.c = stored_in_place(y);
  if (z && !needs_pack(z)) hid.g[0] = stored_in_place(z);
  if (residual && !needs_pack(residual)) hid.in[0] = in_place(residual);
  return run(ctx, t, kLinear, &job, 1, plan(ctx->num_sms, t, kLinear, &job, 1), &hid);
}

extern "C" abcd_status abcd_linear_backward(abcd_ctx* ctx, const abcd_matrix* dy, const abcd_matrix* x,
                                            const abcd_matrix* weight, int activation, const abcd_matrix* z,
                                            const abcd_matrix* dx, const abcd_matrix* dweight, void* dbias, int bias_dtype) {
  const char* what = "abcd_linear_backward";
  if (!ctx) return ABCD_ERR_INVALID_ARG;
  if (!matrix_ok(x) || !matrix_ok(weight)) return fail(ctx, ABCD_ERR_INVALID_ARG, "%s: bad x or weight", what);
  const long long m = x->rows, d = x->cols, n = weight->rows;
  const int t = x->dtype;
  if (n < 1 || n > kMaxNetCols || !shape_is(weight, t, n, d) || !shape_is(dy, t, m, n) || (z && !shape_is(z, t, m, n)))
    return fail(ctx, ABCD_ERR_INVALID_ARG, "%s: the weight, dy or z does not fit x", what);
  if ((dx && !shape_is(dx, t, m, d)) || (dweight && !shape_is(dweight, t, n, d)) || !bias_ok(dbias, bias_dtype, x))
    return fail(ctx, ABCD_ERR_INVALID_ARG, "%s: the gradients do not fit x and the weight", what);
  if (activation < ABCD_SILU || activation > ABCD_NO_ACTIVATION || (activation != ABCD_NO_ACTIVATION && m > 0 && !z))
    return fail(ctx, ABCD_ERR_INVALID_ARG, "%s: unknown activation, or no z", what);
  if (m == 0) {                                   // sums over no rows
    const size_t e = elem_size(t);
    cudaError_t c = cudaSuccess;
    if (dweight) c = cudaMemset2DAsync(dweight->data, (size_t)dweight->stride * e, 0, (size_t)d * e, (size_t)n, ctx->stream);
    if (c == cudaSuccess && dbias) c = cudaMemsetAsync(dbias, 0, (size_t)n * elem_size(bias_dtype), ctx->stream);
    return c == cudaSuccess ? ABCD_OK : fail(ctx, ABCD_ERR_CUDA, "%s: %s", what, cudaGetErrorString(c));
  }
  if (activation == ABCD_NO_ACTIVATION) z = nullptr;
  const abcd_matrix b = row_of(dbias, n, bias_dtype);
  if (same_place({dx, dweight, &b}, {dy, x, weight, z}))
    return fail(ctx, ABCD_ERR_INVALID_ARG, "%s: a gradient overlaps an operand or another gradient", what);
  const bool products = dx || dweight;
  const bool apart = products && (z || needs_pack(dy));      // dz is an operand of its own
  Scratch need{nullptr};
  need.take(kPartBytes);
  if (dbias) need.take((size_t)kSlopeCtas * (size_t)n * 4);
  if (apart) need.operand(m, n, t);
  if (dweight && needs_pack(x)) need.operand(m, d, t);
  if (dx && needs_pack(weight)) need.operand(n, d, t);
  abcd_status st = room(ctx, what, need.at);
  if (st != ABCD_OK) return st;
  Scratch s{ctx->net_base};
  s.take(kPartBytes);
  float* part = dbias ? (float*)s.take((size_t)kSlopeCtas * (size_t)n * 4) : nullptr;
  const Operand odz = apart ? s.operand(m, n, t) : products ? in_place(dy) : Operand{};
  Operands in{s};
  Operand ox{}, ow{};
  if (dweight) ox = in.add(x);
  if (dx) ow = in.add(weight);
  if ((st = in.pack(ctx, t)) != ABCD_OK) return st;
  if (apart || dbias) {
    SlopeArgs a{dy->data, z ? z->data : nullptr, apart ? (unsigned short*)odz.p : nullptr, part, m, dy->stride, z ? z->stride : 0,
                odz.pitch, odz.plane, (int)n, activation, 1, rows_aligned(dy, 16) && (!z || rows_aligned(z, 16))};
    while (a.lanes < 32 && a.lanes * 8 < n) a.lanes *= 2;
    const int groups = 256 / a.lanes;
    const long long across = (n + a.lanes * 8 - 1) / (a.lanes * 8);
    const long long most = std::min<long long>((m + groups - 1) / groups, kSlopeCtas);
    const dim3 grid((unsigned)across, (unsigned)std::max<long long>(1, std::min(most, 8LL * ctx->num_sms / across)));
    st = with_type(t, [&](auto v) {
      return check_launch(ctx, "slope_kernel", launch_pdl(slope_kernel<decltype(v)>, grid, dim3(256), 0, ctx->stream, a));
    });
    if (st == ABCD_OK && dbias)
      st = with_type(bias_dtype, [&](auto v) {
        using W = decltype(v);
        return check_launch(ctx, "bias_sum_kernel", launch_pdl(bias_sum_kernel<W>, dim3((unsigned)((n + 7) / 8)), dim3(1024), 0, ctx->stream,
                                                               (const float*)part, (int)grid.y, (int)n, (W*)dbias));
      });
    if (st != ABCD_OK) return st;
  }
  // planned as for both products, so that no gradient depends on which others are asked for
  const Job all[2] = {Job{odz, {ow}, 1, false, true, m, d, n, 1, {}}, Job{odz, {ox}, 1, true, true, n, d, m, 1, {}}};
  const Plan whole = plan(ctx->num_sms, t, kPlain, all, 2);
  Plan some{whole.shape, {1, 1, 1}};
  Job jobs[2];
  int count = 0;
  for (int k = 0; k < 2; ++k) {
    const abcd_matrix* to = k ? dweight : dx;
    if (!to) continue;
    some.splits[count] = whole.splits[k];
    jobs[count] = all[k];
    jobs[count++].c[0] = out_of(to);
  }
  return count ? run(ctx, t, kPlain, jobs, count, some) : ABCD_OK;
}
