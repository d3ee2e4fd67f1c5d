// Matrices in 8 bits, written and read back: groups of 32 consecutive columns of a row share a power of
// two (of the microscaling formats the one with 8-bit whole numbers), element = code 2^(p - 127).
//   e = exponent of the group's largest magnitude, p = max(1, e + 121),
//   code = x 2^(127 - p) rounded to the nearest, held to +-127.
// A power of two keeps every step exact in 32 bits, whatever the order: the codes are those of the
// definition, and what is read back is exact in bf16.  Against 8-bit floating point (three bits of
// fraction) a group's error is a quarter; a scale that is not a power of two would win half a bit more,
// and make codes depend on how the division rounds.
#include <algorithm>

#include "packed8.cuh"

namespace abcd {
namespace {

struct PackedArgs {
  struct One {
    void* x;                          // the matrix that is read (pack) or written (unpack)
    signed char* codes;
    unsigned char* powers;
    long long rows, cols, sx, sc, sp;
    long long first;                  // units before this matrix's
    unsigned per_row;                 // units of a row: eight columns each, four to a group
    int dtype, vec;                   // vec: x's rows start on 16-byte boundaries
  } m[3];
  int n;
  long long units;
};

// Where a unit lies.
struct Place { long long row; int col, left; };
__device__ __forceinline__ Place place_of(const PackedArgs::One& o, long long at) {
  Place p;
  p.row = at < (1LL << 32) ? (unsigned)at / o.per_row : at / o.per_row;
  p.col = (int)(8 * (at - p.row * o.per_row));
  p.left = (int)(o.cols - p.col);
  return p;
}

template <typename T>
__global__ void __launch_bounds__(256) pack8_kernel(const __grid_constant__ PackedArgs a) {
  pdl_wait();
  const PackedArgs::One& o = a.m[0];
  // whole groups: the four lanes of a group are in or out together
  for (long long i = blockIdx.x * 256LL + threadIdx.x; i < (a.units + 31) / 32 * 32; i += gridDim.x * 256LL) {
    const bool in = i < a.units;
    const Place p = place_of(o, in ? i : 0);
    const T* x = (const T*)o.x + p.row * o.sx + p.col;
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = in && e < p.left ? to_f32(x[e]) : 0.f;
    unsigned top = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(v[e]) & 0x7fffffffu);
    top = max(top, __shfl_xor_sync(~0u, top, 1));
    top = max(top, __shfl_xor_sync(~0u, top, 2));
    const bool finite = top < 0x7f800000u;
    const int power = finite ? max((int)(top >> 23) - 6, 1) : 255;
    const float inverse = finite ? __uint_as_float((unsigned)(254 - power) << 23) : 0.f;
    if (!in) continue;
    signed char* to = o.codes + p.row * o.sc + p.col;
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < p.left) to[e] = (signed char)(finite ? __float2int_rn(fminf(fmaxf(v[e] * inverse, -127.f), 127.f)) : 0);
    if ((i & 3) == 0) o.powers[p.row * o.sp + p.col / 32] = (unsigned char)power;
  }
}

template <typename T>
__device__ __forceinline__ void unpack_unit(const PackedArgs::One& o, const Place& p) {
  const signed char* from = o.codes + p.row * o.sc + p.col;
  const float scale = __uint_as_float((unsigned)o.powers[p.row * o.sp + p.col / 32] << 23);   // 255: infinite, NaN times 0
  T* x = (T*)o.x + p.row * o.sx + p.col;
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (e < p.left) x[e] = from_f32<T>((float)from[e] * scale);
}

__global__ void __launch_bounds__(256) unpack8_kernel(const __grid_constant__ PackedArgs a) {
  pdl_wait();
  for (long long i = blockIdx.x * 256LL + threadIdx.x; i < a.units; i += gridDim.x * 256LL) {
    const int k = (a.n > 1 && i >= a.m[1].first) + (a.n > 2 && i >= a.m[2].first);
    const PackedArgs::One& o = a.m[k];
    const Place p = place_of(o, i - o.first);
    if (p.left <= 0) continue;
    if (o.dtype == ABCD_F32) unpack_unit<float>(o, p);
    else if (o.dtype == ABCD_F16) unpack_unit<__half>(o, p);
    else unpack_unit<__nv_bfloat16>(o, p);
  }
}

void add(PackedArgs& a, const abcd_packed8* q, void* x, long long stride, int dtype) {
  const bool vec = (((uintptr_t)x | (q->rows > 1 ? (size_t)stride * elem_size(dtype) : 0)) & 15) == 0;
  const unsigned per_row = (unsigned)(4 * ((q->cols + 31) / 32));
  a.m[a.n++] = PackedArgs::One{x, q->codes, q->powers, q->rows, q->cols, stride, q->stride, q->power_stride, a.units, per_row, dtype, vec};
  a.units += q->rows * per_row;
}

unsigned grid_of(const abcd_ctx* ctx, long long units) {
  return (unsigned)std::min<long long>((units + 255) / 256, 16LL * ctx->num_sms);
}

}  // namespace

abcd_status unpack(abcd_ctx* ctx, const Unpacked* list, int n) {
  PackedArgs a{};
  for (int k = 0; k < n; ++k) add(a, list[k].from, list[k].to, list[k].stride, list[k].dtype);
  return check_launch(ctx, "unpack8_kernel", launch_pdl(unpack8_kernel, dim3(grid_of(ctx, a.units)), dim3(256), 0, ctx->stream, a));
}

}  // namespace abcd

using namespace abcd;

extern "C" abcd_status abcd_pack8(abcd_ctx* ctx, const abcd_matrix* x, const abcd_packed8* packed) {
  if (!ctx) return ABCD_ERR_INVALID_ARG;
  if (!matrix_ok(x) || !packed_ok(packed) || x->rows != packed->rows || x->cols != packed->cols)
    return fail(ctx, ABCD_ERR_INVALID_ARG, "abcd_pack8: bad matrices");
  if (x->rows == 0) return ABCD_OK;
  if (touches(packed, x)) return fail(ctx, ABCD_ERR_INVALID_ARG, "abcd_pack8: the packed matrix overlaps x");
  PackedArgs a{};
  add(a, packed, x->data, x->stride, x->dtype);
  return with_type(x->dtype, [&](auto t) {
    return check_launch(ctx, "pack8_kernel", launch_pdl(pack8_kernel<decltype(t)>, dim3(grid_of(ctx, a.units)), dim3(256), 0, ctx->stream, a));
  });
}

extern "C" abcd_status abcd_unpack8(abcd_ctx* ctx, const abcd_packed8* packed, const abcd_matrix* y) {
  if (!ctx) return ABCD_ERR_INVALID_ARG;
  if (!matrix_ok(y) || !packed_ok(packed) || y->rows != packed->rows || y->cols != packed->cols)
    return fail(ctx, ABCD_ERR_INVALID_ARG, "abcd_unpack8: bad matrices");
  if (y->rows == 0) return ABCD_OK;
  if (touches(packed, y)) return fail(ctx, ABCD_ERR_INVALID_ARG, "abcd_unpack8: y overlaps the packed matrix");
  const Unpacked one{packed, y->data, y->stride, y->dtype};
  return unpack(ctx, &one, 1);
}
