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
    long long per_row;                // units of a row: eight columns each, four to a group
    int vec;                          // x's rows start on 16-byte boundaries
  } m[3];
  int n;
  long long units;
};

constexpr int kFlight = 4;            // units of a thread that are on their way at once

// Where a unit lies.
struct Place { long long row, col; int left; };
__device__ __forceinline__ Place place_of(const PackedArgs::One& o, long long at) {
  Place p;
  p.row = o.rows == 1 ? 0 : at < (1LL << 32) ? (unsigned)at / (unsigned)o.per_row : at / o.per_row;
  p.col = 8 * (at - p.row * o.per_row);
  p.left = (int)min(8LL, o.cols - p.col);
  return p;
}

// Eight values of a unit as they lie in memory, zeros past the row's end.
template <typename T> struct Eight {
  Pack<T, 16 / sizeof(T)> q[sizeof(T) / 2];
  __device__ __forceinline__ T& at(int e) { return q[e / (16 / sizeof(T))].v[e % (16 / sizeof(T))]; }
  __device__ __forceinline__ void load(const T* p, int left, bool vec) {
    if (vec && left == 8) {
#pragma unroll
      for (int k = 0; k < (int)sizeof(T) / 2; ++k) q[k] = reinterpret_cast<const Pack<T, 16 / sizeof(T)>*>(p)[k];
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) at(e) = e < left ? p[e] : T(0.f);
    }
  }
  __device__ __forceinline__ void store(T* p, int left, bool vec) {
    if (vec && left == 8) {
#pragma unroll
      for (int k = 0; k < (int)sizeof(T) / 2; ++k) reinterpret_cast<Pack<T, 16 / sizeof(T)>*>(p)[k] = q[k];
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e < left) p[e] = at(e);
    }
  }
  // The bits of the largest magnitude, as of a 32-bit value.
  __device__ __forceinline__ unsigned top() const {
    const unsigned* w = reinterpret_cast<const unsigned*>(q);
    unsigned m = 0;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int k = 0; k < 8; ++k) m = max(m, w[k] & 0x7fffffffu);
      return m;
    } else {                          // 16-bit magnitudes in pairs: they order as whole numbers do
#pragma unroll
      for (int k = 0; k < 4; ++k) m = __vmaxu2(m, w[k] & 0x7fff7fffu);
      const unsigned short h = (unsigned short)max(m & 0xffffu, m >> 16);
      return __float_as_uint(to_f32(*reinterpret_cast<const T*>(&h)));
    }
  }
};

// A unit's codes.  A value times a power of two plus 1.5 2^23 has the nearest whole number in its low bits.
template <typename T>
__device__ __forceinline__ uint2 codes_of(Eight<T>& x, int power, unsigned top) {
  const float inverse = __uint_as_float((unsigned)(254 - power) << 23);
  constexpr float kShift = 12582912.f;
  unsigned v[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = __float_as_uint(__fmaf_rn(to_f32(x.at(e)), inverse, kShift));
  if (__uint_as_float(top) * inverse >= 127.5f) {        // the largest one rounds to 128: held to 127
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const unsigned most = __float_as_uint(kShift + 127.f), least = __float_as_uint(kShift - 127.f);
      v[e] = min(max(v[e], least), most);
    }
  }
  uint2 w;
  w.x = __byte_perm(__byte_perm(v[0], v[1], 0x0040), __byte_perm(v[2], v[3], 0x0040), 0x5410);
  w.y = __byte_perm(__byte_perm(v[4], v[5], 0x0040), __byte_perm(v[6], v[7], 0x0040), 0x5410);
  return w;
}

template <typename T>
__global__ void __launch_bounds__(256) pack8_kernel(const __grid_constant__ PackedArgs a) {
  pdl_wait();
  const PackedArgs::One& o = a.m[0];
  const long long step = gridDim.x * 256LL;
  // the four lanes of a group are in or out together
  for (long long i0 = blockIdx.x * 256LL + threadIdx.x; i0 - (threadIdx.x & 31) < a.units; i0 += kFlight * step) {
    Place p[kFlight];
    Eight<T> x[kFlight];
#pragma unroll
    for (int k = 0; k < kFlight; ++k) {
      const long long i = i0 + k * step;
      p[k] = place_of(o, min(i, a.units - 1));
      if (i >= a.units) p[k].left = 0;
      x[k].load((const T*)o.x + p[k].row * o.sx + p[k].col, p[k].left, o.vec);
    }
#pragma unroll
    for (int k = 0; k < kFlight; ++k) {
      unsigned top = x[k].top();
      top = max(top, __shfl_xor_sync(~0u, top, 1));
      top = max(top, __shfl_xor_sync(~0u, top, 2));
      const bool finite = top < 0x7f800000u;
      const int power = finite ? max((int)(top >> 23) - 6, 1) : 255;
      const uint2 w = finite ? codes_of(x[k], power, top) : make_uint2(0u, 0u);
      signed char* to = o.codes + p[k].row * o.sc + p[k].col;
      if (p[k].left == 8) {
        *reinterpret_cast<uint2*>(to) = w;
      } else {
        for (int e = 0; e < p[k].left; ++e) to[e] = (signed char)((e < 4 ? w.x : w.y) >> 8 * (e & 3));
      }
      if ((threadIdx.x & 3) == 0 && p[k].left > 0) o.powers[p[k].row * o.sp + p[k].col / 32] = (unsigned char)power;
    }
  }
}

// A code's value: its byte, 128 added, as the low bits of 2^23.
__device__ __forceinline__ float value_of(unsigned codes, int byte) {
  return __uint_as_float(__byte_perm(codes, 0x4b000000u, 0x7650 + byte)) - 8388736.f;
}

template <typename T>
__global__ void __launch_bounds__(256) unpack8_kernel(const __grid_constant__ PackedArgs a) {
  pdl_wait();
  const long long step = gridDim.x * 256LL;
  for (long long i0 = blockIdx.x * 256LL + threadIdx.x; i0 < a.units; i0 += kFlight * step) {
    Place p[kFlight];
    uint2 w[kFlight];
    unsigned power[kFlight];
    int which[kFlight];
#pragma unroll
    for (int k = 0; k < kFlight; ++k) {
      const long long i = min(i0 + k * step, a.units - 1);
      which[k] = (a.n > 1 && i >= a.m[1].first) + (a.n > 2 && i >= a.m[2].first);
      const PackedArgs::One& o = a.m[which[k]];
      p[k] = place_of(o, i - o.first);
      if (i0 + k * step >= a.units) p[k].left = 0;
      if (p[k].left <= 0) continue;
      // a row of codes has room for whole units
      w[k] = *reinterpret_cast<const uint2*>(o.codes + p[k].row * o.sc + p[k].col);
      power[k] = o.powers[p[k].row * o.sp + p[k].col / 32];
    }
#pragma unroll
    for (int k = 0; k < kFlight; ++k) {
      if (p[k].left <= 0) continue;
      const PackedArgs::One& o = a.m[which[k]];
      const float scale = __uint_as_float(power[k] << 23);     // 255: infinite, and NaN times the codes' zeros
      Eight<T> x;
#pragma unroll
      for (int e = 0; e < 8; ++e) x.at(e) = from_f32<T>(value_of((e < 4 ? w[k].x : w[k].y) ^ 0x80808080u, e & 3) * scale);
      x.store((T*)o.x + p[k].row * o.sx + p[k].col, p[k].left, o.vec);
    }
  }
}

void add(PackedArgs& a, const abcd_packed8* q, void* x, long long stride, int dtype) {
  const bool vec = (((uintptr_t)x | (q->rows > 1 ? (size_t)stride * elem_size(dtype) : 0)) & 15) == 0;
  PackedArgs::One o{x, q->codes, q->powers, q->rows, q->cols, stride, q->stride, q->power_stride, a.units, 4 * ((q->cols + 31) / 32), vec};
  if (q->cols % 32 == 0 && stride == q->cols && q->stride == q->cols && q->power_stride == q->cols / 32) {   // without gaps: one row
    o.cols *= o.rows;
    o.per_row *= o.rows;
    o.rows = 1;
  }
  a.m[a.n++] = o;
  a.units += o.rows * o.per_row;
}

unsigned grid_of(const abcd_ctx* ctx, long long units) {
  return (unsigned)std::min<long long>((units + 255) / 256, 8LL * ctx->num_sms);
}

}  // namespace

abcd_status unpack(abcd_ctx* ctx, const Unpacked* list, int n) {
  for (const int dtype : {ABCD_BF16, ABCD_F16, ABCD_F32}) {          // a launch for each type there is
    PackedArgs a{};
    for (int k = 0; k < n; ++k)
      if (list[k].dtype == dtype) add(a, list[k].from, list[k].to, list[k].stride, dtype);
    if (a.units == 0) continue;
    const abcd_status st = with_type(dtype, [&](auto t) {
      return check_launch(ctx, "unpack8_kernel", launch_pdl(unpack8_kernel<decltype(t)>, dim3(grid_of(ctx, a.units)), dim3(256), 0, ctx->stream, a));
    });
    if (st != ABCD_OK) return st;
  }
  return ABCD_OK;
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
