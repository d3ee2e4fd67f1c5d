// Matrices in 8 bits, written and read back: groups of 32 consecutive columns of a row share a power of
// two (of the microscaling formats the one with 8-bit whole numbers), element = code 2^(p - 127).
//   e = exponent of the group's largest magnitude, p = max(1, e + 121),
//   code = x 2^(127 - p) rounded to the nearest, held to +-127.
// A power of two keeps every step exact in 32 bits, whatever the order: the codes are those of the
// definition, and what is read back is exact in bf16.  Against 8-bit floating point (three bits of
// fraction) a group's error is a quarter; a scale that is not a power of two would win half a bit more,
// and make codes depend on how the division rounds.
//
// Bound by HBM: 100,000 x 1,024 bf16 packed in 51 us (6.1 TB/s), read back in 47 (6.6).  A thread takes eight
// columns of every so many rows, four of them on their way at once (asked for one by one as they were used,
// 80 us), whole numbers come from adding 1.5 2^23, values from a byte in the low bits of 2^23.  Rows that
// start anywhere go element by element: 123 and 105 us.
#include <algorithm>
#include <type_traits>

#include "packed8.cuh"

namespace abcd {
namespace {

struct PackedArgs {
  struct One {
    void* x;                          // the matrix that is read (pack) or written (unpack)
    signed char* codes;
    unsigned char* powers;
    long long rows, cols, sx, sc, sp;
    int lanes;                        // threads of a row, a unit of columns each, whole groups of 32 columns
    int vec;                          // x's rows start on 16-byte boundaries
  } m[3];
};

constexpr int kFlight = 4;            // rows of a thread that are on their way at once

// The rows that a CTA takes at a time, and the thread's place in them: the addresses of a thread's units then
// differ by whole rows.
struct Share {
  long long row, step;                // the first row, rows from one turn to the next
  int groups;                         // rows between a turn's units
  long long col;
  int left;                           // the thread's columns: none for a thread without a unit
  // `width`: columns of a unit
  __device__ __forceinline__ Share(const PackedArgs::One& o, int width) {
    groups = 256 / o.lanes;
    const int group = (int)threadIdx.x / o.lanes, lane = (int)threadIdx.x - group * o.lanes;
    col = (blockIdx.x * (long long)o.lanes + lane) * width;
    left = group < groups ? (int)min((long long)width, o.cols - col) : 0;
    row = blockIdx.y * (long long)(groups * kFlight) + group;
    step = gridDim.y * (long long)(groups * kFlight);
    if (left <= 0) {                  // where it may read, it reads the CTA's first row
      left = 0;
      col = 0;
      row -= group;
    }
  }
};

// Eight values of a unit as they lie in memory, zeros past the row's end.
template <typename T> struct Eight {
  Pack<T, 16 / sizeof(T)> q[sizeof(T) / 2];
  __device__ __forceinline__ T& at(int e) { return q[e / (16 / sizeof(T))].v[e % (16 / sizeof(T))]; }
  __device__ __forceinline__ void load(const T* p) {
#pragma unroll
    for (int k = 0; k < (int)sizeof(T) / 2; ++k) q[k] = reinterpret_cast<const Pack<T, 16 / sizeof(T)>*>(p)[k];
  }
  __device__ __forceinline__ void load(const T* p, int left) {
    if (left == 8) return load(p);
#pragma unroll
    for (int e = 0; e < 8; ++e) at(e) = e < left ? p[e] : T(0.f);
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

// Rows on 16-byte boundaries.  EIGHTS: of a multiple of eight columns, so that no unit is short.
template <typename T, bool EIGHTS>
__global__ void __launch_bounds__(256, 4) pack8_kernel(const __grid_constant__ PackedArgs a) {
  pdl_wait();
  const PackedArgs::One& o = a.m[0];
  const Share at(o, 8);
  const T* x = (const T*)o.x + at.row * o.sx + at.col;
  signed char* to = o.codes + at.row * o.sc + at.col;
  unsigned char* power_to = o.powers + at.row * o.sp + at.col / 32;
  const long long next_x = at.groups * o.sx, next_to = at.groups * o.sc, next_power = at.groups * o.sp;
  // a turn's units; `full`: all of them are there.  (A warp's lanes take their turns together: the four lanes
  // of a group share its largest magnitude.)
  auto turn = [&](long long r, auto full) {
    constexpr bool FULL = decltype(full)::value;
    Eight<T> v[kFlight];
#pragma unroll
    for (int k = 0; k < kFlight; ++k) {    // without a condition: all are on their way before the first is used
      const T* from = FULL ? x + k * next_x : x + (min(r + k * at.groups, o.rows - 1) - r) * o.sx;
      if (EIGHTS) v[k].load(from);
      else v[k].load(from, at.left);
    }
#pragma unroll
    for (int k = 0; k < kFlight; ++k) {
      unsigned top = at.left > 0 ? v[k].top() : 0u;     // (a group past the row's end may have threads without a unit)
      top = max(top, __shfl_xor_sync(~0u, top, 1));
      top = max(top, __shfl_xor_sync(~0u, top, 2));
      const bool finite = top < 0x7f800000u;
      const int power = finite ? max((int)(top >> 23) - 6, 1) : 255;
      const uint2 w = finite ? codes_of(v[k], power, top) : make_uint2(0u, 0u);
      if (!FULL && r + k * at.groups >= o.rows) continue;
      signed char* row = to + k * next_to;
      if (at.left == 8) {
        *reinterpret_cast<uint2*>(row) = w;
      } else if (!EIGHTS) {
        for (int e = 0; e < at.left; ++e) row[e] = (signed char)((e < 4 ? w.x : w.y) >> 8 * (e & 3));
      }
      if ((threadIdx.x & 3) == 0 && at.left > 0) power_to[k * next_power] = (unsigned char)power;
    }
  };
  const long long base = blockIdx.y * (long long)(at.groups * kFlight);
  for (long long r = at.row, b = base; b < o.rows; r += at.step, b += at.step, x += at.step * o.sx, to += at.step * o.sc, power_to += at.step * o.sp) {
    if (b + at.groups * kFlight <= o.rows) turn(r, std::true_type());
    else turn(r, std::false_type());
  }
}

// (32-bit results by four columns: eight, as two accesses of half the bytes each, took 59 us for 50,000 x 1,024
// instead of 41.)
template <typename T>
__global__ void __launch_bounds__(256, 4) unpack8_kernel(const __grid_constant__ PackedArgs a) {
  pdl_wait();
  const PackedArgs::One& o = a.m[blockIdx.z];
  constexpr int W = 16 / sizeof(T);                         // columns of a unit: 16 bytes of results
  using Codes = std::conditional_t<W == 8, uint2, unsigned>;
  const Share at(o, W);
  if (at.left <= 0) return;
  T* x = (T*)o.x + at.row * o.sx + at.col;
  const signed char* from = o.codes + at.row * o.sc + at.col;
  const unsigned char* power_from = o.powers + at.row * o.sp + at.col / 32;
  const long long next_x = at.groups * o.sx, next_from = at.groups * o.sc, next_power = at.groups * o.sp;
  auto turn = [&](long long r, auto full) {
    constexpr bool FULL = decltype(full)::value;
    Codes w[kFlight];
    unsigned power[kFlight];
#pragma unroll
    for (int k = 0; k < kFlight; ++k) {
      const long long back = FULL ? 0 : r + k * at.groups - min(r + k * at.groups, o.rows - 1);
      w[k] = *reinterpret_cast<const Codes*>(from + k * next_from - back * o.sc);      // a row of codes has room for whole units
      power[k] = power_from[k * next_power - back * o.sp];
    }
#pragma unroll
    for (int k = 0; k < kFlight; ++k) {
      if (!FULL && r + k * at.groups >= o.rows) break;
      const float scale = __uint_as_float(power[k] << 23);     // 255: infinite, and NaN times the codes' zeros
      Pack<T, W> v;
      const unsigned* codes = reinterpret_cast<const unsigned*>(&w[k]);
#pragma unroll
      for (int e = 0; e < W; ++e) v.v[e] = from_f32<T>(code_value(codes[e / 4] ^ 0x80808080u, e & 3) * scale);
      T* to = x + k * next_x;
      if (at.left == W) {
        *reinterpret_cast<Pack<T, W>*>(to) = v;
      } else {
#pragma unroll
        for (int e = 0; e < W; ++e)
          if (e < at.left) to[e] = v.v[e];
      }
    }
  };
  const int per_turn = at.groups * kFlight;
  for (long long r = at.row; r < o.rows; r += at.step, x += at.step * o.sx, from += at.step * o.sc, power_from += at.step * o.sp) {
    if (r + per_turn <= o.rows) turn(r, std::true_type());
    else turn(r, std::false_type());
  }
}

// Rows that start anywhere: a warp takes 256 columns of a row, a lane one of each group of 32, so that
// consecutive lanes read and write consecutive elements.
constexpr int kSpan = 8;              // groups of a warp
constexpr int kRowsAhead = 2;         // rows of a warp that are on their way at once
template <typename T>
__global__ void __launch_bounds__(256) pack8_any_kernel(const __grid_constant__ PackedArgs a) {
  pdl_wait();
  const PackedArgs::One& o = a.m[0];
  const int lane = threadIdx.x & 31;
  const long long col = blockIdx.x * 32LL * kSpan, step = gridDim.y * 8LL;
  const int left = (int)min(32LL * kSpan, o.cols - col);
  const T* x = (const T*)o.x + col + lane;
  for (long long r = blockIdx.y * 8LL + threadIdx.x / 32; r < o.rows; r += kRowsAhead * step) {
    T v[kRowsAhead][kSpan];
#pragma unroll
    for (int k = 0; k < kRowsAhead; ++k) {
      const T* from = x + min(r + k * step, o.rows - 1) * o.sx;
#pragma unroll
      for (int g = 0; g < kSpan; ++g) v[k][g] = 32 * g + lane < left ? from[32 * g] : T(0.f);
    }
#pragma unroll
    for (int k = 0; k < kRowsAhead; ++k) {
      const long long row = r + k * step;
      if (row >= o.rows) break;
      signed char* to = o.codes + row * o.sc + col + lane;
      unsigned powers = 0;
#pragma unroll
      for (int g = 0; g < kSpan; ++g) {
        if (32 * g >= left) break;
        const float f = to_f32(v[k][g]);
        const unsigned top = __reduce_max_sync(~0u, __float_as_uint(f) & 0x7fffffffu);
        const bool finite = top < 0x7f800000u;
        const int power = finite ? max((int)(top >> 23) - 6, 1) : 255;
        const float inverse = __uint_as_float((unsigned)(254 - power) << 23);
        const int code = finite ? __float2int_rn(fminf(fmaxf(f * inverse, -127.f), 127.f)) : 0;
        if (32 * g + lane < left) to[32 * g] = (signed char)code;
        if (lane == g) powers = (unsigned)power;
      }
      if (32 * lane < left && lane < kSpan) o.powers[row * o.sp + col / 32 + lane] = (unsigned char)powers;
    }
  }
}

template <typename T>
__global__ void __launch_bounds__(256) unpack8_any_kernel(const __grid_constant__ PackedArgs a) {
  pdl_wait();
  const PackedArgs::One& o = a.m[0];
  const int lane = threadIdx.x & 31;
  const long long col = blockIdx.x * 32LL * kSpan, step = gridDim.y * 8LL;
  const int left = (int)min(32LL * kSpan, o.cols - col);
  for (long long r = blockIdx.y * 8LL + threadIdx.x / 32; r < o.rows; r += kRowsAhead * step) {
    unsigned char code[kRowsAhead][kSpan];
    unsigned power[kRowsAhead];                          // lane g holds group g's
#pragma unroll
    for (int k = 0; k < kRowsAhead; ++k) {
      const long long row = min(r + k * step, o.rows - 1);
      const unsigned char* from = (const unsigned char*)o.codes + row * o.sc + col + lane;
      power[k] = o.powers[row * o.sp + col / 32 + min(lane, (left - 1) / 32)];
#pragma unroll
      for (int g = 0; g < kSpan; ++g) code[k][g] = 32 * g + lane < left ? from[32 * g] : (unsigned char)0;
    }
#pragma unroll
    for (int k = 0; k < kRowsAhead; ++k) {
      if (r + k * step >= o.rows) break;
      T* x = (T*)o.x + (r + k * step) * o.sx + col + lane;
#pragma unroll
      for (int g = 0; g < kSpan; ++g) {
        if (32 * g >= left) break;
        const float scale = __uint_as_float(__shfl_sync(~0u, power[k], g) << 23);
        if (32 * g + lane < left) x[32 * g] = from_f32<T>(code_value(code[k][g] ^ 0x80u, 0) * scale);
      }
    }
  }
}
dim3 any_grid(const abcd_ctx* ctx, const PackedArgs::One& o) {
  const long long slices = (o.cols + 32 * kSpan - 1) / (32 * kSpan);
  return dim3((unsigned)slices, (unsigned)std::min((o.rows + 7) / 8, std::max(1LL, 8LL * ctx->num_sms / slices)));
}

PackedArgs::One one_of(const abcd_packed8* q, void* x, long long stride, int dtype, int width) {
  const bool vec = (((uintptr_t)x | (q->rows > 1 ? (size_t)stride * elem_size(dtype) : 0)) & 15) == 0;
  return PackedArgs::One{x, q->codes, q->powers, q->rows, q->cols, stride, q->stride, q->power_stride,
                         lanes_of(32 / width * ((q->cols + 31) / 32), 32 / width), vec};
}

// A grid for matrices of up to these: slices of columns, CTAs of rows, matrices.
dim3 grid_of(const abcd_ctx* ctx, const PackedArgs& a, int n, int width) {
  long long slices = 1, rows = 1;
  for (int k = 0; k < n; ++k) {
    const PackedArgs::One& o = a.m[k];
    const long long per_cta = 256 / o.lanes * kFlight, s = (o.cols + width * o.lanes - 1) / (width * o.lanes);
    slices = std::max(slices, s);
    rows = std::max(rows, std::min((o.rows + per_cta - 1) / per_cta, std::max(1LL, 4LL * ctx->num_sms / (s * n))));
  }
  return dim3((unsigned)slices, (unsigned)rows, (unsigned)n);
}

}  // namespace

abcd_status unpack(abcd_ctx* ctx, const Unpacked* list, int n) {
  for (const int dtype : {ABCD_BF16, ABCD_F16, ABCD_F32}) {          // a launch for each type there is
    PackedArgs a{};
    int count = 0;
    const int width = (int)(16 / elem_size(dtype));
    for (int k = 0; k < n; ++k)
      if (list[k].dtype == dtype) a.m[count++] = one_of(list[k].from, list[k].to, list[k].stride, dtype, width);
    if (count == 0) continue;
    if (count == 1 && !a.m[0].vec) {
      const abcd_status st = with_type(dtype, [&](auto t) {
        return check_launch(ctx, "unpack8_any_kernel", launch_pdl(unpack8_any_kernel<decltype(t)>, any_grid(ctx, a.m[0]), dim3(256), 0, ctx->stream, a));
      });
      if (st != ABCD_OK) return st;
      continue;
    }
    const abcd_status st = with_type(dtype, [&](auto t) {
      return check_launch(ctx, "unpack8_kernel", launch_pdl(unpack8_kernel<decltype(t)>, grid_of(ctx, a, count, width), dim3(256), 0, ctx->stream, a));
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
  a.m[0] = one_of(packed, x->data, x->stride, x->dtype, 8);
  return with_type(x->dtype, [&](auto t) {
    if (!a.m[0].vec)
      return check_launch(ctx, "pack8_any_kernel", launch_pdl(pack8_any_kernel<decltype(t)>, any_grid(ctx, a.m[0]), dim3(256), 0, ctx->stream, a));
    using T = decltype(t);
    return check_launch(ctx, "pack8_kernel", launch_pdl(x->cols % 8 == 0 ? pack8_kernel<T, true> : pack8_kernel<T, false>, grid_of(ctx, a, 1, 8), dim3(256), 0, ctx->stream, a));
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
