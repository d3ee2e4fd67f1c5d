// What the network calls (layernorm.cu, gatedff.cu, dropout.cu) share: element types, checks of
// their matrices, aligned accesses of several elements.
#pragma once

#include <cuda_bf16.h>

#include <algorithm>
#include <utility>

#include "abcd_internal.cuh"

namespace abcd {

constexpr long long kMaxNetCols = 1LL << 24;   // columns of a matrix, hidden columns
constexpr long long kMaxNetRows = 1LL << 30;   // its rows
constexpr int kNetSms = 160;                   // SMs for which the network workspace has room
// The workspace's header: the status word of the products' waits and, from kNetCounters on, the
// counters of their splits, zero between calls.
constexpr size_t kNetHeader = 65536, kNetCounters = 256;

inline size_t elem_size(int dtype) { return dtype == ABCD_F32 ? 4 : 2; }
inline bool dtype_ok(int dtype) {
  return dtype == ABCD_F16 || dtype == ABCD_F32 || dtype == ABCD_BF16;
}
inline size_t net_align(size_t x) { return (x + 255) & ~(size_t)255; }

// A matrix that a call may read or write: its type and shape within the limits, its rows apart, its
// data there (unless it has no rows) and aligned to its type.
inline bool matrix_ok(const abcd_matrix* m) {
  return m && dtype_ok(m->dtype) && m->rows >= 0 && m->rows <= kMaxNetRows && m->cols >= 1 &&
         m->cols <= kMaxNetCols && m->stride >= m->cols && m->stride <= (1LL << 31) &&
         (m->rows == 0 || m->data) && ((uintptr_t)m->data & (elem_size(m->dtype) - 1)) == 0;
}
inline bool same_form(const abcd_matrix* a, const abcd_matrix* b) {
  return a->dtype == b->dtype && a->rows == b->rows && a->cols == b->cols;
}
// Whether rows of the matrix start on multiples of `bytes` (a power of two).
inline bool rows_aligned(const abcd_matrix* m, size_t bytes) {
  return (((uintptr_t)m->data | (m->rows > 1 ? (size_t)m->stride * elem_size(m->dtype) : 0)) &
          (bytes - 1)) == 0;
}

// The bytes of a matrix: n rows of `width`, `step` apart.
struct ByteRows { uintptr_t first; long long n, width, step; };
// Whether a byte of one matrix lies where one of the other does.  Both may be columns of one buffer,
// their rows in turn: rows equally far apart are compared once, others row by row (of the matrix with
// fewer), which only matrices that reach into one another come to.
inline bool overlap(ByteRows p, ByteRows q) {
  if (p.n == 0 || q.n == 0) return false;
  for (ByteRows* r : {&p, &q})
    if (r->n == 1 || r->step == r->width) *r = ByteRows{r->first, 1, r->n * r->width, r->n * r->width};   // one piece
  if (p.n > q.n) std::swap(p, q);
  const auto end = [](const ByteRows& r) { return r.first + (uintptr_t)(r.n - 1) * (uintptr_t)r.step + (uintptr_t)r.width; };
  if (end(p) <= q.first || end(q) <= p.first) return false;
  // whether the bytes [from, from + width), counted from q's first row, meet a row of q
  const auto meets = [&](long long from, long long width) {
    const long long row = from < 0 ? 0 : from / q.step;          // the last that starts at or before them
    return (row < q.n && row * q.step < from + width && from < row * q.step + q.width) ||
           (row + 1 < q.n && (row + 1) * q.step < from + width);
  };
  const long long from = (long long)(p.first - q.first);
  if (p.step == q.step && p.n > 1) {
    // row i of p against rows i + k of q: the two k whose rows may meet it
    const long long k = from >= 0 ? from / q.step : -((-from + q.step - 1) / q.step);
    const auto pair = [&](long long k) { return std::max(0LL, -k) < std::min(p.n, q.n - k); };
    const long long at = from - k * q.step;                      // of p's row within that of q
    return (pair(k) && at < q.width) || (pair(k + 1) && at + p.width > q.step);
  }
  for (long long i = 0; i < p.n; ++i)
    if (meets(from + i * p.step, p.width)) return true;
  return false;
}
inline bool overlap(const abcd_matrix* a, const abcd_matrix* b) {
  const auto rows_of = [](const abcd_matrix* m) {
    const long long e = (long long)elem_size(m->dtype);
    return ByteRows{(uintptr_t)m->data, m->rows, m->cols * e, m->stride * e};
  };
  return overlap(rows_of(a), rows_of(b));
}

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) {
  return __float2bfloat16_rn(v);
}

// The value of an 8-bit code (one of four, 128 added to each): its byte as the low bits of 2^23.
__device__ __forceinline__ float code_value(unsigned codes, int byte) {
  return __uint_as_float(__byte_perm(codes, 0x4b000000u, 0x7650 + byte)) - 8388736.f;
}

// Threads of a row where a CTA of 256 takes rows in groups of that many threads, a vector each: all of the row's
// vectors up to 256, or an even share of them in up to four slices, where that leaves fewer threads idle
// (160 vectors: one group of 160, or three of 80).  A multiple of `unit`.
inline int lanes_of(long long vectors, int unit = 1) {
  int best = 256 / unit * unit;
  double used = 0;
  for (int slices = 1; slices <= 4; ++slices) {
    const long long lanes = ((vectors + slices - 1) / slices + unit - 1) / unit * unit;
    if (lanes > 256) continue;
    const double share = (double)(256 / lanes) * (double)vectors / (256.0 * slices);
    if (share > used + 0.1) {
      used = share;
      best = (int)lanes;
    }
  }
  return best;
}

// V elements of T as one aligned access.
template <typename T, int V> struct alignas(sizeof(T) * V) Pack { T v[V]; };

// Calls f with a value of the element type that dtype names.
template <typename F> auto with_type(int dtype, F&& f) {
  if (dtype == ABCD_F32) return f(float());
  if (dtype == ABCD_F16) return f(__half());
  return f(__nv_bfloat16());
}

}  // namespace abcd
