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
//
// Bound by HBM in 32 bits (50,000 x 1,024: forward 127 us, 6.5 TB/s, backward 180, 6.8 TB/s), in 16 bits, with
// twice the values for the bytes, also by instructions (100,000 x 1,024 bf16: 139 us, 5.9 TB/s, and 235, 5.2).
// A row is read once: its threads hold it in registers, eight or sixteen values each, and the next rows are
// copied to shared memory meanwhile.  Values go in pairs (one instruction for two), what lies past a row's
// end is zero by the factors there and needs no tests, and the factors of the columns lie in shared memory
// (in registers: 149 and 258 us).  One CTA per row that reads it again for each use took 6,615 us for both.
// Rows that start anywhere are taken element by element from shared memory: 100,001 x 999 bf16 252 and 357.
#include <algorithm>
#include <type_traits>

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
      v.fh = a.f ? (to_f32(f[c]) - first.mean) * first.rstd : 0.f;
      v.yh = a.x ? (close_value(to_f32(x[c]), v.fh, v.k.x, v.k.y) - second.mean) * second.rstd : 0.f;
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

// Pairs of values: one instruction does both (the kernels are bound by what they issue, not by the units).
__device__ __forceinline__ float2 both(float v) { return make_float2(v, v); }
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) { return __ffma2_rn(a, b, c); }
__device__ __forceinline__ float2 add2(float2 a, float2 b) { return __fadd2_rn(a, b); }
__device__ __forceinline__ float2 mul2(float2 a, float2 b) { return __fmul2_rn(a, b); }
// a - b, rounded as the difference is
__device__ __forceinline__ float2 sub2(float2 a, float b) { return __fadd2_rn(a, both(-b)); }
// close_value of a pair
__device__ __forceinline__ float2 close_pair(float2 x, float2 fh, float2 A, float2 C) { return add2(x, fma2(A, fh, C)); }

// How a row lies over threads: E values each, TPR threads a row.  VEC: rows on 16-byte boundaries, E values as
// vectors of 16 bytes, which the threads that use them copy ahead to shared memory.  Else the 16-byte pieces
// that a row reaches into are copied ahead by its threads together, and a thread takes every TPR-th
// element.  Forward, 16-bit rows take 16 values a thread, which halves what a row's sums cost per value;
// backward (with eight vectors of sums and factors in registers) and in 32 bits eight.
template <typename T, int TPR_, int E_, bool BWD, bool VEC_> struct CloseRow {
  static constexpr int TPR = TPR_, E = E_;
  static constexpr bool VEC = VEC_;
  static constexpr int V = VEC ? 16 / (int)sizeof(T) : 1, NV = E / V;
  static constexpr int kThreads = TPR > 256 ? TPR : 256, kGroups = kThreads / TPR;
  static constexpr int kMats = BWD ? 4 : 2;
  static constexpr int kRowBytes = TPR * E * (int)sizeof(T) + (VEC ? 0 : 32);
  static constexpr int kMatBytes = kGroups * kRowBytes, kSlotBytes = kMats * kMatBytes;
  // The factors of the columns (A, C, w_before and, forward, b_before), for all groups, behind the rows: in
  // registers they would cost a third of the warps.  Wide rows forward hold them in registers all the same:
  // there they would take the second CTA's shared memory (25,000 x 4,096 bf16: 266 us, and 163 so).
  static constexpr int kFactors = BWD ? 3 : 4;
  static constexpr bool kHold = !BWD && TPR * E > 2048;
  static constexpr size_t kFactorBytes = kHold ? 0 : (size_t)kFactors * TPR * E * 4;
  // rows that are there or on their way
  static constexpr int kDepth = BWD ? (3 * (size_t)kSlotBytes + kFactorBytes > 224 * 1024 ? 2 : 3) : 4;
  static constexpr size_t kRing = (size_t)kDepth * kSlotBytes, kSums = BWD ? (size_t)4 * TPR * E * 4 : 0;
  static constexpr size_t kRows = kRing > kSums ? kRing : kSums;
  static constexpr size_t kSmem = kRows + kFactorBytes;
  // CTAs per SM, as many as registers and rows leave room for
  static constexpr int kFit = (int)(227 * 1024 / (kSmem + 2048));
  static_assert(kFit >= 1);
  static constexpr int kMost = BWD || kHold ? 2 : 3;
  static constexpr int kCtas = kThreads > 256 ? (kFit < 2 || BWD ? 1 : 2) : kFit < kMost ? kFit : kMost;
};

template <typename T, typename R> struct CloseRows {
  const CloseArgs& a;
  char* slots;                        // the thread's first vector (VEC) or its row's first piece, of the first slot
  float4* factor;                     // the thread's first four factors of A
  float4 held[R::kHold ? R::kFactors * R::E / 4 : 1];
  int bytes[R::NV];                   // VEC: of the thread's vectors
  int rows, turns, lane, cols;        // rows of the group; turns that its threads take together
  int now;                            // the slot of the row at hand
  bool partial;                       // the thread has columns past the row's end
  unsigned row, step;                 // the row at hand, from a turn to the next

  __device__ __forceinline__ CloseRows(char* smem, const CloseArgs& args) : a(args) {
    const int group = threadIdx.x / R::TPR;
    row = blockIdx.x * R::kGroups + group;
    step = gridDim.x * R::kGroups;
    lane = threadIdx.x % R::TPR;
    cols = a.cols;
    rows = row < a.rows ? (int)((a.rows - row + step - 1) / step) : 0;
    // groups of whole warps go on by themselves; rows that share a warp take their turns together
    turns = R::TPR >= 32 ? rows : (int)((a.rows - (long long)blockIdx.x * R::kGroups + step - 1) / step);
    slots = smem + (R::VEC ? threadIdx.x * 16 : group * R::kRowBytes);
    factor = reinterpret_cast<float4*>(smem + R::kRows) + lane;
    now = 0;
    partial = column(R::NV - 1) + R::V > cols;
#pragma unroll
    for (int j = 0; j < R::NV; ++j) bytes[j] = R::VEC ? min(16, (cols - column(j)) * (int)sizeof(T)) : 0;
    // what is never copied reads as zero
    if constexpr (R::VEC) {
#pragma unroll
      for (int q = 0; q < R::kMats; ++q)
#pragma unroll
        for (int j = 0; j < R::NV; ++j)
          if (!base(q) || bytes[j] <= 0)
            for (int d = 0; d < R::kDepth; ++d) *reinterpret_cast<uint4*>(vector(d, q, j)) = make_uint4(0u, 0u, 0u, 0u);
    }
  }
  __device__ __forceinline__ const T* base(int q) const { return (const T*)(q == 0 ? a.f : q == 1 ? a.x : q == 2 ? a.dy : a.dn); }
  __device__ __forceinline__ unsigned stride(int q) const { return (unsigned)(q == 0 ? a.sf : q == 1 ? a.sx : q == 2 ? a.sdy : a.sdn); }
  // Where row r of a matrix starts (rows and strides have 32 bits, their product does not).
  __device__ __forceinline__ const T* start_of(int q, unsigned r) const { return base(q) + (unsigned long long)r * stride(q); }
  __device__ __forceinline__ int column(int j) const { return (j * R::TPR + lane) * R::V; }
  __device__ __forceinline__ char* vector(int slot, int mat, int j) const {
    return slots + slot * R::kSlotBytes + mat * R::kMatBytes + j * R::kThreads * 16;
  }
  __device__ __forceinline__ char* pieces(int slot, int mat) const { return slots + slot * R::kSlotBytes + mat * R::kMatBytes; }
  __device__ __forceinline__ void fetch(int t, int slot, unsigned r) {
    if (t < rows) {
#pragma unroll
      for (int q = 0; q < R::kMats; ++q) {
        if (!base(q)) continue;
        const T* src = start_of(q, r);
        if constexpr (R::VEC) {
#pragma unroll
          for (int j = 0; j < R::NV; ++j)
            if (bytes[j] > 0) copy16(vector(slot, q, j), src + column(j), bytes[j]);
        } else {
          const char* begin = (const char*)src;
          const char* end = begin + cols * (int)sizeof(T);
          const char* lowest = (const char*)base(q);
          const char* highest = (const char*)(start_of(q, (unsigned)a.rows - 1) + cols);
          const char* from = begin - ((uintptr_t)begin & 15) + 16 * lane;
          for (char* to = pieces(slot, q) + 16 * lane; from < end; from += 16 * R::TPR, to += 16 * R::TPR) {
            if (from >= lowest && from + 16 <= highest) {
              copy16(to, from, 16);
            } else {                  // a piece that reaches out of the matrix
#pragma unroll 1
              for (int e = 0; e < 16; e += (int)sizeof(T))
                if (from + e >= begin && from + e < end) *reinterpret_cast<T*>(to + e) = *reinterpret_cast<const T*>(from + e);
            }
          }
        }
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  }
  __device__ __forceinline__ void start() {
#pragma unroll
    for (int d = 0; d < R::kDepth - 1; ++d) fetch(d, d, row + d * step);
  }
  // Asks for a row to come and waits for turn t's.
  __device__ __forceinline__ void turn(int t) {
    if constexpr (!R::VEC) row_sync<R::TPR>();             // the last turn's row is done with
    fetch(t + R::kDepth - 1, now == 0 ? R::kDepth - 1 : now - 1, row + (R::kDepth - 1) * step);
    asm volatile("cp.async.wait_group %0;" ::"n"(R::kDepth - 1) : "memory");
    if constexpr (!R::VEC) row_sync<R::TPR>();
  }
  __device__ __forceinline__ void next() {
    now = now == R::kDepth - 1 ? 0 : now + 1;
    row += step;
  }
  // The thread's values of the row at hand of a matrix: zeros past its end, of no row and of a matrix that is
  // not there.  (Rows that start anywhere: `none`.)
  __device__ __forceinline__ void get(float2 (&pairs)[R::E / 2], int t, int mat, float none = 0.f) const {
    float v[R::E];
    if constexpr (R::VEC) {
#pragma unroll
      for (int j = 0; j < R::NV; ++j) {
        const Pack<T, R::V> w = *reinterpret_cast<const Pack<T, R::V>*>(vector(now, mat, j));
#pragma unroll
        for (int i = 0; i < R::V; ++i) v[j * R::V + i] = R::TPR >= 32 || t < rows ? to_f32(w.v[i]) : 0.f;
      }
    } else {
      const bool there = base(mat) != nullptr && (R::TPR >= 32 || t < rows);
      const T* p = (const T*)(pieces(now, mat) + ((uintptr_t)start_of(mat, row) & 15)) + lane;
#pragma unroll
      for (int e = 0; e < R::E; ++e) v[e] = there && column(e) < cols ? to_f32(p[e * R::TPR]) : none;
    }
#pragma unroll
    for (int e = 0; e < R::E / 2; ++e) pairs[e] = make_float2(v[2 * e], v[2 * e + 1]);
  }
  // The row at hand of a result.
  __device__ __forceinline__ void put(void* matrix, long long stride, const float2 (&v)[R::E / 2], int t) const {
    if (R::TPR < 32 && t >= rows) return;
    T* to = (T*)matrix + (unsigned long long)row * (unsigned)stride;
#pragma unroll
    for (int j = 0; j < R::NV; ++j) {
      float w[R::V];
#pragma unroll
      for (int i = 0; i < R::V; ++i) w[i] = (j * R::V + i) % 2 ? v[(j * R::V + i) / 2].y : v[(j * R::V + i) / 2].x;
      if constexpr (R::VEC) {
        if (bytes[j] > 0) store_vec<T, R::V>(to + column(j), w, bytes[j] / (int)sizeof(T));
      } else {
        if (column(j) < cols) to[column(j)] = from_f32<T>(w[0]);
      }
    }
  }
  // A vector's values of the thread's columns; zero past their end.
  __device__ __forceinline__ void weights(float2 (&pairs)[R::E / 2], const void* w, int wide, float none) const {
    float v[R::E];
#pragma unroll
    for (int j = 0; j < R::NV; ++j) {
      float u[R::V];
      const int left = cols - column(j);
      load_weight<T, R::V>(u, w, wide, column(j), left, none);
#pragma unroll
      for (int i = 0; i < R::V; ++i) v[j * R::V + i] = i < left ? u[i] : 0.f;
    }
#pragma unroll
    for (int e = 0; e < R::E / 2; ++e) pairs[e] = make_float2(v[2 * e], v[2 * e + 1]);
  }
};

// The sum of a over the threads of a row, in each of them; as row_sum2.
template <int TPR> __device__ __forceinline__ void row_sum(float& a, float2 (*red)[32], int turn) {
  if constexpr (TPR > 32) {
    float unused = 0.f;
    row_sum2<TPR>(a, unused, red, turn);
  } else {
#pragma unroll
    for (int o = TPR / 2; o; o >>= 1) a += __shfl_xor_sync(~0u, a, o);
  }
}

// A row's statistics from the threads' values (which are zero past its end).
template <typename T, typename R>
__device__ __forceinline__ Stat stat_of_row(const CloseRows<T, R>& rows, const float2 (&v)[R::E / 2], int kind, float eps, float inv, float2 (*red)[32], int& turn) {
  constexpr int P = R::E / 2;
  float2 s2 = both(0.f), q2 = both(0.f);
  if (kind == ABCD_RMS_NORM) {
#pragma unroll
    for (int e = 0; e < P; ++e) q2 = fma2(v[e], v[e], q2);
    float q = q2.x + q2.y;
    row_sum<R::TPR>(q, red, turn);
    turn ^= 1;
    return Stat{0.f, rsqrtf(q * inv + eps)};
  }
#pragma unroll
  for (int e = 0; e < P; ++e) s2 = add2(s2, v[e]);
  float s = s2.x + s2.y;
  row_sum<R::TPR>(s, red, turn);
  // the division's rounding taken back, then what the sum has rounded
  float mean = s * inv;
  mean = __fmaf_rn(__fmaf_rn(-mean, (float)rows.cols, s), inv, mean);
  s2 = both(0.f);
#pragma unroll
  for (int e = 0; e < P; ++e) {
    float2 d = sub2(v[e], mean);
    // past the row's end nothing deviates
    if (rows.partial) {
      const int c = rows.column(2 * e / R::V) + 2 * e % R::V, next = R::V == 1 ? rows.column(2 * e + 1) : c + 1;
      if (c >= rows.cols) d.x = 0.f;
      if (next >= rows.cols) d.y = 0.f;
    }
    q2 = fma2(d, d, q2);
    s2 = add2(s2, d);
  }
  float q = q2.x + q2.y, off = s2.x + s2.y;
  row_sum2<R::TPR>(q, off, red, turn ^ 1);
  off *= inv;
  return Stat{mean + off, rstd_of(q * inv, off, eps)};
}

// What a row's deviations are multiplied by: rstd, or zero where the mean times it is infinite.  Such a row is of
// one value (a single other one, a step of fp32 away, would leave rstd below 2^24 sqrt(cols) / mean), so
// nothing deviates; but past the row's end zeros lie, and what they would be, an infinity, times the factors'
// zeros is NaN.  (An infinite rstd stays.)
__device__ __forceinline__ float factor_of_row(const Stat& s) {
  constexpr float kMost = 3.402823466e38f;
  return fabsf(s.mean) * s.rstd > kMost && s.rstd <= kMost ? 0.f : s.rstd;
}

// The factors of the columns to shared memory, by the CTA's first group: [factor][four values][thread of a row].
template <typename T, typename R> __device__ __forceinline__ void set_factors(CloseRows<T, R>& rows, const CloseArgs& a) {
  if (R::kHold || threadIdx.x < R::TPR) {
    float2 g[R::E / 2], k[R::E / 2];
    rows.weights(g, a.gate, a.wide_w, 1.f);
#pragma unroll
    for (int q = 0; q < R::kFactors; ++q) {
      rows.weights(k, q == 0 ? a.w[0] : q == 1 ? a.b[0] : q == 2 ? a.w[1] : a.b[1], a.wide_w, q == 0 || q == 2 ? 1.f : 0.f);
#pragma unroll
      for (int e = 0; e < R::E / 2; ++e)
        if (q < 2) k[e] = mul2(k[e], mul2(g[e], both(a.scale)));
#pragma unroll
      for (int e = 0; e < R::E / 4; ++e) {
        const float4 v = make_float4(k[2 * e].x, k[2 * e].y, k[2 * e + 1].x, k[2 * e + 1].y);
        if constexpr (R::kHold) rows.held[q * (R::E / 4) + e] = v;
        else rows.factor[(q * (R::E / 4) + e) * R::TPR] = v;
      }
    }
  }
  __syncthreads();
}
// Four of the thread's factors: pairs 2 e and 2 e + 1.
template <typename T, typename R> __device__ __forceinline__ float4 factor_of(const CloseRows<T, R>& rows, int which, int e) {
  if constexpr (R::kHold) return rows.held[which * (R::E / 4) + e];
  else return rows.factor[(which * (R::E / 4) + e) * R::TPR];
}
__device__ __forceinline__ float2 half_of(const float4& v, int h) { return h ? make_float2(v.z, v.w) : make_float2(v.x, v.y); }

template <typename T, typename R>
__global__ void __launch_bounds__(R::kThreads, R::kCtas) close_fwd_kernel(const __grid_constant__ CloseArgs a) {
  extern __shared__ __align__(16) char smem[];
  __shared__ float2 red[2][32];
  constexpr int P = R::E / 2;
  pdl_wait();
  CloseRows<T, R> rows(smem, a);
  rows.start();
  set_factors(rows, a);
  const float inv = 1.f / (float)a.cols;
  int half = 0;
  for (int t = 0; t < rows.turns; ++t, rows.next()) {
    rows.turn(t);
    float2 f[P], x[P];
    rows.get(f, t, 0);
    rows.get(x, t, 1);
    Stat first{0.f, 1.f}, second{0.f, 1.f};
    if (a.kind[0] != kNone) first = stat_of_row(rows, f, a.kind[0], a.eps[0], inv, red, half);
    const float2 spread = both(factor_of_row(first));
#pragma unroll
    for (int e = 0; e < P; e += 2) {
      const float4 A = factor_of(rows, 0, e / 2), C = factor_of(rows, 1, e / 2);
#pragma unroll
      for (int h = 0; h < 2; ++h) x[e + h] = close_pair(x[e + h], mul2(sub2(f[e + h], first.mean), spread), half_of(A, h), half_of(C, h));
    }
    if (a.kind[1] != kNone) {
      second = stat_of_row(rows, x, a.kind[1], a.eps[1], inv, red, half);
#pragma unroll
      for (int e = 0; e < P; e += 2) {
        const float4 W = factor_of(rows, 2, e / 2), B = factor_of(rows, 3, e / 2);
#pragma unroll
        for (int h = 0; h < 2; ++h) f[e + h] = fma2(mul2(sub2(x[e + h], second.mean), both(second.rstd)), half_of(W, h), half_of(B, h));
      }
      rows.put(a.n, a.sn, f, t);
    }
    rows.put(a.y, a.sy, x, t);
    if ((R::TPR >= 32 || t < rows.rows) && rows.lane == 0) {
      const Stat s[2] = {first, second};
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        if (a.mean[k]) a.mean[k][rows.row] = s[k].mean;
        if (a.rstd[k]) a.rstd[k][rows.row] = s[k].rstd;
      }
    }
  }
}

template <typename T, typename R>
__global__ void __launch_bounds__(R::kThreads, R::kCtas) close_bwd_kernel(const __grid_constant__ CloseArgs a) {
  extern __shared__ __align__(16) char smem[];
  __shared__ float2 red[2][32];
  constexpr int P = R::E / 2;
  pdl_wait();
  CloseRows<T, R> rows(smem, a);
  rows.start();
  set_factors(rows, a);
  float2 sums[4][P];
#pragma unroll
  for (int k = 0; k < 4; ++k)
#pragma unroll
    for (int e = 0; e < P; ++e) sums[k][e] = both(0.f);
  const float inv = 1.f / (float)a.cols;
  const float centre[2] = {a.kind[0] == ABCD_LAYER_NORM ? inv : 0.f, a.kind[1] == ABCD_LAYER_NORM ? inv : 0.f};
  Stat next[2] = {{0.f, 0.f}, {0.f, 0.f}};
  if (rows.rows > 0) {
    next[0] = stat_of(a, 0, rows.row);
    next[1] = stat_of(a, 1, rows.row);
  }
  for (int t = 0; t < rows.turns; ++t, rows.next()) {
    rows.turn(t);
    const Stat first = next[0], second = next[1];
    if (t + 1 < rows.rows) {
      next[0] = stat_of(a, 0, rows.row + rows.step);
      next[1] = stat_of(a, 1, rows.row + rows.step);
    } else if (R::TPR < 32) {
      // a turn without a row: of an earlier row's statistics and the factors could come infinities, and NaN in
      // the sums, where dn's zeros meet them
      next[0] = next[1] = Stat{0.f, 0.f};
    }
    float2 fh[P], g[P], p1 = both(0.f), p2 = both(0.f);
    // past the end of a row that starts anywhere the mean, which costs no more than zero there (the other factor
    // would: 100,001 x 999 bf16 377 us instead of 357)
    rows.get(fh, t, 0, first.mean);
    rows.get(g, t, 2);
    const float2 spread = both(R::VEC ? factor_of_row(first) : first.rstd);
#pragma unroll
    for (int e = 0; e < P; ++e) fh[e] = mul2(sub2(fh[e], first.mean), spread);
    if (a.dn) {
      float2 yh[P], dn[P];
      rows.get(yh, t, 1, second.mean);
      rows.get(dn, t, 3);
      const float2 spread = both(R::VEC ? factor_of_row(second) : second.rstd);
#pragma unroll
      for (int e = 0; e < P; e += 2) {
        const float4 A = factor_of(rows, 0, e / 2), C = factor_of(rows, 1, e / 2), W = factor_of(rows, 2, e / 2);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int i = e + h;
          // the forward pass's, bit for bit
          yh[i] = mul2(sub2(close_pair(yh[i], fh[i], half_of(A, h), half_of(C, h)), second.mean), spread);
          sums[2][i] = add2(sums[2][i], dn[i]);
          sums[3][i] = fma2(dn[i], yh[i], sums[3][i]);
          dn[i] = mul2(dn[i], half_of(W, h));
          p1 = add2(p1, dn[i]);
          p2 = fma2(dn[i], yh[i], p2);
        }
      }
      float s1 = p1.x + p1.y, s2 = p2.x + p2.y;
      row_sum2<R::TPR>(s1, s2, red, 0);
      s1 *= centre[1];
      s2 *= inv;
#pragma unroll
      for (int e = 0; e < P; ++e) g[e] = fma2(fma2(yh[e], both(-s2), sub2(dn[e], s1)), both(second.rstd), g[e]);
    }
    if (a.y) rows.put(a.y, a.sy, g, t);
    p1 = p2 = both(0.f);
#pragma unroll
    for (int e = 0; e < P; e += 2) {
      const float4 A = factor_of(rows, 0, e / 2);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int i = e + h;
        if (R::TPR < 32 && t >= rows.rows) g[i] = both(0.f);
        sums[0][i] = add2(sums[0][i], g[i]);
        sums[1][i] = fma2(g[i], fh[i], sums[1][i]);
        g[i] = mul2(g[i], half_of(A, h));
        p1 = add2(p1, g[i]);
        p2 = fma2(g[i], fh[i], p2);
      }
    }
    if (a.n) {
      if (a.kind[0] != kNone) {
        float s1 = p1.x + p1.y, s2 = p2.x + p2.y;
        row_sum2<R::TPR>(s1, s2, red, 1);
        s1 *= centre[0];
        s2 *= inv;
#pragma unroll
        for (int e = 0; e < P; ++e) g[e] = mul2(fma2(fh[e], both(-s2), sub2(g[e], s1)), both(first.rstd));
      }
      rows.put(a.n, a.sn, g, t);
    }
    // a row's use of `red` ends before the next but one begins; where only one sum is taken, the row's
    // threads meet here
    if (R::TPR > 32 && (!a.dn || !a.n || a.kind[0] == kNone)) row_sync<R::TPR>();
  }
  // the CTA's sums: rows that share a warp by shuffles, then the warps of a column one after another
  asm volatile("cp.async.wait_group 0;" ::: "memory");
  float* total = (float*)smem;
#pragma unroll
  for (int k = 0; k < 4; ++k)
#pragma unroll
    for (int e = 0; e < P; ++e)
#pragma unroll
      for (int o = 16; o >= R::TPR; o >>= 1)
        sums[k][e] = add2(sums[k][e], make_float2(__shfl_xor_sync(~0u, sums[k][e].x, o), __shfl_xor_sync(~0u, sums[k][e].y, o)));
  constexpr int ROUNDS = R::TPR > 32 ? R::kGroups : R::kThreads / 32, CAPACITY = R::TPR * R::E;
  const int mine = R::TPR > 32 ? threadIdx.x / R::TPR : threadIdx.x / 32;
  const bool one = R::TPR >= 32 || (threadIdx.x & 31) < R::TPR;
  for (int q = 0; q < ROUNDS; ++q) {
    __syncthreads();
    if (mine != q || !one) continue;
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int e = 0; e < R::E; ++e) {
        float* to = total + k * CAPACITY + rows.column(e / R::V) + e % R::V;
        *to = (q ? *to : 0.f) + (e % 2 ? sums[k][e / 2].y : sums[k][e / 2].x);
      }
  }
  __syncthreads();
  float* part = a.part + (long long)blockIdx.x * 4 * a.cols;
  for (int k = 0; k < 4; ++k)
    for (int c = threadIdx.x; c < a.cols; c += R::kThreads) part[k * (long long)a.cols + c] = total[k * CAPACITY + c];
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

// The vectors' gradients from the CTAs' sums: COLS columns a CTA, whose lanes are the four sums of each; 256 /
// COLS runs of consecutive CTAs are added side by side and then in their order (a warp's in pairs, the
// warps' one after another).  Few columns go by two (59 columns of 304 CTAs: 5.7 us by eight), many by
// eight (3,584 columns: 17 us by two).
template <typename T, int COLS>
__global__ void __launch_bounds__(1024) close_sum_kernel(const __grid_constant__ CloseSums a) {
  pdl_wait();
  constexpr int LANES = 4 * COLS, RUNS = 1024 / LANES;
  __shared__ float run[32][LANES + 1];
  const int lane = threadIdx.x % LANES, k = threadIdx.x / LANES, which = lane / COLS, c = blockIdx.x * COLS + lane % COLS;
  float s = 0.f;
  if (c < a.cols) {
    const float* p = a.part + (long long)which * a.cols + c;
    const int q1 = (int)((long long)a.ctas * (k + 1) / RUNS);
#pragma unroll 5
    for (int q = (int)((long long)a.ctas * k / RUNS); q < q1; ++q) s += p[(long long)q * 4 * a.cols];
  }
#pragma unroll
  for (int o = LANES; o < 32; o *= 2) s += __shfl_xor_sync(~0u, s, o);
  if ((threadIdx.x & 31) < LANES) run[threadIdx.x / 32][lane] = s;
  __syncthreads();
  if (threadIdx.x >= 32) return;
  s = 0.f;
#pragma unroll
  for (int q = 0; q < 32; ++q) s += run[q][lane];
  const float s1 = __shfl_sync(~0u, s, lane % COLS), s2 = __shfl_sync(~0u, s, COLS + lane % COLS);
  if (threadIdx.x >= LANES || c >= a.cols) return;
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

constexpr int kCloseCtasPerSm = 2;    // backward at most, with sums in the workspace

// Calls f with the row shape for `cols` columns of T; f of an int where registers do not hold a row.
template <typename T, bool BWD, typename F> abcd_status with_row(long long cols, bool aligned, F&& f) {
  if (aligned) {
    constexpr int N = !BWD && sizeof(T) == 2 ? 2 : 1, E = 8 * N;
    if (cols <= 64) return f(CloseRow<T, 8 / N, E, BWD, true>());
    if (cols <= 128) return f(CloseRow<T, 16 / N, E, BWD, true>());
    if (cols <= 256) return f(CloseRow<T, 32 / N, E, BWD, true>());
    if (cols <= 512) return f(CloseRow<T, 64 / N, E, BWD, true>());
    if (cols <= 1024) return f(CloseRow<T, 128 / N, E, BWD, true>());
    if (cols <= 2048) return f(CloseRow<T, 256 / N, E, BWD, true>());
    if (cols <= 4096) return f(CloseRow<T, 512 / N, E, BWD, true>());
  } else {
    if (cols <= 64) return f(CloseRow<T, 8, 8, BWD, false>());
    if (cols <= 128) return f(CloseRow<T, 16, 8, BWD, false>());
    if (cols <= 256) return f(CloseRow<T, 32, 8, BWD, false>());
    if (cols <= 512) return f(CloseRow<T, 64, 8, BWD, false>());
    if (cols <= 1024) return f(CloseRow<T, 128, 8, BWD, false>());
    if (cols <= 2048) return f(CloseRow<T, 256, 8, BWD, false>());
    if (cols <= 4096) return f(CloseRow<T, 512, 8, BWD, false>());
  }
  return f(0);
}

template <typename K>
abcd_status launch_rows(abcd_ctx* ctx, const char* what, K* kernel, int grid, int threads, size_t smem, const CloseArgs& a) {
  if (smem > 47 * 1024) {
    const cudaError_t e = allow_smem(ctx, (const void*)kernel);
    if (e != cudaSuccess) return fail(ctx, ABCD_ERR_CUDA, "%s: %s", what, cudaGetErrorString(e));
  }
  return check_launch(ctx, what, launch_pdl(kernel, dim3((unsigned)grid), dim3((unsigned)threads), smem, ctx->stream, a));
}

// CTAs for rows of shape R: all of their rows at once, or as many as stay resident on `sms` SMs.
template <typename R> int grid_of(long long rows, int sms) {
  if constexpr (std::is_same_v<R, int>) return (int)std::min<long long>(rows, 2LL * sms);
  else return (int)std::min<long long>((rows + R::kGroups - 1) / R::kGroups, (long long)R::kCtas * sms);
}

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

// What a call is given, and whether a vector that it writes overlaps any of that, or a matrix that it writes a vector
// (matrices among themselves: same_or_apart).  Most bounds lie apart, which is all that is looked at then.
class Places {
  struct Range { uintptr_t first, end; };
  Range matrix_[6];                   // x, f, dy, dn and two results
  Range vector_[9], written_[5];      // two norms' four vectors and the gate; the gradients, or (of vector_) the statistics
  const abcd_matrix* of_[6];
  unsigned results_ = 0;              // of the matrices, a bit each
  int matrices_ = 0, vectors_ = 0, writtens_ = 0;
  static bool meet(const Range& p, const Range& q) { return p.first < q.end && q.first < p.end; }
  bool in_matrix(const Range& v, int k) const {
    if (!meet(v, matrix_[k])) return false;
    const long long halves = (long long)(v.end - v.first) / 2;          // as 16-bit elements
    const abcd_matrix row{(void*)v.first, 1, halves, halves, ABCD_F16};
    return overlap(&row, of_[k]);
  }

 public:
  void matrix(const abcd_matrix* m, bool result) {
    if (!m || m->rows == 0) return;
    const uintptr_t first = (uintptr_t)m->data, elements = (uintptr_t)((m->rows - 1) * m->stride + m->cols);
    matrix_[matrices_] = Range{first, first + elements * elem_size(m->dtype)};
    of_[matrices_] = m;
    results_ |= (result ? 1u : 0u) << matrices_++;
  }
  void vector(const void* p, long long n, int dtype, bool written) {
    if (!p || n == 0) return;
    const Range r{(uintptr_t)p, (uintptr_t)p + (uintptr_t)n * elem_size(dtype)};
    if (written) written_[writtens_++] = r;
    else vector_[vectors_++] = r;
  }
  void norm(const abcd_norm* q, long long rows, long long cols, int dtype, bool written) {
    if (!q) return;
    vector(q->weight, cols, dtype, false);
    vector(q->bias, cols, dtype, false);
    vector(q->mean, rows, ABCD_F32, written);
    vector(q->rstd, rows, ABCD_F32, written);
  }
  bool clash() const {
    for (int i = 0; i < writtens_; ++i) {
      for (int k = 0; k < matrices_; ++k)
        if (in_matrix(written_[i], k)) return true;
      for (int k = 0; k < vectors_; ++k)
        if (meet(written_[i], vector_[k])) return true;
      for (int k = 0; k < i; ++k)
        if (meet(written_[i], written_[k])) return true;
    }
    for (int k = 0; k < matrices_; ++k)
      if (results_ >> k & 1)
        for (int i = 0; i < vectors_; ++i)
          if (in_matrix(vector_[i], k)) return true;
    return false;
  }
};

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
  Places all;
  all.matrix(x, false);
  all.matrix(f, false);
  all.matrix(y, true);
  all.matrix(n, true);
  all.norm(after, x->rows, x->cols, weight_dtype, true);
  all.norm(before, x->rows, x->cols, weight_dtype, true);
  all.vector(gate, x->cols, weight_dtype, false);
  if (all.clash()) return fail(ctx, ABCD_ERR_INVALID_ARG, "%s: the statistics or an output overlap a vector or a matrix", what);
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
    const bool aligned = rows_aligned(x, 16) && rows_aligned(f, 16) && rows_aligned(y, 16) && (!n || rows_aligned(n, 16));
    return with_row<T, false>(x->cols, aligned, [&](auto shape) {
      using R = decltype(shape);
      const int grid = grid_of<R>(x->rows, ctx->num_sms);
      if constexpr (std::is_same_v<R, int>) return launch_rows(ctx, "close_fwd_long_kernel", close_fwd_long_kernel<T>, grid, kLongThreads, 0, a);
      else return launch_rows(ctx, "close_fwd_kernel", close_fwd_kernel<T, R>, grid, R::kThreads, R::kSmem, a);
    });
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
  Places all;
  for (const abcd_matrix* m : {dy, dn, x, f}) all.matrix(m, false);
  for (const abcd_matrix* m : {dx, df}) all.matrix(m, true);
  all.norm(after, x->rows, x->cols, weight_dtype, false);
  all.norm(before, x->rows, x->cols, weight_dtype, false);
  all.vector(gate, x->cols, weight_dtype, false);
  for (const void* p : to) all.vector(p, x->cols, weight_dtype, true);
  if (all.clash()) return fail(ctx, ABCD_ERR_INVALID_ARG, "%s: a vector's gradient overlaps what the call is given, or a gradient a vector", what);
  CloseArgs a{};
  a.x = x->data; a.f = f->data; a.dy = dy ? dy->data : nullptr; a.dn = dn ? dn->data : nullptr;
  a.y = dx ? dx->data : nullptr; a.n = df ? df->data : nullptr;
  a.sx = x->stride; a.sf = f->stride; a.sdy = dy ? dy->stride : 0; a.sdn = dn ? dn->stride : 0;
  a.sy = dx ? dx->stride : 0; a.sn = df ? df->stride : 0;
  a.gate = gate;
  take_norm(a, 0, after);
  take_norm(a, 1, before);
  // what the results do not depend on is not read: x without `before`, f without either norm and dgate
  if (!before) a.x = nullptr;
  if (!before && !after && !dgate) a.f = nullptr;
  a.scale = scale;
  a.wide_w = weight_dtype == ABCD_F32;
  a.rows = x->rows;
  a.cols = (int)x->cols;
  a.part = (float*)(ctx->net_base + kNetHeader);
  const int sms = std::min(ctx->num_sms, kNetSms);
  bool aligned = true;
  for (const abcd_matrix* m : {dy, dn, x, f, dx, df}) aligned = aligned && (!m || rows_aligned(m, 16));
  return with_type(x->dtype, [&](auto t) {
    using T = decltype(t);
    int ctas = 0;
    const abcd_status st = with_row<T, true>(x->cols, aligned, [&](auto shape) {
      using R = decltype(shape);
      ctas = grid_of<R>(x->rows, sms);
      const size_t need = kNetHeader + (size_t)ctas * 4 * (size_t)x->cols * sizeof(float);
      if (need > ctx->net_bytes)
        return fail(ctx, ABCD_ERR_WORKSPACE, "%s: the network workspace has %zu bytes, needs %zu", what, ctx->net_bytes, need);
      if (ctas == 0) return ABCD_OK;
      if constexpr (std::is_same_v<R, int>) {
        return launch_rows(ctx, "close_bwd_long_kernel", close_bwd_long_kernel<T>, ctas, kLongThreads, 0, a);
      } else {
        static_assert(R::kCtas <= kCloseCtasPerSm);
        return launch_rows(ctx, "close_bwd_kernel", close_bwd_kernel<T, R>, ctas, R::kThreads, R::kSmem, a);
      }
    });
    if (st != ABCD_OK) return st;
    if (std::all_of(to, to + 5, [](void* p) { return !p; })) return ABCD_OK;
    CloseSums s{a.part, ctas, a.cols, a.wide_w, scale, gate, a.w[0], a.b[0], {}};
    std::copy(to, to + 5, s.to);
    const bool wide = a.cols >= 8 * sms;                 // eight columns a CTA still give every SM one
    return check_launch(ctx, "close_sum_kernel", launch_pdl(wide ? close_sum_kernel<T, 8> : close_sum_kernel<T, 2>, dim3((unsigned)((a.cols + (wide ? 7 : 1)) / (wide ? 8 : 2))), dim3(1024), 0, ctx->stream, s));
  });
}
