// Layer norm over the rows of a matrix, forward and backward.
//   y = (x - mean) rstd w + b,   rstd = 1 / sqrt(mean((x - mean)^2) + eps)
//   g = dy w, xh = (x - mean) rstd:  dx = rstd (g - mean(g) - xh mean(g xh)),
//   dw = sum_rows dy xh,  db = sum_rows dy.
// The variance is taken from the deviations, not from the difference of two moments, so a mean far
// from zero costs it no digits.  Rows of one value have that value as their mean: what the division rounds
// is taken back, and where the sum may have rounded too, the deviations' own mean is.  (With a sum times a
// rounded reciprocal alone, 1,000 columns of 1000.0 had a mean one unit higher, and xh of 0.019 instead of 0.)
//
// Bound by HBM (forward x -> y, backward x, dy -> dx).  A row is read once: TPR lanes (part of a
// warp, a warp, or a CTA) hold it in registers, NV vectors of V consecutive elements (16 bytes) each;
// rows too long for that are read again from L2.  A group of lanes takes many rows: the weights (and backward dw
// and db of its own columns) stay in registers, and the next rows are copied to shared memory
// meanwhile (cp.async), which keeps the loads in flight that the few warps of so many registers could
// not.  100,000 x 1,024 bf16: forward 66 us and backward 101 (both 6.2 TB/s), and 2.4 us for the sums;
// one CTA per row without any of this took 520 and 820.  The CTAs' sums go to the workspace and a
// second kernel adds them in their order.
// Rows that start anywhere are bound by instructions (each vector is put together from two pieces, results
// go to shared memory element by element, and the row's threads meet three times a turn): 1,000,000 x 59
// without gaps 156 and 208 us in fp32, 124 and 190 in fp16; with rows 64 apart 120 and 138, 74 and 89.
#include <algorithm>
#include <type_traits>

#include "network.cuh"

namespace abcd {
namespace {

struct NormArgs {
  const void* x;
  const void* dy;
  const void* w;
  const void* b;
  void* y;                            // forward: y; backward: dx
  const void* res;                    // backward: added to dx, or NULL
  float* mean;
  float* rstd;
  float* part;                        // [grid][2][cols] sums of a CTA's rows
  long long rows;
  int cols;
  long long sx, sdy, sy, sres;
  float eps;
  int wide_w;                         // weight and bias are fp32 whatever the matrices' type
  void* dw;                           // backward in one CTA: the sums' places, or NULL
  void* db;
};

// How a row lies over threads, forward (one matrix is read) and backward (two); SHIFT: rows that
// start anywhere.
template <int TPR_, int V_, int NV_, bool BWD, bool SHIFT> struct RowShape {
  static constexpr int TPR = TPR_, V = V_, NV = NV_;
  static constexpr bool kShift = SHIFT;
  static constexpr int kThreads = TPR > 256 ? TPR : 256;
  static constexpr int kGroups = kThreads / TPR;          // rows of a CTA at a time
  static constexpr int kCapacity = TPR * V * NV;
  // Shared memory: four rows of each matrix per group (three where four leave no room for a second
  // CTA), a row as its vectors (and one more, which a row that starts between two reaches into), and,
  // backward, the sums of the CTA's columns at its end.
  static constexpr int kMats = BWD ? 2 : 1;
  static constexpr int kRowBytes = (TPR * NV + (SHIFT ? 1 : 0)) * 16;
  static constexpr size_t kAhead = (size_t)kMats * kGroups * kRowBytes;
  static constexpr int kDepth = 4 * kAhead > 100 * 1024 ? 3 : 4;
  static constexpr size_t kRing = kDepth * kAhead, kSums = BWD ? (size_t)2 * kCapacity * 4 : 0;
  static constexpr size_t kSmem = kRing > kSums ? kRing : kSums;
  // CTAs per SM: as many as their registers (and rows) leave room for.  Short rows backward are held to
  // the registers of three CTAs, or of four in 32 bits (1,000,000 x 64 bf16: 75 us, and 89 with two CTAs
  // of as many registers as they like; rows that start anywhere of eight values a thread spill at three).
  static constexpr bool kShort = V * NV <= 8;
  // Whether the sum of a row of one value may round: of up to 8,192 16-bit values (11 bits each) it is exact.
  static constexpr bool kRounds = V == 4 || kCapacity > 8192;
  static constexpr int kCtas = kThreads > 256 || kSmem > 100 * 1024 ? 1
                               : !kShort || (BWD && SHIFT && V * NV == 8) ? 2
                               : BWD && (SHIFT || V * NV == 8) ? 3 : 4;
};

template <typename T, int V>
__device__ __forceinline__ void load_vec(float (&v)[V], const T* p, int left) {
  if (V > 1 && left >= V) {
    const Pack<T, V> q = *reinterpret_cast<const Pack<T, V>*>(p);
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = to_f32(q.v[i]);
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = i < left ? to_f32(p[i]) : 0.f;
  }
}
template <typename T, int V>
__device__ __forceinline__ void store_vec(T* p, const float (&v)[V], int left) {
  if (V > 1 && left >= V) {
    Pack<T, V> q;
#pragma unroll
    for (int i = 0; i < V; ++i) q.v[i] = from_f32<T>(v[i]);
    *reinterpret_cast<Pack<T, V>*>(p) = q;
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (i < left) p[i] = from_f32<T>(v[i]);
  }
}
// V elements of a weight vector of T or fp32, `none` where there is no vector.
template <typename T, int V>
__device__ __forceinline__ void load_weight(float (&v)[V], const void* w, int wide, int c, int left, float none) {
  if (!w) {
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = none;
  } else if (wide && V % 4 == 0 && left >= V && ((uintptr_t)w & 15) == 0) {
#pragma unroll
    for (int i = 0; i < V / 4 * 4; i += 4) {
      const float4 q = __ldg(reinterpret_cast<const float4*>((const float*)w + c + i));
      v[i] = q.x; v[i + 1] = q.y; v[i + 2] = q.z; v[i + 3] = q.w;
    }
  } else if (wide) {
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = i < left ? __ldg((const float*)w + c + i) : 0.f;
  } else if (V > 1 && left >= V && ((uintptr_t)w & (sizeof(T) * V - 1)) == 0) {
    load_vec<T, V>(v, (const T*)w + c, V);
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = i < left ? to_f32(((const T*)w)[c + i]) : 0.f;
  }
}

// Sums of a and b over the TPR threads of a row, in each of them.  Rows of several warps meet in
// red (turn: which half of it this row uses; a row's use ends before the next but one begins).
template <int TPR>
__device__ __forceinline__ void row_sum2(float& a, float& b, float2 (*red)[32], int turn) {
#pragma unroll
  for (int o = (TPR < 32 ? TPR : 32) / 2; o; o >>= 1) {
    a += __shfl_xor_sync(~0u, a, o);
    b += __shfl_xor_sync(~0u, b, o);
  }
  if constexpr (TPR > 32) {
    constexpr int WARPS = TPR / 32;
    const int w = threadIdx.x / 32, first = w / WARPS * WARPS;
    if ((threadIdx.x & 31) == 0) red[turn][w] = make_float2(a, b);
    // the row's warps alone: barriers 1 ... of the CTA's rows
    asm volatile("bar.sync %0, %1;" ::"r"(1 + (int)threadIdx.x / TPR), "n"(TPR) : "memory");
    a = b = 0.f;
#pragma unroll
    for (int k = 0; k < WARPS; ++k) {
      a += red[turn][first + k].x;
      b += red[turn][first + k].y;
    }
  }
}

// rstd from the mean of the squared deviations from a point that lies `off` below the mean.
__device__ __forceinline__ float rstd_of(float squares, float off, float eps) {
  const float var = squares - off * off;
  return rsqrtf((var < 0.f ? 0.f : var) + eps);        // NaN stays NaN
}

// Asynchronous copy of min(16, bytes) bytes to 16 bytes of shared memory, zeros after them.
__device__ __forceinline__ void copy16(void* dst, const void* src, int bytes) {
  const unsigned d = (unsigned)__cvta_generic_to_shared(dst);
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(d), "l"(src), "r"(bytes < 16 ? bytes : 16) : "memory");
}

// The threads of a row meet.
template <int TPR> __device__ __forceinline__ void row_sync() {
  if constexpr (TPR <= 32) __syncwarp();
  else asm volatile("bar.sync %0, %1;" ::"r"(1 + (int)threadIdx.x / TPR), "n"(TPR) : "memory");
}

// The rows that a group of TPR threads takes one after another, their next ones on the way to shared
// memory [depth][matrix][group][vectors of 16 bytes].
//
// Rows on 16-byte boundaries: each thread copies the vectors that it will use itself, so nobody waits
// for another.  Rows that start anywhere (SHIFT): the 16-byte pieces that they reach into are copied,
// the group meets, and each thread puts its vectors together from two pieces.  A piece then also holds
// up to 14 bytes of what lies before or behind the row in its matrix; pieces that reach outside the
// matrix (of its first and last row) are copied element by element.
template <typename T, typename R> struct RowRing {
  static constexpr int kDepth = R::kDepth;
  char* slots;                        // the group's first slot
  const T* src[R::kMats];             // the start of the next row to fetch
  const char* lowest[R::kMats];       // the matrices' first bytes, and the ones behind their last
  const char* highest[R::kMats];
  long long jump[R::kMats];           // elements from one of the group's rows to its next
  int rows, turns;                    // the group's rows; turns of the CTA, alike in all its groups
  int cols, lane;
  int left;                           // elements of a row from the thread's first vector on

  __device__ __forceinline__ RowRing(char* smem, const NormArgs& a) {
    const int group = threadIdx.x / R::TPR;
    const long long first = (long long)blockIdx.x * R::kGroups + group, step = (long long)gridDim.x * R::kGroups;
    lane = threadIdx.x % R::TPR;
    cols = a.cols;
    slots = smem + group * R::kRowBytes;
    left = a.cols - lane * R::V;
    rows = first < a.rows ? (int)((a.rows - first + step - 1) / step) : 0;
    turns = (int)((a.rows - (long long)blockIdx.x * R::kGroups + step - 1) / step);
    const T* base[2] = {(const T*)a.x, (const T*)a.dy};
    const long long stride[2] = {a.sx, a.sdy};
#pragma unroll
    for (int q = 0; q < R::kMats; ++q) {
      src[q] = base[q] + first * stride[q];
      jump[q] = step * stride[q];
      lowest[q] = (const char*)base[q];
      highest[q] = (const char*)(base[q] + (a.rows - 1) * stride[q] + a.cols);
    }
  }
  __device__ __forceinline__ char* slot(int t, int mat) const {
    return slots + (t % kDepth * R::kMats + mat) * R::kGroups * R::kRowBytes;
  }
  // Piece i of a row that starts anywhere.
  __device__ __forceinline__ void piece(int t, int q, int i) const {
    const char* begin = (const char*)src[q];
    const char* from = begin - ((uintptr_t)begin & 15) + 16 * i;
    const char* end = (const char*)(src[q] + cols);
    if (from >= end) return;
    char* to = slot(t, q) + 16 * i;
    if (from >= lowest[q] && from + 16 <= highest[q]) {
      copy16(to, from, 16);
    } else {
#pragma unroll
      for (int e = 0; e < 16; e += (int)sizeof(T))
        if (from + e >= begin && from + e < end) *reinterpret_cast<T*>(to + e) = *reinterpret_cast<const T*>(from + e);
    }
  }
  __device__ __forceinline__ void fetch(int t) {
    if (t < rows) {
#pragma unroll
      for (int q = 0; q < R::kMats; ++q) {
#pragma unroll
        for (int j = 0; j < R::NV; ++j) {
          const int n = left - j * R::TPR * R::V;
          if constexpr (R::kShift) piece(t, q, j * R::TPR + lane);
          else if (n > 0) copy16(slot(t, q) + (j * R::TPR + lane) * 16, src[q] + lane * R::V + j * R::TPR * R::V, n < R::V ? n * (int)sizeof(T) : 16);
        }
        if (R::kShift && lane == 0) piece(t, q, R::NV * R::TPR);
        src[q] += jump[q];
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  }
  __device__ __forceinline__ void start() {
#pragma unroll
    for (int d = 0; d < kDepth - 1; ++d) fetch(d);
  }
  // Asks for the row kDepth - 1 turns on and waits for the one of turn t.
  __device__ __forceinline__ void turn(int t) {
    if constexpr (R::kShift) row_sync<R::TPR>();       // the last turn's row is done with
    fetch(t + kDepth - 1);
    asm volatile("cp.async.wait_group %0;" ::"n"(kDepth - 1) : "memory");
    if constexpr (R::kShift) row_sync<R::TPR>();
  }
  // Vector j of the turn's row of a matrix (at: where the row starts); zeros past its end.
  __device__ __forceinline__ void get(float (&v)[R::V], int t, int mat, int j, const T* at) const {
    const int n = t < rows ? left - j * R::TPR * R::V : 0, c = (j * R::TPR + lane) * R::V;
    if constexpr (!R::kShift) {
      load_vec<T, R::V>(v, (const T*)(slot(t, mat) + c * sizeof(T)), n > 0 ? R::V : 0);
    } else {
      const int p = (int)((uintptr_t)at & 15) + c * (int)sizeof(T);
      const unsigned* w = reinterpret_cast<const unsigned*>(slot(t, mat) + (p & ~3));
      unsigned u[5];
#pragma unroll
      for (int i = 0; i < 5; ++i) u[i] = n > 0 && (i < 4 || (p & 2)) ? w[i] : 0u;
      if (p & 2) {
#pragma unroll
        for (int i = 0; i < 4; ++i) u[i] = u[i] >> 16 | u[i + 1] << 16;
      }
      Pack<T, R::V> q;
#pragma unroll
      for (int i = 0; i < 4; ++i) reinterpret_cast<unsigned*>(&q)[i] = u[i];
#pragma unroll
      for (int i = 0; i < R::V; ++i) v[i] = i < n ? to_f32(q.v[i]) : 0.f;
    }
  }
  // The turn's row of results to `to`: each thread puts its vectors' values, then all store pieces.
  __device__ __forceinline__ void put(const float (&v)[R::V], int t, int j, T* to) const {
    const int c = (j * R::TPR + lane) * R::V, n = t < rows ? left - j * R::TPR * R::V : 0;
    if (n <= 0) return;
    if constexpr (!R::kShift) {
      store_vec<T, R::V>(to + c, v, n);
    } else {
      T* s = reinterpret_cast<T*>(slot(t, 0) + ((uintptr_t)to & 15)) + c;
#pragma unroll
      for (int i = 0; i < R::V; ++i) s[i] = from_f32<T>(v[i]);     // the row's place has room for a vector more
    }
  }
  __device__ __forceinline__ void flush(int t, T* to) const {
    if constexpr (R::kShift) {
      row_sync<R::TPR>();
      if (t >= rows) return;
      char* begin = (char*)to;
      char* end = (char*)(to + cols);
      char* base = begin - ((uintptr_t)begin & 15);
      const char* s = slot(t, 0);
#pragma unroll
      for (int j = 0; j <= R::NV; ++j) {
        const int i = j * R::TPR + lane;
        if (j == R::NV && lane > 0) break;
        char* at = base + 16 * i;
        if (at >= end) break;
        if (at >= begin && at + 16 <= end) {
          *reinterpret_cast<uint4*>(at) = *reinterpret_cast<const uint4*>(s + 16 * i);
        } else {
#pragma unroll
          for (int e = 0; e < 16; e += (int)sizeof(T))
            if (at + e >= begin && at + e < end) *reinterpret_cast<T*>(at + e) = *reinterpret_cast<const T*>(s + 16 * i + e);
        }
      }
    }
  }
};

// (Rows of 32 values a thread are held to the registers of the CTAs that the grid counts on: 10,000 x 1,500
// fp32 25 us, and 29 with 141 registers.)
template <typename T, typename R>
__global__ void __launch_bounds__(R::kThreads, R::V * R::NV == 32 ? R::kCtas : 0) norm_fwd_kernel(const __grid_constant__ NormArgs a) {
  constexpr int V = R::V, NV = R::NV, TPR = R::TPR;
  extern __shared__ char smem[];
  __shared__ float2 red[2][32];
  pdl_wait();
  const int lane = threadIdx.x % TPR;
  RowRing<T, R> ring(smem, a);
  ring.start();
  float w[NV][V], b[NV][V];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int c = (j * TPR + lane) * V;
    load_weight<T, V>(w[j], a.w, a.wide_w, c, a.cols - c, 1.f);
    load_weight<T, V>(b[j], a.b, a.wide_w, c, a.cols - c, 0.f);
  }
  const float inv = 1.f / (float)a.cols;
  const long long step = (long long)gridDim.x * R::kGroups;
  long long r = (long long)blockIdx.x * R::kGroups + threadIdx.x / TPR;
  const T* x = (const T*)a.x + r * a.sx;
  T* y = (T*)a.y + r * a.sy;
  for (int t = 0; t < ring.turns; ++t, r += step, x += step * a.sx, y += step * a.sy) {
    ring.turn(t);
    float v[NV][V], s = 0.f, q = 0.f, unused = 0.f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      ring.get(v[j], t, 0, j, x);
#pragma unroll
      for (int i = 0; i < V; ++i) s += v[j][i];
    }
    row_sum2<TPR>(s, unused, red, 0);
    // the division's rounding taken back, then, where the sum has rounded too, the sum's
    float mean = s * inv;
    mean = __fmaf_rn(__fmaf_rn(-mean, (float)a.cols, s), inv, mean);
    float e = 0.f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int left = ring.left - j * TPR * V;
      if (left < V) {                                  // past the row's end nothing deviates
#pragma unroll
        for (int i = 0; i < V; ++i) v[j][i] = i < left ? v[j][i] : mean;
      }
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float d = v[j][i] - mean;
        q += d * d;
        if constexpr (R::kRounds) e += d;
        else v[j][i] = d;
      }
    }
    row_sum2<TPR>(q, e, red, 1);
    e *= inv;
    if constexpr (R::kRounds) {
      mean += e;
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < V; ++i) v[j][i] -= mean;
    }
    const float rstd = rstd_of(q * inv, e, a.eps);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
#pragma unroll
      for (int i = 0; i < V; ++i) v[j][i] = v[j][i] * rstd * w[j][i] + b[j][i];
      ring.put(v[j], t, j, y);
    }
    ring.flush(t, y);
    if (t >= ring.rows) continue;
    if (a.mean && lane == 0) {
      a.mean[r] = mean;
      a.rstd[r] = rstd;
    }
  }
}

template <typename T, typename R>
__global__ void __launch_bounds__(R::kThreads, R::kShort ? R::kCtas : 0) norm_bwd_kernel(const __grid_constant__ NormArgs a) {
  constexpr int V = R::V, NV = R::NV, TPR = R::TPR;
  extern __shared__ char smem[];
  __shared__ float2 red[2][32];
  pdl_wait();
  const int lane = threadIdx.x % TPR;
  RowRing<T, R> ring(smem, a);
  ring.start();
  float w[NV][V], dw[NV][V] = {}, db[NV][V] = {};
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int c = (j * TPR + lane) * V;
    load_weight<T, V>(w[j], a.w, a.wide_w, c, a.cols - c, 1.f);
  }
  const float inv = 1.f / (float)a.cols;
  const long long step = (long long)gridDim.x * R::kGroups;
  long long r = (long long)blockIdx.x * R::kGroups + threadIdx.x / TPR;
  const T* x = (const T*)a.x + r * a.sx;
  const T* dy = (const T*)a.dy + r * a.sdy;
  T* dx = (T*)a.y + r * a.sy;
  const T* res = (const T*)a.res + r * a.sres + lane * V;
  // mean and rstd of the rows come two turns ahead too
  auto stat_of = [&](int t, long long row) {
    return t < ring.rows ? make_float2(__ldg(a.mean + row), __ldg(a.rstd + row)) : make_float2(0.f, 0.f);
  };
  float2 stat[2] = {stat_of(0, r), stat_of(1, r + step)};
  for (int t = 0; t < ring.turns; ++t, r += step, x += step * a.sx, dy += step * a.sdy, dx += step * a.sy, res += step * a.sres) {
    ring.turn(t);
    const bool in = t < ring.rows;
    const float mean = stat[0].x, rstd = stat[0].y;
    stat[0] = stat[1];
    stat[1] = stat_of(t + 2, r + 2 * step);
    // past the row's end dy is zero, and so is what xh meets there
    float xh[NV][V], g[NV][V], s1 = 0.f, s2 = 0.f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      ring.get(xh[j], t, 0, j, x);
      ring.get(g[j], t, 1, j, dy);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        xh[j][i] = (xh[j][i] - mean) * rstd;           // the forward pass's value, bit for bit
        dw[j][i] += g[j][i] * xh[j][i];
        db[j][i] += g[j][i];
        g[j][i] *= w[j][i];
        s1 += g[j][i];
        s2 += g[j][i] * xh[j][i];
      }
    }
    row_sum2<TPR>(s1, s2, red, t & 1);
    s1 *= -inv * rstd;
    s2 *= -inv * rstd;
    if (a.y) {
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const int left = in ? ring.left - j * TPR * V : 0;
        float v[V];
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = xh[j][i] * s2 + (rstd * g[j][i] + s1);
        if (a.res && left > 0) {
          float add[V];
          if constexpr (R::kShift) {
#pragma unroll
            for (int i = 0; i < V; ++i) add[i] = i < left ? to_f32(res[j * TPR * V + i]) : 0.f;
          } else {
            load_vec<T, V>(add, res + j * TPR * V, left);
          }
#pragma unroll
          for (int i = 0; i < V; ++i) v[i] += add[i];
        }
        ring.put(v, t, j, dx);
      }
      ring.flush(t, dx);
    }
  }
  // the CTA's sums: rows that share a warp by shuffles, then the warps of a column one after another
  if (V > 1) asm volatile("cp.async.wait_group 0;" ::: "memory");
  float* sums = (float*)smem;
#pragma unroll
  for (int j = 0; j < NV; ++j)
#pragma unroll
    for (int i = 0; i < V; ++i)
#pragma unroll
      for (int o = 16; o >= TPR; o >>= 1) {
        dw[j][i] += __shfl_xor_sync(~0u, dw[j][i], o);
        db[j][i] += __shfl_xor_sync(~0u, db[j][i], o);
      }
  constexpr int ROUNDS = TPR > 32 ? R::kGroups : R::kThreads / 32;
  const int mine = TPR > 32 ? threadIdx.x / TPR : threadIdx.x / 32;
  const bool one = TPR >= 32 || (threadIdx.x & 31) < TPR;
  for (int k = 0; k < ROUNDS; ++k) {
    __syncthreads();
    if (mine != k || !one) continue;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const int c = (j * TPR + lane) * V + i;
        sums[c] = (k ? sums[c] : 0.f) + dw[j][i];
        sums[R::kCapacity + c] = (k ? sums[R::kCapacity + c] : 0.f) + db[j][i];
      }
  }
  __syncthreads();
  if (gridDim.x == 1) {                // nothing to add up
    for (int c = threadIdx.x; c < a.cols; c += R::kThreads) {
      const float s[2] = {sums[c], sums[R::kCapacity + c]};
      void* const to[2] = {a.dw, a.db};
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        if (!to[k]) continue;
        if (a.wide_w) ((float*)to[k])[c] = s[k];
        else ((T*)to[k])[c] = from_f32<T>(s[k]);
      }
    }
    return;
  }
  float* part = a.part + (long long)blockIdx.x * 2 * a.cols;
  for (int c = threadIdx.x; c < a.cols; c += R::kThreads) {
    part[c] = sums[c];
    part[a.cols + c] = sums[R::kCapacity + c];
  }
}

// Rows too long for registers (past 16,384 columns forward and 8,192 backward): one CTA
// per row, read again for each use (from L2), element by element.  2,000 x 32,768 bf16 takes 142 and 535 us
// for bytes of 39 and 58; no part of this package makes tokens that wide.
constexpr int kLongThreads = 1024;

template <typename T>
__global__ void __launch_bounds__(kLongThreads) norm_fwd_long_kernel(const __grid_constant__ NormArgs a) {
  pdl_wait();
  __shared__ float2 red[2][32];
  for (long long r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const T* x = (const T*)a.x + r * a.sx;
    T* y = (T*)a.y + r * a.sy;
    float s = 0.f, q = 0.f, unused = 0.f;
    for (int c = threadIdx.x; c < a.cols; c += kLongThreads) s += to_f32(x[c]);
    row_sum2<kLongThreads>(s, unused, red, 0);
    const float about = s / (float)a.cols;
    float e = 0.f;
    for (int c = threadIdx.x; c < a.cols; c += kLongThreads) {
      const float d = to_f32(x[c]) - about;
      q += d * d;
      e += d;
    }
    row_sum2<kLongThreads>(q, e, red, 1);
    e /= (float)a.cols;
    const float mean = about + e, rstd = rstd_of(q / (float)a.cols, e, a.eps);
    for (int c = threadIdx.x; c < a.cols; c += kLongThreads) {
      float w[1], b[1];
      load_weight<T, 1>(w, a.w, a.wide_w, c, 1, 1.f);
      load_weight<T, 1>(b, a.b, a.wide_w, c, 1, 0.f);
      y[c] = from_f32<T>((to_f32(x[c]) - mean) * rstd * w[0] + b[0]);
    }
    if (a.mean && threadIdx.x == 0) {
      a.mean[r] = mean;
      a.rstd[r] = rstd;
    }
  }
}

template <typename T>
__global__ void __launch_bounds__(kLongThreads) norm_bwd_long_kernel(const __grid_constant__ NormArgs a) {
  pdl_wait();
  __shared__ float2 red[2][32];
  float* pw = a.part + (long long)blockIdx.x * 2 * a.cols;
  float* pb = pw + a.cols;
  for (int c = threadIdx.x; c < a.cols; c += kLongThreads) pw[c] = pb[c] = 0.f;
  const float inv = 1.f / (float)a.cols;
  int turn = 0;
  for (long long r = blockIdx.x; r < a.rows; r += gridDim.x, turn ^= 1) {
    const T* x = (const T*)a.x + r * a.sx;
    const T* dy = (const T*)a.dy + r * a.sdy;
    T* dx = (T*)a.y + r * a.sy;
    const float mean = a.mean[r], rstd = a.rstd[r];
    float s1 = 0.f, s2 = 0.f;
    for (int c = threadIdx.x; c < a.cols; c += kLongThreads) {
      const float d = to_f32(dy[c]), xh = (to_f32(x[c]) - mean) * rstd;
      float w[1];
      load_weight<T, 1>(w, a.w, a.wide_w, c, 1, 1.f);
      s1 += d * w[0];
      s2 += d * w[0] * xh;
      pw[c] += d * xh;
      pb[c] += d;
    }
    row_sum2<kLongThreads>(s1, s2, red, turn);
    s1 *= inv;
    s2 *= inv;
    if (a.y)
      for (int c = threadIdx.x; c < a.cols; c += kLongThreads) {
        const float d = to_f32(dy[c]), xh = (to_f32(x[c]) - mean) * rstd;
        float w[1];
        load_weight<T, 1>(w, a.w, a.wide_w, c, 1, 1.f);
        const float res = a.res ? to_f32(((const T*)a.res)[r * a.sres + c]) : 0.f;
        dx[c] = from_f32<T>(rstd * (d * w[0] - s1 - xh * s2) + res);
      }
  }
}

// dw and db from the CTAs' sums: COLS columns per CTA, 1024 / COLS runs of consecutive CTAs added side by
// side and then in their order (the runs of a warp in pairs, the warps' one after another).  Of 32
// columns, which are few CTAs and a long chain of loads, 59 columns take 4.6 us; of eight 2.2.
template <typename W, int COLS>
__global__ void __launch_bounds__(1024) norm_sum_kernel(const float* part, int ctas, int cols, W* dw, W* db) {
  pdl_wait();
  constexpr int RUNS = 1024 / COLS;
  __shared__ float run[32][COLS + 1];
  const int lane = threadIdx.x % COLS, k = threadIdx.x / COLS;
  const int c = blockIdx.x * COLS + lane;          // of [dw | db]
  float s = 0.f;
  if (c < 2 * cols) {
    const int k0 = ctas * k / RUNS, k1 = ctas * (k + 1) / RUNS;
#pragma unroll 5
    for (int q = k0; q < k1; ++q) s += part[(long long)q * 2 * cols + c];
  }
#pragma unroll
  for (int o = COLS; o < 32; o *= 2) s += __shfl_xor_sync(~0u, s, o);
  if ((threadIdx.x & 31) < COLS) run[threadIdx.x / 32][lane] = s;
  __syncthreads();
  if (k || c >= 2 * cols) return;
  s = 0.f;
#pragma unroll
  for (int q = 0; q < 32; ++q) s += run[q][lane];
  W* out = c < cols ? dw : db;
  if (out) out[c < cols ? c : c - cols] = from_f32<W>(s);
}

constexpr int kNormCtasPerSm = 4;

// Calls f with the row shape for `cols` columns of T: the fewest threads whose registers hold a row,
// 32 elements a thread forward (with as many weights and biases) and 16 backward (with as many
// weights and sums); f of an int where none does.  Backward, 100,000 x 1,024 bf16 with 32 elements a
// thread (eight warps per SM) took 164 us, with 16 it takes 100.
template <typename T, bool BWD, bool SHIFT, typename F> abcd_status with_shape(long long cols, F&& f) {
  constexpr int V = 16 / sizeof(T), N = (BWD ? 16 : 32) / V;   // vectors of 16 bytes per thread
  if (cols <= 8 * V) return f(RowShape<8, V, 1, BWD, SHIFT>());
  if (cols <= 16 * V) return f(RowShape<16, V, 1, BWD, SHIFT>());
  if (cols <= 32 * V) return f(RowShape<32, V, 1, BWD, SHIFT>());
  if (cols <= 64 * V) return f(RowShape<32, V, 2, BWD, SHIFT>());
  if (cols <= 32 * V * N) return f(RowShape<32, V, N, BWD, SHIFT>());
  if (cols <= 64 * V * N) return f(RowShape<64, V, N, BWD, SHIFT>());
  if (cols <= 128 * V * N) return f(RowShape<128, V, N, BWD, SHIFT>());
  if (cols <= 256 * V * N) return f(RowShape<256, V, N, BWD, SHIFT>());
  if (cols <= 512 * V * N) return f(RowShape<512, V, N, BWD, SHIFT>());
  return f(0);
}
template <typename T, bool BWD, typename F> abcd_status with_shape(long long cols, bool aligned, F&& f) {
  return aligned ? with_shape<T, BWD, false>(cols, f) : with_shape<T, BWD, true>(cols, f);
}

abcd_status room_for(abcd_ctx* ctx, const void* kernel, size_t smem) {
  if (smem <= 47 * 1024) return ABCD_OK;
  const cudaError_t e = allow_smem(ctx, kernel);
  return e == cudaSuccess ? ABCD_OK : fail(ctx, ABCD_ERR_CUDA, "layer norm: %s", cudaGetErrorString(e));
}

bool weights_ok(const abcd_matrix* x, int wtype, const void* a, const void* b) {
  return (wtype == ABCD_F32 || wtype == x->dtype) &&
         (((uintptr_t)a | (uintptr_t)b) & (elem_size(wtype) - 1)) == 0;
}

}  // namespace

int norm_bwd_ctas(int num_sms) { return kNormCtasPerSm * num_sms; }

}  // namespace abcd

using namespace abcd;

extern "C" abcd_status abcd_layer_norm(abcd_ctx* ctx, const abcd_matrix* x, const void* weight,
                                       const void* bias, int weight_dtype, float eps,
                                       const abcd_matrix* y, float* mean, float* rstd) {
  if (!ctx) return ABCD_ERR_INVALID_ARG;
  if (!matrix_ok(x) || !matrix_ok(y) || !same_form(x, y))
    return fail(ctx, ABCD_ERR_INVALID_ARG, "abcd_layer_norm: bad matrices");
  if (!weights_ok(x, weight_dtype, weight, bias))
    return fail(ctx, ABCD_ERR_INVALID_ARG, "abcd_layer_norm: bad weight or bias");
  if (!(eps >= 0.f && eps < 1e30f) || (mean == nullptr) != (rstd == nullptr))
    return fail(ctx, ABCD_ERR_INVALID_ARG, "abcd_layer_norm: bad eps or statistics");
  if (x->rows == 0) return ABCD_OK;
  const NormArgs a{x->data, nullptr, weight, bias, y->data, nullptr, mean, rstd, nullptr, x->rows,
                   (int)x->cols, x->stride, 0, y->stride, 0, eps, weight_dtype == ABCD_F32, nullptr, nullptr};
  return with_type(x->dtype, [&](auto t) {
    using T = decltype(t);
    return with_shape<T, false>(x->cols, rows_aligned(x, 16) && rows_aligned(y, 16), [&](auto shape) {
      using R = decltype(shape);
      if constexpr (std::is_same_v<R, int>) {
        const unsigned grid = (unsigned)std::min<long long>(x->rows, 2LL * ctx->num_sms);
        return check_launch(ctx, "norm_fwd_long_kernel", launch_pdl(norm_fwd_long_kernel<T>, dim3(grid), dim3(kLongThreads), 0, ctx->stream, a));
      } else {
        auto* kernel = norm_fwd_kernel<T, R>;
        const abcd_status st = room_for(ctx, (const void*)kernel, R::kSmem);
        if (st != ABCD_OK) return st;
        const unsigned grid = (unsigned)std::min<long long>((x->rows + R::kGroups - 1) / R::kGroups, R::kCtas * ctx->num_sms);
        return check_launch(ctx, "norm_fwd_kernel", launch_pdl(kernel, dim3(grid), dim3(R::kThreads), R::kSmem, ctx->stream, a));
      }
    });
  });
}

extern "C" abcd_status abcd_layer_norm_backward(abcd_ctx* ctx, const abcd_matrix* dy,
                                                const abcd_matrix* x, const void* weight,
                                                int weight_dtype, const float* mean,
                                                const float* rstd, const abcd_matrix* d_residual,
                                                const abcd_matrix* dx, void* dweight, void* dbias) {
  if (!ctx) return ABCD_ERR_INVALID_ARG;
  if (!matrix_ok(x) || !matrix_ok(dy) || !same_form(x, dy) ||
      (dx && (!matrix_ok(dx) || !same_form(x, dx))) ||
      (d_residual && (!dx || !matrix_ok(d_residual) || !same_form(x, d_residual))))
    return fail(ctx, ABCD_ERR_INVALID_ARG, "abcd_layer_norm_backward: bad matrices");
  if (!weights_ok(x, weight_dtype, weight, nullptr) || !weights_ok(x, weight_dtype, dweight, dbias))
    return fail(ctx, ABCD_ERR_INVALID_ARG, "abcd_layer_norm_backward: bad weight or gradients");
  if (x->rows > 0 && (!mean || !rstd))
    return fail(ctx, ABCD_ERR_INVALID_ARG, "abcd_layer_norm_backward: no statistics");
  const int sms = std::min(ctx->num_sms, kNetSms);
  float* part = (float*)(ctx->net_base + kNetHeader);
  const bool aligned = rows_aligned(x, 16) && rows_aligned(dy, 16) && (!dx || rows_aligned(dx, 16)) &&
                       (!d_residual || rows_aligned(d_residual, 16));
  NormArgs a{x->data, dy->data, weight, nullptr, dx ? dx->data : nullptr, d_residual ? d_residual->data : nullptr,
             (float*)mean, (float*)rstd, part, x->rows, (int)x->cols, x->stride, dy->stride, dx ? dx->stride : 0,
             d_residual ? d_residual->stride : 0, 0.f, weight_dtype == ABCD_F32, dweight, dbias};
  int ctas = 0;
  bool one = false;
  const abcd_status st = with_type(x->dtype, [&](auto t) {
    using T = decltype(t);
    return with_shape<T, true>(x->cols, aligned, [&](auto shape) {
      using R = decltype(shape);
      // CTAs: as many rows at a time as stay resident, each with its sums in the workspace
      constexpr bool kLong = std::is_same_v<R, int>;
      if constexpr (kLong) {
        ctas = (int)std::min<long long>(x->rows, 2LL * sms);
      } else {
        static_assert(R::kCtas <= kNormCtasPerSm);
        // with fewer than twelve turns a CTA, a third and fourth CTA per SM cost the kernel that adds up
        // their sums more than they gain (100,000 x 64 bf16: 11.7 us with two, 12.1 with three)
        const long long turns = (x->rows + R::kGroups - 1) / R::kGroups;
        ctas = (int)std::min<long long>(turns, std::clamp<long long>(turns / (12 * sms), std::min(2, R::kCtas), R::kCtas) * sms);
        // a few turns of one CTA take less than a launch to add up several CTAs' sums
        one = ctas > 0 && ctas <= 4;
        if (one) ctas = 1;
      }
      const size_t need = kNetHeader + (size_t)ctas * 2 * (size_t)x->cols * sizeof(float);
      if (need > ctx->net_bytes)
        return fail(ctx, ABCD_ERR_WORKSPACE, "abcd_layer_norm_backward: the network workspace has %zu bytes, needs %zu", ctx->net_bytes, need);
      if (ctas == 0) return ABCD_OK;
      if constexpr (kLong) {
        return check_launch(ctx, "norm_bwd_long_kernel", launch_pdl(norm_bwd_long_kernel<T>, dim3(ctas), dim3(kLongThreads), 0, ctx->stream, a));
      } else {
        auto* kernel = norm_bwd_kernel<T, R>;
        const abcd_status st = room_for(ctx, (const void*)kernel, R::kSmem);
        if (st != ABCD_OK) return st;
        return check_launch(ctx, "norm_bwd_kernel", launch_pdl(kernel, dim3(ctas), dim3(R::kThreads), R::kSmem, ctx->stream, a));
      }
    });
  });
  if (st != ABCD_OK || one || (!dweight && !dbias)) return st;
  // columns in eights until 32 a CTA give half the SMs one (3,000 x 4,096 bf16: both kernels 20.6 us by
  // 32, 23.7 by eight)
  const bool wide = 2 * x->cols >= 16LL * sms;
  const dim3 grid((unsigned)((2 * x->cols + (wide ? 31 : 7)) / (wide ? 32 : 8)));
  return with_type(weight_dtype, [&](auto w) {
    using W = decltype(w);
    return check_launch(ctx, "norm_sum_kernel", launch_pdl(wide ? norm_sum_kernel<W, 32> : norm_sum_kernel<W, 8>, grid, dim3(1024), 0,
                                                           ctx->stream, (const float*)part, ctas, (int)x->cols, (W*)dweight, (W*)dbias));
  });
}
