// What kernels over the rows of matrices share (layernorm.cu, residualnorm.cu): vectors of a row, sums over
// its threads, copies ahead.
#pragma once

#include "network.cuh"

namespace abcd {

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

}  // namespace abcd
