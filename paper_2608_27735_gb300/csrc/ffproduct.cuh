// The matrix products of the gated feed-forward layer (gatedff.cu) and the linear layer (linear.cu), one
// kernel template.
//
// C = sum over segments of A_s B_s^T with 16-bit operands and 32-bit sums, A_s [m][k], B_s [n][k].
// Either operand may lie with k or with its other dimension contiguous.  Segments are how sums of
// several products stay one pass: dx = dG Wg + dU Wu has two, and an operand in 32 bits is three
// 16-bit terms v = t0 + t1 + t2 (each the rounding of what the ones before leave, 24 bits
// together), whose product keeps the six pairs t_i u_j with i + j <= 2: what is left out is below
// 2^-24 of the product.
//
// What bounds it: the tensor cores for wide layers, HBM (the hidden matrices) for narrow ones, the
// weights' bytes for few tokens.  Layout: a persistent grid, one CTA (or pair of CTAs, which share a
// 256 x 256 tile: each stages half of B) per SM; one warp issues the TMA loads of 128-byte swizzled
// tiles into a ring of stages, one the tcgen05 matrix instructions, the others turn the sums that
// lie in tensor memory into results while the next tile's are made in its other half.  Where the
// tiles do not fill the SMs, k is split: each part leaves its 32-bit sums in the workspace, and they
// are added in their order, by a kernel of its own (whose CTAs share the work: dWd of 20,000 x 64 x
// 256 in 32 bits took 64 us with a tile's parts added by its last warps) or, where the sums are
// not yet the result, by the warp that comes last.
//
// 16,384 x 2,048 x 8,192 bf16: y 297 us (1,850 TFLOP/s, the rate of a library's product), gate, up and
// the hidden matrix 639 (1,720), dH with dG, dU and H 461 (1,190: its epilogue's blocks share the
// shared memory's bandwidth with the operands), dx and the weights' gradients 1,510 (1,820).
#pragma once

#include <type_traits>

#include "network.cuh"
#include "tensor_core.cuh"

namespace abcd {

// What becomes of the sums.  kDown8 is kDown with the saved projections in 8 bits, of the large tile alone.
enum { kPlain, kUp, kDown, kLinear, kDown8 };

constexpr int kMaxSegments = 12;
constexpr int kBlockK = 64;           // elements of k per stage: 128 bytes, the swizzle's row

// A result: a matrix of the call (one 32-bit or 16-bit value per element), or an operand of a later
// product (terms planes of 16-bit values).
struct Out {
  void* p;
  long long stride;                   // elements between rows
  long long plane;                    // elements between the terms' planes (operands in 32 bits)
  int vec;                            // rows start on 16-byte boundaries
};

// One of up to three products of a launch (kPlain; the others have one).
struct ProductJob {
  CUtensorMap a, b[2];
  // the operand lies with its own dimension contiguous instead of k: neither (kUp), B (kDown) or, of
  // kPlain, none, B or both
  int a_rows_last, b_rows_last;
  int m, n;                           // rows of A and B (kUp: of each B)
  int kblocks;                        // stages per segment
  int segments;
  unsigned char az[kMaxSegments], bsel[kMaxSegments], bz[kMaxSegments];
  int batch_az;                       // added to az for the second batch
  int tiles_m, tiles_n, batches, splits;
  int first;                          // the job's first item
  Out c[2];                           // the result per batch (kUp, kDown: c[0] the hidden matrix)
  // sums of the splits: kPlain [split][batch][m][part_ld], which a kernel of its own adds up; otherwise
  // per warp of a tile, which the last warp to come adds up
  float* part;
  long long part_ld;
};
constexpr int kMaxJobs = 3;

struct ProductArgs {
  ProductJob job[kMaxJobs];
  int jobs, items;
  // the large tile of 16-bit matrices: kUp and kLinear store c and, where their rows allow it, gate and up, or z
  // (g); kLinear loads the residual (in);
  // kDown loads gate, up (in) and stores
  // c, dG and dU (planes 0 and 1 of g[0])
  CUtensorMap c_map, g_map[2], in_map[2];
  int dtype;
  int act;
  Out g[2];                           // kUp: gate and up (p NULL: not wanted); kDown: dG and dU
  // kDown8: the powers of gate's and up's groups of 32 columns
  const unsigned char* power[2];
  long long power_stride[2];
  Out in[2];                          // kDown: the saved gate and up; kLinear: the residual (p NULL: none)
  const void* bias;                   // kLinear, or NULL; z goes to g[0]
  int wide_bias;                      // it is fp32 whatever the matrices' type
  unsigned* count;                    // finished splits per warp of a tile; zero between calls
  unsigned* status;
  unsigned limit;                     // polls of a wait
};

// The activations and their slopes.  The device's approximations of 2^x and 1/x, each within a few
// units of 2^-23, are enough for sums whose terms were rounded to as much.
__device__ __forceinline__ float exp2_of(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float inverse_of(float x) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float sigmoid_of(float z) { return inverse_of(1.f + exp2_of(-1.44269504f * z)); }
// The normal distribution's Phi(z) and e = exp(-z^2 / 2).  Far below zero Phi is as small as e, and an
// error that is small beside one is large beside it, so the tail is taken relative to itself: of 32-bit
// matrices by the device's erfc (z^2 / 2 units of z's rounding, and a few of its own), of 16-bit ones as e
// times a polynomial in t = 1 / (1 + 0.3 |z|), whose coefficients were fitted here to
// exp(z^2 / 2) Phi(-|z|) by weighted minimax: in 32 bits Phi within 4.2e-7, and within 1.8e-5 of itself down
// to z = -13, below half a unit of the 16-bit types.
//
// QUICK (the linear layer, whatever the number of its tokens, and its slope): of 32-bit matrices too as e times a
// polynomial, in t = 1 / (1 + 0.25 |z|) and fitted the same way to 1.8e-8 of the tail, 3.5 units of 2^-23 with its
// arithmetic in 32 bits.  e adds to that what its argument loses in two roundings, about 0.7 z^2 units of 2^-24: the
// tail is off by some 4 of its units of 2^-23 at z = -2, 12 at -5 and 60 at -12.  erfc takes several times the
// instructions, and there the epilogue is most of the time (20,000 x 59 x 256 fp32: the product 28 us with
// erfc).
template <bool F32, bool QUICK = false> __device__ __forceinline__ float phi_of(float z, float& e) {
  e = exp2_of(-0.72134752f * z * z);
  if constexpr (F32 && QUICK) {
    const float t = inverse_of(1.f + 0.25f * fabsf(z));
    float p = 0.02050131931900978f;
    p = p * t - 0.08396998792886734f;
    p = p * t + 0.10110922157764435f;
    p = p * t - 0.03697000816464424f;
    p = p * t + 0.06656643003225327f;
    p = p * t + 0.05809324234724045f;
    p = p * t + 0.08173637837171555f;
    p = p * t + 0.0934624895453453f;
    p = p * t + 0.09973527491092682f;
    p = p * t + 0.09973565489053726f;
    const float tail = e * (p * t);
    return z < 0.f ? tail : 1.f - tail;
  } else if constexpr (F32) {
    return 0.5f * erfcf(-0.70710678f * z);
  } else {
    const float t = inverse_of(1.f + 0.3f * fabsf(z));
    const float tail = e * t * (0.120121039f + t * (0.113127187f + t * (0.147127926f + t * (-0.0232996624f + t * (0.222333118f + t * -0.0794098675f)))));
    return z < 0.f ? tail : 1.f - tail;
  }
}
__device__ __forceinline__ float relu_of(float z) { return z > 0.f ? z : (z == z ? 0.f : z); }

template <bool F32, int N, bool QUICK = false> __device__ __forceinline__ void act_values(float (&z)[N], int act) {
  if (act == ABCD_SILU) {
#pragma unroll
    for (int i = 0; i < N; ++i) z[i] *= sigmoid_of(z[i]);
  } else if (act == ABCD_GELU) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float e;
      z[i] *= phi_of<F32, QUICK>(z[i], e);
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) z[i] = relu_of(z[i]);
  }
}
// z becomes act(z), s its slope.
template <bool F32, int N, bool QUICK = false> __device__ __forceinline__ void act_slopes(float (&z)[N], float (&s)[N], int act) {
  if (act == ABCD_SILU) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float g = sigmoid_of(z[i]), v = z[i] * g;
      s[i] = g + v * (1.f - g);
      z[i] = v;
    }
  } else if (act == ABCD_GELU) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float e;
      const float c = phi_of<F32, QUICK>(z[i], e);
      s[i] = c + z[i] * 0.39894228f * e;
      z[i] *= c;
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      s[i] = z[i] > 0.f ? 1.f : 0.f;
      z[i] = relu_of(z[i]);
    }
  }
}

__device__ __forceinline__ unsigned pack2(float a, float b, bool bf16) {
  if (bf16) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const unsigned*>(&v);
  }
  const __half2 v = __floats2half2_rn(a, b);
  return *reinterpret_cast<const unsigned*>(&v);
}
__device__ __forceinline__ float unpack(unsigned short v, bool bf16) {
  return bf16 ? __uint_as_float((unsigned)v << 16) : __half2float(__ushort_as_half(v));
}
// The next 16-bit terms of two 32-bit values as a pair, and the values with what they leave.  (Of an
// infinity NaN is left, and NaN is what a product with it gives: with the exact rest, none, it would
// be so too, wherever a lower term of the other factor is zero.)
__device__ __forceinline__ unsigned take_terms(float& a, float& b) {
  const unsigned w = pack2(a, b, true);
  a -= __uint_as_float(w << 16);
  b -= __uint_as_float(w & 0xffff0000u);
  return w;
}

// Pairs of v as 16-bit values.
template <int CW>
__device__ __forceinline__ void pack_all(const float (&v)[CW], unsigned (&w)[CW / 2], bool bf16) {
  if (bf16) {
#pragma unroll
    for (int i = 0; i < CW / 2; ++i) w[i] = pack2(v[2 * i], v[2 * i + 1], true);
  } else {
#pragma unroll
    for (int i = 0; i < CW / 2; ++i) w[i] = pack2(v[2 * i], v[2 * i + 1], false);
  }
}

// A warp's 32 rows in a buffer, as rows of PIECES 16-byte pieces swapped by row so that neither a lane
// per row nor lanes along the rows meet bank conflicts.
template <int PIECES> __device__ __forceinline__ int turned(int row, int j) {
  constexpr int SPREAD = 8 / PIECES > 0 ? 8 / PIECES : 1;   // rows within 128 bytes of the buffer
  return row * PIECES * 16 + ((j ^ ((row / SPREAD) % PIECES)) * 16);
}
// Such rows to a matrix whose rows start anywhere, or the part of them that is inside it: consecutive
// lanes write consecutive elements.
template <int PIECES, typename E>
static __device__ __noinline__ void store_elements(const char* buf, char* base, long long stride_bytes, int rows, int cols) {
  constexpr int WIDTH = PIECES * 16 / (int)sizeof(E);       // elements of a row
  constexpr int ROWS = WIDTH < 32 ? 32 / WIDTH : 1;         // rows that the lanes take at a time
  const int lane = threadIdx.x & 31, at = lane % WIDTH * (int)sizeof(E);
  if (at >= cols * (int)sizeof(E)) return;
  base += at;
  for (int row0 = lane / WIDTH; row0 < rows; row0 += 8 * ROWS) {
    E v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = *reinterpret_cast<const E*>(buf + turned<PIECES>((row0 + i * ROWS) & 31, at / 16) + at % 16);
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (row0 + i * ROWS < rows) *reinterpret_cast<E*>(base + (row0 + i * ROWS) * stride_bytes) = v[i];
  }
}

// A warp's 32 rows x CW columns of elements E, lane l holding row l as words: turned round in the
// warp's buffer, so that consecutive lanes write consecutive 16 bytes of a row.
template <typename E, int WORDS>
__device__ __forceinline__ void store_words(const unsigned (&w)[WORDS], char* buf, void* base,
                                            long long stride_bytes, int rows, int cols, bool vec) {
  constexpr int PIECES = WORDS / 4;                 // 16-byte pieces of a row
  constexpr int ROWS = 32 / PIECES;                 // rows that the lanes take at a time
  const int lane = threadIdx.x & 31;
  __syncwarp();
#pragma unroll
  for (int j = 0; j < PIECES; ++j)
    *reinterpret_cast<uint4*>(buf + turned<PIECES>(lane, j)) = make_uint4(w[4 * j], w[4 * j + 1], w[4 * j + 2], w[4 * j + 3]);
  __syncwarp();
  if (vec && rows >= 32 && cols * (int)sizeof(E) >= PIECES * 16) {
    const int row0 = lane / PIECES, j = lane % PIECES;
    char* at = (char*)base + row0 * stride_bytes + 16 * j;
#pragma unroll
    for (int i = 0; i < PIECES; ++i, at += ROWS * stride_bytes)
      *reinterpret_cast<uint4*>(at) = *reinterpret_cast<const uint4*>(buf + turned<PIECES>(i * ROWS + row0, j));
  } else {
    store_elements<PIECES, E>(buf, (char*)base, stride_bytes, rows, cols);
  }
}

// v as values of the call's type, to rows m... of matrix o from column n on.
template <bool F32, int CW>
__device__ __forceinline__ void store_matrix(const float (&v)[CW], const Out& o, long long m, int n,
                                             int rows, int cols, bool bf16, char* buf) {
  if constexpr (F32) {
    unsigned w[CW];
#pragma unroll
    for (int i = 0; i < CW; ++i) w[i] = __float_as_uint(v[i]);
    store_words<unsigned, CW>(w, buf, (float*)o.p + m * o.stride + n, o.stride * 4, rows, cols, o.vec);
  } else {
    unsigned w[CW / 2];
    pack_all(v, w, bf16);
    store_words<unsigned short, CW / 2>(w, buf, (unsigned short*)o.p + m * o.stride + n, o.stride * 2, rows, cols, o.vec);
  }
}

// v as an operand of a later product: of the 16-bit types the values, of 32 bits three terms.
template <bool F32, int CW>
__device__ __forceinline__ void store_operand(const float (&v)[CW], const Out& o, long long m, int n,
                                              int rows, int cols, bool bf16, char* buf) {
  if constexpr (!F32) {
    store_matrix<false, CW>(v, o, m, n, rows, cols, bf16, buf);
  } else {
    float rest[CW];
#pragma unroll
    for (int i = 0; i < CW; ++i) rest[i] = v[i];
#pragma unroll 1
    for (int t = 0; t < 3; ++t) {
      unsigned w[CW / 2];
#pragma unroll
      for (int i = 0; i < CW / 2; ++i) w[i] = take_terms(rest[2 * i], rest[2 * i + 1]);
      store_words<unsigned short, CW / 2>(w, buf, (unsigned short*)o.p + t * o.plane + m * o.stride + n, o.stride * 2,
                                          rows, cols, o.vec);
    }
  }
}

// Asynchronous copy of `bytes` (16 at most) to 16 bytes of shared memory, zeros after them.
__device__ __forceinline__ void copy_piece(uint32_t dst, const void* src, int bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes < 0 ? 0 : bytes < 16 ? bytes : 16) : "memory");
}
// A warp's buffer of 32 rows of sixteen values: 16-byte pieces, swapped by row so that lanes which
// read the same piece of their rows meet no bank conflicts.
template <bool F32> struct RowBuffer {
  static constexpr int kPieces = F32 ? 4 : 2;
  static constexpr int kBytes = 32 * kPieces * 16;
  __device__ static __forceinline__ int at(int row, int j) {
    return (row * kPieces + (j ^ (row * kPieces / 8 % kPieces))) * 16;
  }
};
// Rows m ... m + rows of sixteen columns from column n on, on their way to such a buffer: by 16 bytes
// (16-bit matrices always lie so), or 32-bit values whose rows start anywhere one by one.
template <bool F32>
__device__ __forceinline__ void rows_ahead(char* buf, const Out& o, long long m, int n, int rows, int cols) {
  using B = RowBuffer<F32>;
  constexpr int SIZE = F32 ? 4 : 2;
  const int lane = threadIdx.x & 31;
  if (!F32 || o.vec) {
    const int j = lane % B::kPieces;
#pragma unroll
    for (int i = 0; i < B::kPieces; ++i) {
      const int row = i * (32 / B::kPieces) + lane / B::kPieces, bytes = row < rows ? SIZE * cols - 16 * j : 0;
      const char* src = (const char*)o.p + ((m + row) * o.stride + n) * SIZE + 16 * j;
      copy_piece(smem_addr(buf + B::at(row, j)), bytes > 0 ? src : (const char*)o.p, bytes);
    }
  } else {
    const int e = lane % 16;
    for (int row = lane / 16; row < rows; row += 2)
      if (e < cols)
        asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(smem_addr(buf + B::at(row, e / 4) + e % 4 * 4)),
                     "l"((const float*)o.p + (m + row) * o.stride + n + e) : "memory");
  }
}
// Eight 16-bit values of 16 bytes.
__device__ __forceinline__ void unpack8(float* v, const uint4& x, bool bf16) {
  const unsigned w[4] = {x.x, x.y, x.z, x.w};
  if (bf16) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = unpack((unsigned short)(w[e / 2] >> (16 * (e & 1))), true);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = unpack((unsigned short)(w[e / 2] >> (16 * (e & 1))), false);
  }
}
// The lane's row of such a buffer.
template <bool F32>
__device__ __forceinline__ void row_of(float (&v)[16], const char* buf, bool bf16) {
  using B = RowBuffer<F32>;
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int q = 0; q < B::kPieces; ++q) {
    const uint4 x = *reinterpret_cast<const uint4*>(buf + B::at(lane, q));
    if constexpr (F32) {
      v[4 * q] = __uint_as_float(x.x); v[4 * q + 1] = __uint_as_float(x.y);
      v[4 * q + 2] = __uint_as_float(x.z); v[4 * q + 3] = __uint_as_float(x.w);
    } else {
      unpack8(v + 8 * q, x, bf16);
    }
  }
}

// kLinear: the lane's row of sixteen columns of the residual, from column n of row m + lane on; zeros
// outside of it.
template <bool F32, int CW>
__device__ __forceinline__ void residual_ahead(float (&v)[CW], const Out& o, long long m, int n, int rows, int cols, bool bf16) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int q = 0; q < CW; ++q) v[q] = 0.f;
  if (!o.p || lane >= rows) return;
  const long long at = (m + lane) * o.stride + n;
  if constexpr (F32) {
    const float* p = (const float*)o.p + at;
    if (o.vec && cols >= CW) {
#pragma unroll
      for (int q = 0; q < CW; q += 4) {
        const float4 x = *reinterpret_cast<const float4*>(p + q);
        v[q] = x.x; v[q + 1] = x.y; v[q + 2] = x.z; v[q + 3] = x.w;
      }
    } else {
#pragma unroll
      for (int q = 0; q < CW; ++q)
        if (q < cols) v[q] = p[q];
    }
  } else {
    const unsigned short* p = (const unsigned short*)o.p + at;
    if (o.vec && cols >= CW) {
#pragma unroll
      for (int q = 0; q < CW; q += 8) unpack8(v + q, *reinterpret_cast<const uint4*>(p + q), bf16);
    } else {
#pragma unroll
      for (int q = 0; q < CW; ++q)
        if (q < cols) v[q] = unpack(p[q], bf16);
    }
  }
}

// The same for rows that start anywhere, through the warp's buffer: consecutive lanes read consecutive elements.
// (Each lane by itself, 20,000 x 512 x 1,001 bf16 took 199 us, so 98.)
template <bool F32, int CW>
static __device__ __noinline__ void fill_rows(char* buf, const Out& o, long long m, int n, int rows, int cols) {
  using E = std::conditional_t<F32, unsigned, unsigned short>;
  constexpr int PIECES = CW * (int)sizeof(E) / 16, ROWS = CW < 32 ? 32 / CW : 1, BATCH = 8;
  const int lane = threadIdx.x & 31, e = lane % CW;
  const E* from = (const E*)o.p + m * o.stride + n + e;
#pragma unroll 1
  for (int row0 = lane / CW; row0 < 32; row0 += BATCH * ROWS) {
    E x[BATCH];
#pragma unroll
    for (int i = 0; i < BATCH; ++i) x[i] = row0 + i * ROWS < rows && e < cols ? from[(row0 + i * ROWS) * o.stride] : E(0);
#pragma unroll
    for (int i = 0; i < BATCH; ++i)
      if (row0 + i * ROWS < 32) *reinterpret_cast<E*>(buf + turned<PIECES>(row0 + i * ROWS, e * (int)sizeof(E) / 16) + e * (int)sizeof(E) % 16) = x[i];
  }
}
template <bool F32, int CW>
__device__ __forceinline__ void residual_elements(float (&v)[CW], char* buf, const Out& o, long long m, int n, int rows, int cols, bool bf16) {
  constexpr int PIECES = CW * (F32 ? 4 : 2) / 16;
  const int lane = threadIdx.x & 31;
  // the turn before reads its results from the buffer.  (Within fill_rows this costs the kernel registers: 20,000 x 512
  // x 1,001 bf16 121 us instead of 98, 20,000 x 59 x 256 fp32, which has no residual, 28.7 instead of 26.6.)
  __syncwarp();
  fill_rows<F32, CW>(buf, o, m, n, rows, cols);
  __syncwarp();
#pragma unroll
  for (int j = 0; j < PIECES; ++j) {
    const uint4 x = *reinterpret_cast<const uint4*>(buf + turned<PIECES>(lane, j));
    if constexpr (F32) {
      v[4 * j] = __uint_as_float(x.x); v[4 * j + 1] = __uint_as_float(x.y);
      v[4 * j + 2] = __uint_as_float(x.z); v[4 * j + 3] = __uint_as_float(x.w);
    } else {
      unpack8(v + 8 * j, x, bf16);
    }
  }
  __syncwarp();
}

// Where 16-byte piece j of a row lies in a block of 128 rows of 64 bytes under TMA's 64-byte swizzle.
__device__ __forceinline__ int block_at(int row, int j) { return row * 64 + ((j ^ ((row / 2) % 4)) * 16); }
// Sixteen columns, from piece j on, of a block's rows first ... first + 31 to a matrix whose rows start
// anywhere: consecutive lanes write consecutive elements.
static __device__ __noinline__ void block_elements(const char* block, int first, int j, const Out& o, long long m, int n, int rows, int cols) {
  const int lane = threadIdx.x & 31, e = lane % 16;
  if (e >= cols) return;
  unsigned short* to = (unsigned short*)o.p + m * o.stride + n + e;
  for (int row0 = lane / 16; row0 < rows; row0 += 16) {
    unsigned short v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i)
      v[i] = *reinterpret_cast<const unsigned short*>(block + block_at(first + ((row0 + 2 * i) & 31), j + e / 8) + e % 8 * 2);
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (row0 + 2 * i < rows) to[(row0 + 2 * i) * o.stride] = v[i];
  }
}
// What TMA leaves of such columns: those from column `whole` of the matrix on, behind a row's last whole piece.
static __device__ __noinline__ void block_tail(const char* block, int first, int j, const Out& o, long long m, int n, int rows, int cols, int whole) {
  const int skip = whole - n;
  if (skip >= 0 && skip < 16 && skip < cols) block_elements(block, first, j + skip / 8, o, m, whole, rows, cols - skip);
}
__device__ __forceinline__ void put_block(char* block, int row, int j, const unsigned (&w)[8]) {
  *reinterpret_cast<uint4*>(block + block_at(row, j)) = make_uint4(w[0], w[1], w[2], w[3]);
  *reinterpret_cast<uint4*>(block + block_at(row, j + 1)) = make_uint4(w[4], w[5], w[6], w[7]);
}

// kLinear: sixteen columns of the bias, in every lane (one address for the warp).
__device__ __forceinline__ void bias_columns(float (&v)[16], const void* bias, int wide, int n, int cols, bool bf16) {
  const char* p = (const char*)bias + (long long)n * (wide ? 4 : 2);
  if (cols >= 16 && ((uintptr_t)p & 15) == 0) {
    if (wide) {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const float4 x = __ldg(reinterpret_cast<const float4*>(p) + q);
        v[4 * q] = x.x; v[4 * q + 1] = x.y; v[4 * q + 2] = x.z; v[4 * q + 3] = x.w;
      }
    } else {
#pragma unroll
      for (int q = 0; q < 2; ++q) unpack8(v + 8 * q, __ldg(reinterpret_cast<const uint4*>(p) + q), bf16);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 16; ++e) v[e] = e >= cols ? 0.f : wide ? __ldg((const float*)p + e) : unpack(__ldg((const unsigned short*)p + e), bf16);
  }
}

// kDown8: the powers of eight groups of 32 columns of a row, from group g on (a multiple of eight); 0, which
// makes values nothing, outside of the matrix.
__device__ __forceinline__ uint2 row_powers(const unsigned char* p, long long stride, int row, int rows, int g, int groups) {
  uint2 v = make_uint2(0u, 0u);
  if (row >= rows) return v;
  p += row * stride + g;
  if (((uintptr_t)p & 7) == 0 && g + 8 <= groups) return __ldg(reinterpret_cast<const uint2*>(p));
#pragma unroll
  for (int k = 0; k < 8; ++k)
    if (g + k < groups) (k < 4 ? v.x : v.y) |= (unsigned)__ldg(p + k) << (8 * (k & 3));
  return v;
}
// 2^(p - 127) of group s.
__device__ __forceinline__ float scale_at(const uint2& power, int s) {
  return __uint_as_float(((s < 4 ? power.x : power.y) >> (8 * (s & 3)) & 255u) << 23);
}
// Sixteen codes' values.
__device__ __forceinline__ void decode16(float (&v)[16], const uint4& x, float scale) {
  const unsigned w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
  for (int e = 0; e < 16; ++e) v[e] = code_value(w[e / 4] ^ 0x80808080u, e & 3) * scale;
}

// A work item of the persistent loop.
struct Item {
  int job, batch, split, tm, tn;
  int tile;                           // number of (batch, tm, tn)
  int k0, k1;                         // stages [k0, k1) of every segment
};

// Items in order: the jobs one after another, the splits of a tile next to each other (they finish
// together), tiles in bands of eight along m, so that the CTAs that run at once share operands in L2.
__device__ __forceinline__ Item item_of(const ProductArgs& a, int i) {
  constexpr int BAND = 8;
  Item it;
  it.job = (a.jobs > 1 && i >= a.job[1].first) + (a.jobs > 2 && i >= a.job[2].first);
  const ProductJob& q = a.job[it.job];
  i -= q.first;
  it.split = i % q.splits;
  int t = i / q.splits;
  it.tile = t;
  const int per_batch = q.tiles_m * q.tiles_n;
  it.batch = t / per_batch;
  t -= it.batch * per_batch;
  const int band = t / (BAND * q.tiles_n);
  t -= band * BAND * q.tiles_n;
  const int height = min(BAND, q.tiles_m - band * BAND);
  it.tn = t / height;
  it.tm = band * BAND + t % height;
  it.k0 = (int)((long long)q.kblocks * it.split / q.splits);
  it.k1 = (int)((long long)q.kblocks * (it.split + 1) / q.splits);
  return it;
}

// CG: CTAs that share a tile (1 or 2) of 128 CG rows and BN sums per row; EPI: what becomes of the
// sums; F32: whether the call's matrices are in 32 bits.
template <int CG, int BN, int EPI, bool F32>
struct Product {
  static constexpr int kRows = 128;                      // rows of A per CTA
  static constexpr int kBRows = BN / CG;                 // rows of B per CTA
  static constexpr int kABytes = kRows * 128, kBBytes = kBRows * 128;
  static constexpr int kStageBytes = kABytes + kBBytes;
  static constexpr int kTmemCols = 2 * BN;
  static constexpr int kOutCols = EPI == kUp ? BN / 2 : BN;   // results per row of a tile
  // Epilogue warps: each takes 32 rows (a quarter of tensor memory's lanes) and a share of the
  // columns.  Sixteen for the large tile of 16-bit matrices, whose products of few stages wait for
  // them.
  static constexpr int kWarps = BN == 256 && !F32 ? 16 : 8;
  // There the results (and the saved projections) also go through shared memory by TMA, in blocks of
  // 128 rows x 32 columns that two groups of eight warps take in turn; kDown has a warp more, which
  // asks for the blocks of the saved projections up to three ahead.  With accesses of the warps' own
  // instead (32 bytes of a row at a time), 100,000 x 256 x 1,024 took 167 and 196 us for kUp and kDown;
  // with the blocks 119 and 171.  (kLinear, 16,384 x 4,096 x 4,096 with residual and z: 630 and 332.)
  static constexpr bool kBlocks = BN == 256 && !F32 && EPI != kPlain;
  static constexpr int kBlockBytes = 128 * 64;
  // Blocks of results per group (three, of kLinear two), and for kDown slots of a block of gate and one of up,
  // for kLinear of one of the residual.
  // (A slot's blocks go to the groups in turn.  So it has two barriers that say it is full, one for each
  // group: a wait for a phase is right only for who has seen the phase before it end.)
  static constexpr int kSlots = 3;
  static constexpr bool kIsDown = EPI == kDown || EPI == kDown8;
  static constexpr int kResults = EPI == kLinear ? 2 : 3, kAsked = kIsDown ? 2 : EPI == kLinear ? 1 : 0;
  static constexpr int kBlockRoom = (2 * kResults + kAsked * kSlots) * kBlockBytes;
  static constexpr int kThreads = 64 + 32 * kWarps + (kBlocks && kAsked ? 32 : 0);
  static constexpr int kWarpCols = kOutCols / (kWarps / 4);
  static constexpr int CW = EPI == kUp || EPI == kDown || EPI == kDown8 || kWarpCols < 32 ? 16 : 32;    // taken at a time
  // Elsewhere a warp turns its rows round in a buffer of its own.  The smallest tile leaves room for a
  // second CTA on the SM, whose warps fill the waits of the first's; kDown takes that room for the
  // saved projections, which come two turns ahead (20,000 x 64 x 256 in 32 bits: 45 us, and 58 with
  // two CTAs instead).
  static constexpr int kCtas = BN == 64 && EPI != kDown ? 2 : 1;
  static constexpr bool kAhead = EPI == kDown;
  static constexpr int kTurn = 32 * CW * (F32 ? 4 : 2);
  static constexpr int kBuffer = kTurn + (kAhead ? 4 * RowBuffer<F32>::kBytes : 0);
  static constexpr int kEpilogueBytes = kBlocks ? kBlockRoom : kWarps * kBuffer;
  static constexpr int kRoom = ((kCtas == 2 ? 113 : 227) * 1024 - 512 - 1024 - kEpilogueBytes) / kStageBytes;
  static constexpr int kStages = kRoom > 8 ? 8 : kRoom;
  static_assert(kTurn >= (EPI == kPlain ? 32 * 16 * 4 : 0) && kStages >= 3);
  static_assert(kWarpCols % CW == 0 || EPI == kPlain);
  static constexpr size_t kSmem = 1024 + (size_t)kStages * kStageBytes + kEpilogueBytes;
};

// ODD, of the large tile of 16-bit matrices: the rows of the caller's results end inside a piece of 16 bytes.  (A kernel
// of its own: the test for it in the loop cost kUp 2 to 14 us of the 172 of 100,000 x 256 x 1,024.)
template <int CG, int BN, int EPI, bool F32, bool ODD>
__global__ void __launch_bounds__(Product<CG, BN, EPI, F32>::kThreads, Product<CG, BN, EPI, F32>::kCtas) product_kernel(const __grid_constant__ ProductArgs a) {
  using P = Product<CG, BN, EPI, F32>;
  extern __shared__ char smem_raw[];
  __shared__ uint64_t bars[2 * P::kStages + 4 + 3 * P::kSlots];
  __shared__ uint32_t tmem_base;
  __shared__ volatile int dead;
  const int warp = threadIdx.x / 32, lane = threadIdx.x & 31;
  const uint32_t rank = CG == 2 ? cluster_rank() : 0;
  const uint32_t ring = (smem_addr(smem_raw) + 1023u) & ~1023u;
  char* buffers = smem_raw + (ring - smem_addr(smem_raw)) + P::kStages * P::kStageBytes;
  const uint32_t full = smem_addr(bars), empty = full + 8 * P::kStages;
  const uint32_t sums_full = empty + 8 * P::kStages, sums_empty = sums_full + 16;
  const uint32_t slot_full = sums_empty + 16, slot_empty = slot_full + 16 * P::kSlots;
  if (threadIdx.x == 0) {
    dead = 0;
    for (int s = 0; s < P::kStages; ++s) {
      mbar_init(full + 8 * s, 1);
      mbar_init(empty + 8 * s, 1);
    }
    for (int s = 0; s < 2; ++s) {
      mbar_init(sums_full + 8 * s, 1);
      mbar_init(sums_empty + 8 * s, P::kWarps * CG);
    }
    for (int s = 0; s < P::kSlots; ++s) {
      mbar_init(slot_full + 16 * s, 1);
      mbar_init(slot_full + 16 * s + 8, 1);
      mbar_init(slot_empty + 8 * s, 8);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    prefetch_map(&a.job[0].a);
    prefetch_map(&a.job[0].b[0]);
    prefetch_map(&a.job[0].b[1]);
  }
  if (warp == 1) tmem_alloc<CG>(smem_addr(&tmem_base), P::kTmemCols);
  tc_fence_before();
  __syncthreads();
  if (CG == 2) cluster_sync();
  tc_fence_after();
  pdl_wait();
  const uint32_t tmem = tmem_base;
  const int first = blockIdx.x / CG, step = gridDim.x / CG;
  const int items = a.items;

  if (warp == 0) {
    if (lane == 0) {
      const uint32_t full0 = CG == 2 ? at_rank(full, 0) : full;   // the barriers of the pair's first CTA
      int stage = 0;
      uint32_t phase = 0;
      bool ok = true;
      for (int i = first; ok && i < items; i += step) {
        const Item it = item_of(a, i);
        // the job by a constant, so that its tensor maps have constant addresses (with addresses of run
        // time, the loads kept the matrix instructions waiting: 16,384 x 2,048 x 8,192 in 16 bits, y in
        // 355 us instead of 295)
        auto feed = [&](auto number) {
          const ProductJob& job = a.job[decltype(number)::value];
          const bool a_last = job.a_rows_last, b_last = job.b_rows_last;
          const int row_a = (it.tm * CG + (int)rank) * P::kRows;
          const int row_b = EPI == kUp ? it.tn * P::kOutCols : it.tn * BN + (int)rank * P::kBRows;
          for (int seg = 0, kb = it.k0; seg < job.segments; kb + 1 < it.k1 ? ++kb : (++seg, kb = it.k0)) {
            if (!(ok = mbar_wait(empty + 8 * stage, phase ^ 1, a.limit, &dead))) break;
            const uint32_t bar = full0 + 8 * stage;
            if (rank == 0) mbar_expect(full + 8 * stage, P::kStageBytes * CG);
            const int k = kb * kBlockK;
            const uint32_t sa = ring + stage * P::kStageBytes, sb = sa + P::kABytes;
            const int az = job.az[seg] + it.batch * job.batch_az, bz = job.bz[seg];
            if (EPI == kPlain && a_last) {
#pragma unroll
              for (int c = 0; c < P::kRows / 64; ++c) tma_load<CG>(sa + c * 8192, &job.a, row_a + c * 64, k, az, bar);
            } else {
              tma_load<CG>(sa, &job.a, k, row_a, az, bar);
            }
            if (EPI == kUp) {
              // gate and up rows of the same hidden columns: sums [0, BN/2) and [BN/2, BN)
              if (CG == 2) {
                tma_load<CG>(sb, &job.b[rank], k, row_b, bz, bar);
              } else {
                tma_load<CG>(sb, &job.b[0], k, row_b, bz, bar);
                tma_load<CG>(sb + P::kBBytes / 2, &job.b[1], k, row_b, bz, bar);
              }
            } else {
              const CUtensorMap* b = P::kIsDown ? &job.b[0] : &job.b[job.bsel[seg]];
              if (P::kIsDown || b_last) {
#pragma unroll
                for (int c = 0; c < P::kBRows / 64; ++c) tma_load<CG>(sb + c * 8192, b, row_b + c * 64, k, bz, bar);
              } else {
                tma_load<CG>(sb, b, k, row_b, bz, bar);
              }
            }
            if (++stage == P::kStages) {
              stage = 0;
              phase ^= 1;
            }
          }
        };
        if (EPI != kPlain || it.job == 0) feed(std::integral_constant<int, 0>());
        else if (it.job == 1) feed(std::integral_constant<int, 1>());
        else feed(std::integral_constant<int, 2>());
      }
    }
  } else if (warp == 1) {
    if (lane == 0 && rank == 0) {
      const uint32_t type = a.dtype == ABCD_F16 ? 0u : 1u;
      const uint32_t form = (1u << 4) | (type << 7) | (type << 10) | ((uint32_t)(BN / 8) << 17) | ((uint32_t)(128 * CG / 16) << 24);
      int stage = 0;
      uint32_t phase = 0;
      int buf = 0;
      uint32_t sums_phase = 0;
      bool ok = true;
      for (int i = first; ok && i < items; i += step) {
        const Item it = item_of(a, i);
        if (!(ok = mbar_wait(sums_empty + 8 * buf, sums_phase ^ 1, a.limit, &dead))) break;
        tc_fence_after();
        const ProductJob& job = a.job[it.job];
        const int stages = job.segments * (it.k1 - it.k0);
        // the operands' forms, and with them the descriptors' steps, are constants of the loop
        auto multiply = [&](auto a_last, auto b_last) {
          constexpr uint32_t A_STEP = decltype(a_last)::value ? 2048 : 32, B_STEP = decltype(b_last)::value ? 2048 : 32;   // bytes of 16 k
          const uint32_t idesc = form | ((uint32_t)decltype(a_last)::value << 15) | ((uint32_t)decltype(b_last)::value << 16);
          for (int kb = 0; kb < stages; ++kb) {
            if (!(ok = mbar_wait(full + 8 * stage, phase, a.limit, &dead))) break;
            tc_fence_after();
            const uint32_t sa = ring + stage * P::kStageBytes, sb = sa + P::kABytes;
#pragma unroll
            for (int q = 0; q < kBlockK / 16; ++q)
              mma16<CG>(tmem + buf * BN, tile_descriptor(sa + q * A_STEP, 8192), tile_descriptor(sb + q * B_STEP, 8192), idesc,
                        kb > 0 || q > 0);
            mma_commit<CG>(empty + 8 * stage);
            if (++stage == P::kStages) {
              stage = 0;
              phase ^= 1;
            }
          }
        };
        if constexpr (EPI == kUp || EPI == kLinear) {
          multiply(std::false_type(), std::false_type());
        } else if constexpr (P::kIsDown) {
          multiply(std::false_type(), std::true_type());
        } else {
          if (job.a_rows_last) multiply(std::true_type(), std::true_type());
          else if (job.b_rows_last) multiply(std::false_type(), std::true_type());
          else multiply(std::false_type(), std::false_type());
        }
        if (ok) mma_commit<CG>(sums_full + 8 * buf);
        buf ^= 1;
        if (buf == 0) sums_phase ^= 1;
      }
    }
  } else if constexpr (P::kBlocks) {
    // Blocks of 32 result columns: the two groups take them in turn.  A wait that gave up skips the
    // later waits and stores, not the groups' barriers; it gives up for the whole warp, whose lanes
    // meet again below.  Nor does it say that a slot or sums are free: the slots' loader would expect a
    // slot's next block while the last one is still in flight, an arrival too many for its barrier.
    constexpr int BLOCKS = P::kOutCols / 32;
    const int row0 = (int)rank * P::kRows;
    bool ok = true;
    if (warp == 2 + P::kWarps) {
      if (lane == 0 && (EPI != kLinear || (a.in[0].p && a.in[0].vec))) {
        unsigned q = 0;
        for (int i = first; ok && i < items; i += step) {
          const Item it = item_of(a, i);
          const int m = it.tm * CG * P::kRows + row0;
          if (m >= a.job[0].m) continue;
          for (int s = 0; s < BLOCKS; ++s) {
            const int n = it.tn * P::kOutCols + 32 * s;
            if (n >= a.job[0].n) break;
            const int slot = q % P::kSlots;
            if (!(ok = mbar_wait(slot_empty + 8 * slot, (q / P::kSlots & 1) ^ 1, a.limit, &dead))) break;
            const uint32_t bar = slot_full + 8 * (q % (2 * P::kSlots)), at = smem_addr(buffers) + (2 * P::kResults + P::kAsked * slot) * P::kBlockBytes;
            mbar_expect(bar, P::kAsked * (EPI == kDown8 ? 128 * 32 : P::kBlockBytes));
            tma_load<1>(at, &a.in_map[0], n, m, 0, bar);
            if (P::kIsDown) tma_load<1>(at + P::kBlockBytes, &a.in_map[1], n, m, 0, bar);
            ++q;
          }
        }
      }
    } else {
      const int quarter = warp & 3, share = (warp - 2) / 4, group = share / 2, half = share & 1;
      const int row = quarter * 32 + lane;
      const bool bf16 = a.dtype == ABCD_BF16;
      // kUp's gate and up, kLinear's z
      const bool saved = (EPI == kUp || EPI == kLinear) && a.g[0].p;
      const bool saved_by_tma = saved && a.g[0].vec && (EPI == kLinear || a.g[1].vec);
      const bool result_by_tma = EPI != kLinear || a.job[0].c[0].vec;
      const bool elected = (warp - 2) % 8 == 0 && lane == 0;   // of the group
      const uint32_t empty0 = at_rank(sums_empty, 0);
      char* own = buffers + group * P::kResults * P::kBlockBytes;
      int buf = 0;
      uint32_t phase = 0;
      unsigned q = 0;                                          // blocks of the CTA so far
      for (int i = first; i < items; i += step) {
        const Item it = item_of(a, i);
        const int m = it.tm * CG * P::kRows + row0, n0 = it.tn * P::kOutCols;
        uint2 power[2];                                        // kDown8: of the row's eight groups of 32 columns
        if constexpr (EPI == kDown8) {
#pragma unroll
          for (int k = 0; k < 2; ++k) power[k] = row_powers(a.power[k], a.power_stride[k], m + row, a.job[0].m, n0 / 32, (a.job[0].n + 31) / 32);
        }
        ok = __all_sync(~0u, ok && mbar_wait(sums_full + 8 * buf, phase, a.limit, &dead));
        tc_fence_after();
        const uint32_t sums = tmem + buf * BN + ((uint32_t)(quarter * 32) << 16);
        const int blocks = m < a.job[0].m ? min(BLOCKS, (a.job[0].n - n0 + 31) / 32) : 0;
#pragma unroll 1
        for (int s = (q + group) & 1; s < blocks; s += 2) {
          const int c = 32 * s + 16 * half;
          float v[16], u[16];
          unsigned x[3][8];                                    // of the matrices c, g[0], g[1]
          tmem_load(sums + c, v);
          if constexpr (EPI == kUp) {
            tmem_load(sums + BN / 2 + c, u);
            tmem_load_wait(v);
            tmem_load_wait(u);
            if (saved) {
              pack_all(v, x[1], bf16);
              pack_all(u, x[2], bf16);
            }
            act_values<F32>(v, a.act);
#pragma unroll
            for (int e = 0; e < 16; ++e) v[e] *= u[e];
            pack_all(v, x[0], bf16);
          } else {
            // the saved projections' (or the residual's) block of the slot
            const unsigned at = q + s;
            const int slot = at % P::kSlots;
            const char* block = buffers + (2 * P::kResults + P::kAsked * slot) * P::kBlockBytes;
            const bool asked = P::kIsDown || (a.in[0].p && a.in[0].vec);
            if (asked)
              ok = __all_sync(~0u, ok && mbar_wait(slot_full + 8 * (at % (2 * P::kSlots)), at / (2 * P::kSlots) & 1, a.limit, &dead));
            float z[16], d[16];
            if constexpr (EPI == kDown8) {
              // the codes' blocks: rows of 32 bytes under TMA's 32-byte swizzle
              const int piece = row * 32 + ((half ^ (row / 4 & 1)) * 16);
              decode16(z, *reinterpret_cast<const uint4*>(block + piece), scale_at(power[0], s));
              decode16(u, *reinterpret_cast<const uint4*>(block + P::kBlockBytes + piece), scale_at(power[1], s));
            } else if (asked) {
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                if (EPI == kDown) unpack8(z + 8 * e, *reinterpret_cast<const uint4*>(block + block_at(row, 2 * half + e)), bf16);
                unpack8(u + 8 * e, *reinterpret_cast<const uint4*>(block + (EPI == kDown ? P::kBlockBytes : 0) + block_at(row, 2 * half + e)), bf16);
              }
            } else {
              residual_ahead<F32>(u, a.in[0], m + quarter * 32, n0 + c, a.job[0].m - m - quarter * 32, a.job[0].n - n0 - c, bf16);
            }
            if (asked) {
              __syncwarp();
              if (ok && lane == 0) mbar_arrive(slot_empty + 8 * slot);
              __syncwarp();
            }
            if constexpr (EPI == kLinear) {
              if (a.bias) bias_columns(z, a.bias, a.wide_bias, n0 + c, a.job[0].n - n0 - c, bf16);
              tmem_load_wait(v);
              if (a.bias) {
#pragma unroll
                for (int e = 0; e < 16; ++e) v[e] += z[e];
              }
              if (saved) pack_all(v, x[1], bf16);
              if (a.act != ABCD_NO_ACTIVATION) act_values<F32>(v, a.act);
#pragma unroll
              for (int e = 0; e < 16; ++e) v[e] += u[e];
              pack_all(v, x[0], bf16);
            } else {
              act_slopes<F32>(z, d, a.act);
              tmem_load_wait(v);
#pragma unroll
              for (int e = 0; e < 16; ++e) {
                d[e] *= v[e] * u[e];
                u[e] *= z[e];                                  // the hidden matrix
                z[e] *= v[e];
              }
              pack_all(u, x[0], bf16);
              pack_all(d, x[1], bf16);
              pack_all(z, x[2], bf16);
            }
          }
          // once TMA has read the group's last blocks
          if (elected) tma_store_read();
          named_barrier(1 + group, 256);
          put_block(own, row, 2 * half, x[0]);
          if (P::kIsDown || saved) {
            put_block(own + P::kBlockBytes, row, 2 * half, x[1]);
            if (EPI != kLinear) put_block(own + 2 * P::kBlockBytes, row, 2 * half, x[2]);
          }
          const int whole = a.job[0].n & ~7;                   // ODD: columns of the caller's matrices that TMA stores
          if (ODD && ok) {
            __syncwarp();
            const int rows = min(32, a.job[0].m - m - quarter * 32), cols = min(16, a.job[0].n - n0 - c);
            if (EPI == kLinear && result_by_tma) block_tail(own, quarter * 32, 2 * half, a.job[0].c[0], m + quarter * 32, n0 + c, rows, cols, whole);
            if (saved_by_tma)
              for (int k = 0; k < P::kResults - 1; ++k)
                block_tail(own + (k + 1) * P::kBlockBytes, quarter * 32, 2 * half, a.g[k], m + quarter * 32, n0 + c, rows, cols, whole);
          }
          if (!result_by_tma && ok) {
            __syncwarp();
            block_elements(own, quarter * 32, 2 * half, a.job[0].c[0], m + quarter * 32, n0 + c, min(32, a.job[0].m - m - quarter * 32),
                           min(16, a.job[0].n - n0 - c));
          }
          if (saved && !saved_by_tma && ok) {
            __syncwarp();
            for (int k = 0; k < P::kResults - 1; ++k)
              block_elements(own + (k + 1) * P::kBlockBytes, quarter * 32, 2 * half, a.g[k], m + quarter * 32, n0 + c,
                             min(32, a.job[0].m - m - quarter * 32), min(16, a.job[0].n - n0 - c));
          }
          smem_to_tma();
          named_barrier(1 + group, 256);
          if (elected && ok) {
            const int n = n0 + 32 * s;
            const uint32_t from = smem_addr(own);
            const bool pieces = !ODD || n < whole;
            if (result_by_tma && (EPI != kLinear || pieces)) tma_store(&a.c_map, n, m, 0, from);
            if (EPI == kLinear) {
              if (saved_by_tma && pieces) tma_store(&a.g_map[0], n, m, 0, from + P::kBlockBytes);
            } else if (P::kIsDown) {
              tma_store(&a.g_map[0], n, m, 0, from + P::kBlockBytes);
              tma_store(&a.g_map[0], n, m, 1, from + 2 * P::kBlockBytes);
            } else if (saved_by_tma && pieces) {
              tma_store(&a.g_map[0], n, m, 0, from + P::kBlockBytes);
              tma_store(&a.g_map[1], n, m, 0, from + 2 * P::kBlockBytes);
            }
            tma_store_commit();
          }
        }
        // the sums have been read: the next tile but one may overwrite them
        q += blocks;
        tc_fence_before();
        __syncwarp();
        if (ok && lane == 0) mbar_arrive_cluster(empty0 + 8 * buf);
        buf ^= 1;
        if (buf == 0) phase ^= 1;
      }
      if (elected) tma_store_done();
    }
  } else {
    // a warp reads the quarter of tensor memory's lanes that its number in the CTA gives it
    const int quarter = warp & 3, share = (warp - 2) / 4, ewarp = warp - 2;
    const bool bf16 = a.dtype == ABCD_BF16;
    char* buffer = buffers + ewarp * P::kBuffer;
    const uint32_t empty0 = CG == 2 ? at_rank(sums_empty, 0) : sums_empty;
    int buf = 0;
    uint32_t phase = 0;
    // the warp's rows and columns of an item
    struct Part { int m, n, rows, cols; };
    auto part_of = [&](const Item& it) {
      Part p;
      p.m = (it.tm * CG + (int)rank) * P::kRows + quarter * 32;
      p.n = it.tn * P::kOutCols + share * P::kWarpCols;
      p.rows = min(32, a.job[it.job].m - p.m);
      p.cols = min(P::kWarpCols, a.job[it.job].n - p.n);
      return p;
    };
    constexpr bool ahead = P::kAhead;
    // kDown: the saved projections of turn t of an item (16 columns), to one of two pairs of buffers
    char* saved = buffer + P::kTurn;
    constexpr int TURNS = P::kWarpCols / P::CW, SAVED = RowBuffer<F32>::kBytes;
    auto ask = [&](const Part& p, int t) {
      if (p.rows > 0 && p.cols > t * 16) {
        rows_ahead<F32>(saved + (t & 1) * 2 * SAVED, a.in[0], p.m, p.n + t * 16, p.rows, p.cols - t * 16);
        rows_ahead<F32>(saved + (t & 1) * 2 * SAVED + SAVED, a.in[1], p.m, p.n + t * 16, p.rows, p.cols - t * 16);
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
    };
    Item it{};
    Part p{0, 0, 0, 0};
    if (first < items) {
      it = item_of(a, first);
      p = part_of(it);
    }
    if (ahead) {
      ask(p, 0);
      ask(p, 1);
    }
    for (int i = first; i < items; i += step) {
      const Item next = item_of(a, min(i + step, items - 1));
      Part then = part_of(next);
      if (i + step >= items) then.rows = 0;
      const ProductJob& job = a.job[it.job];
      const int m = p.m, n = p.n, rows = p.rows, cols = p.cols;
      if (!__all_sync(~0u, mbar_wait(sums_full + 8 * buf, phase, a.limit, &dead))) break;
      tc_fence_after();
      const uint32_t sums = tmem + buf * BN + ((uint32_t)(quarter * 32) << 16) + share * P::kWarpCols;
      // the sums have been read: the next tile but one may overwrite them
      auto release = [&] {
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster(empty0 + 8 * buf);
      };
      bool mine = rows > 0 && cols > 0, held = true;
      float* part = nullptr;
      constexpr int PARTS = EPI == kUp ? 2 : 1;
      constexpr long long PIECE = (long long)CG * P::kWarps * PARTS * P::kWarpCols * 32;
      if (EPI != kPlain && job.splits > 1) {
        // this part's sums to the workspace [column][row]; the last warp to have done so goes on
        part = job.part + (long long)it.tile * job.splits * PIECE +
               ((long long)rank * P::kWarps + ewarp) * PARTS * P::kWarpCols * 32 + lane;
        if (mine) {
          float* mypart = part + it.split * PIECE;
#pragma unroll 1
          for (int c = 0; c < PARTS * P::kWarpCols; c += P::CW) {
            float v[P::CW];
            tmem_load(sums + (c < P::kWarpCols ? c : BN / 2 + c - P::kWarpCols), v);
            tmem_load_wait(v);
#pragma unroll
            for (int q = 0; q < P::CW; ++q) mypart[(c + q) * 32] = v[q];
          }
          release();
          held = false;
          __threadfence();
          __syncwarp();
          unsigned done = 0;
          unsigned* count = a.count + ((long long)it.tile * CG + rank) * P::kWarps + ewarp;
          if (lane == 0) {
            done = atomicAdd(count, 1u);
            if (done == (unsigned)job.splits - 1) *count = 0;
          }
          done = __shfl_sync(~0u, done, 0);
          __threadfence();
          mine = done == (unsigned)job.splits - 1;
        }
      }
      auto sum_columns = [&](int c, int which, float (&v)[P::CW]) {
        if (EPI == kPlain || job.splits == 1) {
          tmem_load(sums + which * (BN / 2) + c, v);
        } else {
#pragma unroll
          for (int q = 0; q < P::CW; ++q) v[q] = 0.f;
#pragma unroll 2
          for (int s = 0; s < job.splits; ++s) {
            const float* from = part + s * PIECE + (which * P::kWarpCols + c) * 32;
#pragma unroll
            for (int q = 0; q < P::CW; ++q) v[q] += __ldcg(from + q * 32);
          }
        }
      };
      const int end = mine ? min(cols, P::kWarpCols) : 0;
#pragma unroll 1
      for (int c = 0; c < P::kWarpCols; c += P::CW) {
        if (c >= end) {
          if (!ahead) break;
          asm volatile("cp.async.wait_group 1;" ::: "memory");
          if (c / 16 + 2 < TURNS) ask(p, c / 16 + 2);
          else ask(then, c / 16 + 2 - TURNS);
          continue;
        }
        const int w = min(end - c, P::CW);
        const bool last = held && c + P::CW >= end;
        float v[P::CW];
        if constexpr (EPI == kUp) {
          float u[P::CW];
          sum_columns(c, 0, v);
          sum_columns(c, 1, u);
          tmem_load_wait(v);
          tmem_load_wait(u);
          if (last) release();
          if (a.g[0].p) {
            store_matrix<F32, P::CW>(v, a.g[0], m, n + c, rows, w, bf16, buffer);
            store_matrix<F32, P::CW>(u, a.g[1], m, n + c, rows, w, bf16, buffer);
          }
          act_values<F32>(v, a.act);
#pragma unroll
          for (int q = 0; q < P::CW; ++q) v[q] *= u[q];
          store_operand<F32, P::CW>(v, job.c[0], m, n + c, rows, w, bf16, buffer);
        } else if constexpr (EPI == kDown) {
          float z[P::CW], u[P::CW], s[P::CW];
          const char* zbuf = saved + (c / 16 & 1) * 2 * SAVED;
          asm volatile("cp.async.wait_group 1;" ::: "memory");
          __syncwarp();
          row_of<F32>(z, zbuf, bf16);
          row_of<F32>(u, zbuf + SAVED, bf16);
          __syncwarp();
          if (c / 16 + 2 < TURNS) ask(p, c / 16 + 2);
          else ask(then, c / 16 + 2 - TURNS);
          sum_columns(c, 0, v);
          act_slopes<F32>(z, s, a.act);
          tmem_load_wait(v);
          if (last) release();
#pragma unroll
          for (int q = 0; q < P::CW; ++q) {
            s[q] *= v[q] * u[q];
            u[q] *= z[q];                              // the hidden matrix
            z[q] *= v[q];
          }
          store_operand<F32, P::CW>(s, a.g[0], m, n + c, rows, w, bf16, buffer);
          store_operand<F32, P::CW>(z, a.g[1], m, n + c, rows, w, bf16, buffer);
          store_operand<F32, P::CW>(u, job.c[0], m, n + c, rows, w, bf16, buffer);
        } else if constexpr (EPI == kLinear) {
          // the residual's and the bias's columns are on their way while the sums come
          float add[P::CW];
          if (a.in[0].p && !a.in[0].vec) residual_elements<F32, P::CW>(add, buffer, a.in[0], m, n + c, rows, w, bf16);
          else residual_ahead<F32>(add, a.in[0], m, n + c, rows, w, bf16);
          float b = 0.f;
          if (a.bias && lane < w) {
            if (F32 || a.wide_bias) b = __ldg((const float*)a.bias + n + c + lane);
            else b = unpack(__ldg((const unsigned short*)a.bias + n + c + lane), bf16);
          }
          sum_columns(c, 0, v);
          tmem_load_wait(v);
          if (last) release();
          if (a.bias) {
#pragma unroll
            for (int q = 0; q < P::CW; ++q) v[q] += __shfl_sync(~0u, b, q);
          }
          if (a.g[0].p) store_matrix<F32, P::CW>(v, a.g[0], m, n + c, rows, w, bf16, buffer);
          if (a.act != ABCD_NO_ACTIVATION) act_values<F32, P::CW, true>(v, a.act);
#pragma unroll
          for (int q = 0; q < P::CW; ++q) v[q] += add[q];
          store_matrix<F32, P::CW>(v, job.c[0], m, n + c, rows, w, bf16, buffer);
        } else {
          sum_columns(c, 0, v);
          tmem_load_wait(v);
          if (last) release();
          if (job.splits == 1) {
            store_matrix<F32, P::CW>(v, job.c[it.batch], m, n + c, rows, w, bf16, buffer);
          } else {
            const Out o{job.part + ((long long)it.split * job.batches + it.batch) * job.m * job.part_ld, job.part_ld, 0, 1};
#pragma unroll
            for (int e = 0; e < P::CW; e += 16) {      // sixteen of 32 bits take the buffer of 32 of 16
              float x[16];
#pragma unroll
              for (int q = 0; q < 16; ++q) x[q] = v[e + q];
              if (w > e) store_matrix<true, 16>(x, o, m, n + c + e, rows, min(16, w - e), false, buffer);
            }
          }
        }
      }
      if (held && end <= 0) release();
      it = next;
      p = then;
      buf ^= 1;
      if (buf == 0) phase ^= 1;
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
  }
  __syncthreads();
  // a wait gave up: the copies and matrix instructions that are still in flight get time to end
  // before their memory is given back (about 2 ms, far above what any of them takes)
  if (dead)
    for (int q = 0; q < 2000; ++q) __nanosleep(1000);
  tc_fence_before();
  __syncthreads();
  if (CG == 2) cluster_sync();
  tc_fence_after();
  if (warp == 1) tmem_free<CG>(tmem, P::kTmemCols);
  if (threadIdx.x == 0 && dead) atomicOr(a.status, kStatusTimeout);
}

template <int CG, int BN, int EPI, bool F32, bool ODD = false>
abcd_status launch_product(abcd_ctx* ctx, const ProductArgs& a) {
  using P = Product<CG, BN, EPI, F32>;
  auto* kernel = product_kernel<CG, BN, EPI, F32, ODD>;
  const cudaError_t e = allow_smem(ctx, (const void*)kernel);
  if (e != cudaSuccess) return fail(ctx, ABCD_ERR_CUDA, "product_kernel: %s", cudaGetErrorString(e));
  const int items = a.items;
  const int units = P::kCtas * ctx->num_sms / CG;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(CG * (items < units ? items : units)));
  cfg.blockDim = dim3(P::kThreads);
  cfg.dynamicSmemBytes = P::kSmem;
  cfg.stream = ctx->stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = CG;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return check_launch(ctx, "product_kernel", cudaLaunchKernelEx(&cfg, kernel, a));
}

// The tiles that the products come in: 256 x 256 on a pair of CTAs, 128 x 128 or 128 x 64 on one (two
// of them per SM).
// What they cost, in us: fitted to 324 products of 300 to 20,000 tokens of widths 64 x 256, 256 x 1,024
// and 768 x 2,048 in 16 and 32 bits, each timed in all three shapes (the fit is within 8% rms, and its
// choices took 0.6% longer in all than the best ones).  Outside of those, both passes of 1,500 x 28 x 112,
// 8,000 x 1,024 x 4,096 and 1,000,000 x 64 x 256 in 32 bits and of 300 x 2,048 x 8,192, 5,430 x 1,713 x
// 1,601, 40,000 x 1,024 x 1,024 and 16,384 x 2,048 x 8,192 in 16 take at most 4% more than with the best
// one shape for all products of a call.  6,007 x 39 x 6,591 in 32 bits does not: its forward pass takes 363
// us in the smallest tile, 237 in the large one.
// kLinear's epilogues, which move a residual and z besides, are from eleven layers of 300 to 100,000 tokens,
// each timed in all three shapes.
struct Shape {
  int cg, bn, ctas;          // CTAs of a tile, its sums per row, CTAs per SM (one for kDown)
  double fixed;              // of a launch
  double idle, busy;         // of a stage (64 of k) where few SMs, where all ask for operands
  double epilogue[4][2];     // of a tile, by kPlain, kUp, kDown, kLinear and 16 or 32 bits
};
constexpr Shape kShapes[3] = {{2, 256, 1, 7.1, 0.25, 0.34, {{1.7, 1.8}, {2.7, 9.2}, {7.0, 36.0}, {6.0, 10.0}}},
                              {1, 128, 1, 5.9, 0.22, 0.33, {{0.5, 0.8}, {2.5, 4.5}, {6.1, 17.0}, {4.0, 5.5}}},
                              {1, 64, 2, 5.2, 0.24, 0.36, {{0.8, 1.0}, {2.1, 3.6}, {3.3, 8.3}, {5.4, 5.5}}}};

template <int EPI, bool F32> abcd_status launch_shape(abcd_ctx* ctx, int shape, const ProductArgs& a) {
  if (shape == 0) return launch_product<2, 256, EPI, F32>(ctx, a);
  if (shape == 1) return launch_product<1, 128, EPI, F32>(ctx, a);
  return launch_product<1, 64, EPI, F32>(ctx, a);
}
template <bool F32> abcd_status launch_any(abcd_ctx* ctx, int epi, int shape, const ProductArgs& a) {
  if (epi == kUp) return launch_shape<kUp, F32>(ctx, shape, a);
  if (epi == kDown) return launch_shape<kDown, F32>(ctx, shape, a);
  if (epi == kLinear) return launch_shape<kLinear, F32>(ctx, shape, a);
  return launch_shape<kPlain, F32>(ctx, shape, a);
}
// One translation unit each.
abcd_status launch_16(abcd_ctx* ctx, int epi, int shape, const ProductArgs& a);
abcd_status launch_32(abcd_ctx* ctx, int epi, int shape, const ProductArgs& a);

}  // namespace abcd
