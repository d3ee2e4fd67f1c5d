// Lookups in a table of learned rows, and the table's gradient.
//   y[t] = add[t] + s table[i_t] (no row for i_t < 0),   dtable[v] = s sum of dy[t] over the t with i_t = v.
// Forward: bound by HBM (y, add; the table's rows come from L2 when it fits there).
// Backward: the tokens are sorted by the row that they name (a stable radix sort, 8 to 10 bits a pass), so
// that a row's tokens lie next to each other in their own order; runs of equal rows are then summed in
// registers, `kChunk` tokens at a time, and runs that pass the end of a chunk are joined from the chunks'
// parts in order.  No atomic adds a gradient, so every run gives the same sums, whether all tokens name
// one row or each its own.
#include <algorithm>

#include "network.cuh"

namespace abcd {
namespace {

constexpr unsigned kBadIndex = 1u << ABCD_ERR_INVALID_ARG;    // the status bit of an index past the table

// The row that token t names; `rows` for none.
__device__ __forceinline__ unsigned row_of_token(const void* index, int wide, long long t, unsigned rows, unsigned* status) {
  const long long i = wide ? ((const long long*)index)[t] : ((const int*)index)[t];
  if (i >= (long long)rows) atomicOr(status, kBadIndex);
  return i >= 0 && i < (long long)rows ? (unsigned)i : rows;
}

struct LookupArgs {
  const void* table;
  const void* index;
  const void* add;
  void* y;
  long long rows, st, sa, sy;
  unsigned table_rows, cols;
  int wide;                           // 64-bit indices
  float scale;
  unsigned* status;
};

template <typename T>
__global__ void __launch_bounds__(256) embed_kernel(const __grid_constant__ LookupArgs a) {
  pdl_wait();
  const long long n = a.rows * a.cols;
  for (long long i = blockIdx.x * 256LL + threadIdx.x; i < n; i += gridDim.x * 256LL) {
    const long long row = n < (1LL << 32) ? (unsigned)i / a.cols : i / a.cols;
    const unsigned c = (unsigned)(i - row * a.cols);
    const unsigned at = row_of_token(a.index, a.wide, row, a.table_rows, a.status);
    float v = at < a.table_rows ? a.scale * to_f32(((const T*)a.table)[(long long)at * a.st + c]) : 0.f;
    if (a.add) v += to_f32(((const T*)a.add)[row * a.sa + c]);
    ((T*)a.y)[row * a.sy + c] = from_f32<T>(v);
  }
}

// ---- the sort

constexpr int kMaxDigits = 1024;      // bins of a pass
constexpr int kSortThreads = 1024, kSortWarps = kSortThreads / 32;

struct SortArgs {
  const void* index;                  // the first pass's keys; then key, id
  const unsigned* key;
  const unsigned* id;
  unsigned* to_key;
  unsigned* to_id;
  unsigned* count;                    // [digit][tile], then their places
  unsigned* total;                    // [digit] tokens, then their places
  long long n;
  int tiles, per_tile;                // tokens of a tile: a multiple of 1,024
  int shift, bits;
  int wide;
  unsigned table_rows;
  unsigned* status;
};

__device__ __forceinline__ unsigned sort_key(const SortArgs& a, long long i) {
  return a.key ? a.key[i] : row_of_token(a.index, a.wide, i, a.table_rows, a.status);
}

// The tiles' tokens per digit.
__global__ void __launch_bounds__(kSortThreads) sort_count_kernel(const __grid_constant__ SortArgs a) {
  pdl_wait();
  __shared__ unsigned bins[kMaxDigits];
  const int digits = 1 << a.bits;
  for (int d = threadIdx.x; d < digits; d += kSortThreads) bins[d] = 0;
  __syncthreads();
  const long long first = (long long)blockIdx.x * a.per_tile, end = min(first + a.per_tile, a.n);
  for (long long i = first + threadIdx.x; i < end; i += kSortThreads)
    atomicAdd(&bins[sort_key(a, i) >> a.shift & (digits - 1)], 1u);
  __syncthreads();
  for (int d = threadIdx.x; d < digits; d += kSortThreads) a.count[(long long)d * a.tiles + blockIdx.x] = bins[d];
}

// A digit's counts become the tokens of the tiles before; a warp per digit.
__global__ void __launch_bounds__(256) sort_scan_kernel(const __grid_constant__ SortArgs a) {
  pdl_wait();
  const int lane = threadIdx.x & 31, d = blockIdx.x * 8 + threadIdx.x / 32;
  if (d >= 1 << a.bits) return;
  unsigned* c = a.count + (long long)d * a.tiles;
  unsigned before = 0;
  for (int t0 = 0; t0 < a.tiles; t0 += 32) {
    const int t = t0 + lane;
    const unsigned v = t < a.tiles ? c[t] : 0u;
    unsigned s = v;
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
      const unsigned u = __shfl_up_sync(~0u, s, o);
      if (lane >= o) s += u;
    }
    if (t < a.tiles) c[t] = before + s - v;
    before += __shfl_sync(~0u, s, 31);
  }
  if (lane == 0) a.total[d] = before;
}

// A warp's inclusive sum.
__device__ __forceinline__ unsigned warp_sums(unsigned v) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int o = 1; o < 32; o *= 2) {
    const unsigned u = __shfl_up_sync(~0u, v, o);
    if (lane >= o) v += u;
  }
  return v;
}

// Tokens to their places, equal digits in their order: a warp takes consecutive tokens of the tile, 32 at a
// time, and knows how many of a digit the warps before it have.
__global__ void __launch_bounds__(kSortThreads) sort_place_kernel(const __grid_constant__ SortArgs a) {
  pdl_wait();
  extern __shared__ unsigned short before[];          // [warp][digit]: the warp's tokens, then those before it
  __shared__ unsigned place[kMaxDigits], sums[32];
  const int digits = 1 << a.bits, lane = threadIdx.x & 31, warp = threadIdx.x / 32;
  for (int i = threadIdx.x; i < kSortWarps * digits; i += kSortThreads) before[i] = 0;
  const unsigned mine = threadIdx.x < digits ? a.total[threadIdx.x] : 0u;
  const unsigned up_to = warp_sums(mine);
  if (lane == 31) sums[warp] = up_to;
  __syncthreads();
  if (warp == 0) sums[lane] = warp_sums(sums[lane]);
  __syncthreads();
  if (threadIdx.x < digits)
    place[threadIdx.x] = (warp ? sums[warp - 1] : 0u) + up_to - mine + a.count[(long long)threadIdx.x * a.tiles + blockIdx.x];
  const int per_warp = a.per_tile / kSortWarps;
  const long long first = (long long)blockIdx.x * a.per_tile + (long long)warp * per_warp;
  unsigned short* own = before + warp * digits;
  for (int k = 0; k < per_warp; k += 32) {
    const long long i = first + k + lane;
    const bool in = i < a.n;
    const unsigned d = in ? sort_key(a, i) >> a.shift & (digits - 1) : ~0u;
    const unsigned same = __match_any_sync(~0u, d);
    if (in && lane == __ffs(same) - 1) own[d] += (unsigned short)__popc(same);
    __syncwarp();
  }
  __syncthreads();
  if (threadIdx.x < digits) {
    unsigned s = 0;
    for (int w = 0; w < kSortWarps; ++w) {
      const unsigned v = before[w * digits + threadIdx.x];
      before[w * digits + threadIdx.x] = (unsigned short)s;
      s += v;
    }
  }
  __syncthreads();
  for (int k = 0; k < per_warp; k += 32) {
    const long long i = first + k + lane;
    const bool in = i < a.n;
    const unsigned key = in ? sort_key(a, i) : 0u, d = in ? key >> a.shift & (digits - 1) : ~0u;
    const unsigned same = __match_any_sync(~0u, d);
    if (in) {
      const unsigned at = place[d] + own[d] + __popc(same & ((1u << lane) - 1));
      a.to_key[at] = key;
      a.to_id[at] = a.id ? a.id[i] : (unsigned)i;
    }
    __syncwarp();
    if (in && lane == __ffs(same) - 1) own[d] += (unsigned short)__popc(same);
    __syncwarp();
  }
}

// ---- the sums

constexpr int kChunk = 256;           // sorted tokens of a CTA

struct SumArgs {
  const void* dy;
  const unsigned* key;
  const unsigned* id;
  void* dtable;
  float* part;                        // [chunk][2][cols]: a run that began before the chunk; one that goes on after it
  long long n, sdy, st;
  unsigned table_rows, cols;
  float scale;
  long long chunks;
};

template <typename T> __device__ __forceinline__ void put_row(const SumArgs& a, unsigned row, unsigned c, float v) {
  ((T*)a.dtable)[(long long)row * a.st + c] = from_f32<T>(a.scale * v);
}

// One CTA per chunk and 256 columns: a thread walks the chunk's tokens with its column.
template <typename T>
__global__ void __launch_bounds__(256) embed_sum_kernel(const __grid_constant__ SumArgs a) {
  pdl_wait();
  __shared__ unsigned key[kChunk + 2], id[kChunk];
  const long long chunk = blockIdx.x, first = chunk * kChunk;
  const int n = (int)min((long long)kChunk, a.n - first);
  for (int i = threadIdx.x; i < n; i += 256) {
    key[i + 1] = a.key[first + i];
    id[i] = a.id[first + i];
  }
  if (threadIdx.x == 0) {
    key[0] = first > 0 ? a.key[first - 1] : a.table_rows;
    key[n + 1] = first + n < a.n ? a.key[first + n] : a.table_rows;
  }
  __syncthreads();
  const unsigned c = blockIdx.y * 256 + threadIdx.x;
  if (c >= a.cols) return;
  float s = 0.f;
  bool began = key[1] == key[0];      // the run began before the chunk
  for (int i = 0; i < n && key[i + 1] < a.table_rows; ++i) {
    s += to_f32(((const T*)a.dy)[(long long)id[i] * a.sdy + c]);
    const bool last = key[i + 2] != key[i + 1];
    if (!last && i + 1 < n) continue;
    if (began) a.part[2 * chunk * a.cols + c] = s;
    else if (!last) a.part[(2 * chunk + 1) * a.cols + c] = s;
    else put_row<T>(a, key[i + 1], c, s);
    s = 0.f;
    began = false;
  }
}

// Runs that pass a chunk's end: the CTA of the chunk that they begin in adds their parts in order.
template <typename T>
__global__ void __launch_bounds__(256) embed_join_kernel(const __grid_constant__ SumArgs a) {
  pdl_wait();
  const long long chunk = blockIdx.x, end = (chunk + 1) * kChunk;
  if (end >= a.n) return;
  const unsigned row = a.key[end - 1];
  if (row >= a.table_rows || a.key[end] != row) return;
  if (a.key[end - kChunk] == row && end > kChunk && a.key[end - kChunk - 1] == row) return;   // it began earlier
  const unsigned c = blockIdx.y * 256 + threadIdx.x;
  if (c >= a.cols) return;
  float s = a.part[(2 * chunk + 1) * a.cols + c];
  for (long long q = chunk + 1; q < a.chunks && a.key[q * kChunk] == row; ++q) s += a.part[2 * q * a.cols + c];
  put_row<T>(a, row, c, s);
}

// How the tokens are sorted: passes of equal bits for the rows and one more (none).
struct SortPlan {
  int bits, passes, tiles, per_tile;
};
SortPlan sort_plan(long long tokens, long long table_rows) {
  SortPlan p;
  int need = 1;
  while ((1LL << need) <= table_rows) ++need;
  p.passes = (need + 9) / 10;
  p.bits = (need + p.passes - 1) / p.passes;
  const long long least = 4096;
  long long per = std::max(least, (tokens + kNetSms - 1) / kNetSms);
  per = (per + kSortThreads - 1) / kSortThreads * kSortThreads;
  // a warp counts its tokens of a digit in 16 bits
  per = std::min<long long>(per, 32768 / 32 * kSortThreads);
  p.per_tile = (int)per;
  p.tiles = (int)((tokens + per - 1) / per);
  return p;
}

// The workspace behind its header.
struct EmbedScratch {
  unsigned *key[2], *id[2], *count, *total;
  float* part;
  size_t bytes;
};
EmbedScratch scratch_of(char* base, long long tokens, long long table_rows, long long cols) {
  const SortPlan p = sort_plan(tokens, table_rows);
  size_t at = kNetHeader;
  const auto take = [&](size_t bytes) { char* q = base ? base + at : nullptr; at += net_align(bytes); return q; };
  EmbedScratch s;
  for (int k = 0; k < 2; ++k) {
    s.key[k] = (unsigned*)take(4 * (size_t)tokens);
    s.id[k] = (unsigned*)take(4 * (size_t)tokens);
  }
  s.count = (unsigned*)take((size_t)4 * kMaxDigits * (size_t)p.tiles);
  s.total = (unsigned*)take((size_t)4 * kMaxDigits);
  s.part = (float*)take((size_t)8 * (size_t)cols * (size_t)((tokens + kChunk - 1) / kChunk));
  s.bytes = at;
  return s;
}

bool index_ok(const void* index, int dtype, long long n) {
  return (dtype == ABCD_I32 || dtype == ABCD_I64) && (n == 0 || index) && ((uintptr_t)index & (dtype == ABCD_I64 ? 7 : 3)) == 0;
}
bool scale_ok(float s) { return s > -3e38f && s < 3e38f; }
// Whether a matrix reaches into an index vector.
bool on_index(const abcd_matrix* m, const void* index, int dtype, long long n) {
  const abcd_matrix v{const_cast<void*>(index), n ? 1LL : 0LL, n * (dtype == ABCD_I64 ? 2 : 1), n * (dtype == ABCD_I64 ? 2 : 1), ABCD_F32};
  return overlap(m, &v);
}

}  // namespace
}  // namespace abcd

using namespace abcd;

extern "C" abcd_status abcd_embedding_workspace_size(long long tokens, long long table_rows, long long cols, size_t* bytes) {
  if (!bytes || tokens < 0 || tokens > kMaxNetRows || table_rows < 1 || table_rows > kMaxNetRows || cols < 1 || cols > kMaxNetCols)
    return ABCD_ERR_INVALID_ARG;
  *bytes = scratch_of(nullptr, tokens, table_rows, cols).bytes;
  return ABCD_OK;
}

extern "C" abcd_status abcd_embedding(abcd_ctx* ctx, const abcd_matrix* table, const void* index, int index_dtype,
                                      float scale, const abcd_matrix* add, const abcd_matrix* y) {
  const char* what = "abcd_embedding";
  if (!ctx) return ABCD_ERR_INVALID_ARG;
  if (!matrix_ok(table) || !matrix_ok(y) || table->dtype != y->dtype || table->cols != y->cols || table->rows < 1 ||
      (add && (!matrix_ok(add) || !same_form(add, y))))
    return fail(ctx, ABCD_ERR_INVALID_ARG, "%s: bad matrices", what);
  if (!index_ok(index, index_dtype, y->rows)) return fail(ctx, ABCD_ERR_INVALID_ARG, "%s: bad indices", what);
  if (!scale_ok(scale)) return fail(ctx, ABCD_ERR_INVALID_ARG, "%s: scale must be finite", what);
  if (!ctx->net_base) return fail(ctx, ABCD_ERR_WORKSPACE, "%s: no network workspace", what);
  if (y->rows == 0) return ABCD_OK;
  const bool on_add = add && overlap(add, y) && !(add->data == y->data && (add->stride == y->stride || y->rows == 1));
  if (overlap(table, y) || on_add || on_index(y, index, index_dtype, y->rows))
    return fail(ctx, ABCD_ERR_INVALID_ARG, "%s: y overlaps an operand", what);
  const LookupArgs a{table->data, index, add ? add->data : nullptr, y->data, y->rows, table->stride, add ? add->stride : 0, y->stride,
                     (unsigned)table->rows, (unsigned)y->cols, index_dtype == ABCD_I64, scale, (unsigned*)ctx->net_base};
  return with_type(y->dtype, [&](auto t) {
    using T = decltype(t);
    const long long grid = std::min<long long>((y->rows * y->cols + 255) / 256, 8LL * ctx->num_sms);
    return check_launch(ctx, "embed_kernel", launch_pdl(embed_kernel<T>, dim3((unsigned)grid), dim3(256), 0, ctx->stream, a));
  });
}

extern "C" abcd_status abcd_embedding_backward(abcd_ctx* ctx, const abcd_matrix* dy, const void* index, int index_dtype,
                                               float scale, const abcd_matrix* dtable) {
  const char* what = "abcd_embedding_backward";
  if (!ctx) return ABCD_ERR_INVALID_ARG;
  if (!matrix_ok(dy) || !matrix_ok(dtable) || dy->dtype != dtable->dtype || dy->cols != dtable->cols || dtable->rows < 1)
    return fail(ctx, ABCD_ERR_INVALID_ARG, "%s: bad matrices", what);
  if (!index_ok(index, index_dtype, dy->rows)) return fail(ctx, ABCD_ERR_INVALID_ARG, "%s: bad indices", what);
  if (!scale_ok(scale)) return fail(ctx, ABCD_ERR_INVALID_ARG, "%s: scale must be finite", what);
  if (overlap(dy, dtable) || on_index(dtable, index, index_dtype, dy->rows))
    return fail(ctx, ABCD_ERR_INVALID_ARG, "%s: dtable overlaps an operand", what);
  const long long n = dy->rows;
  const EmbedScratch s = scratch_of(ctx->net_base, n, dtable->rows, dy->cols);
  if (!ctx->net_base || s.bytes > ctx->net_bytes)
    return fail(ctx, ABCD_ERR_WORKSPACE, "%s: the network workspace has %zu bytes, needs %zu", what, ctx->net_bytes, s.bytes);
  const size_t e = elem_size(dtable->dtype);
  const cudaError_t z = cudaMemset2DAsync(dtable->data, (size_t)dtable->stride * e, 0, (size_t)dtable->cols * e, (size_t)dtable->rows, ctx->stream);
  if (z != cudaSuccess) return fail(ctx, ABCD_ERR_CUDA, "%s: %s", what, cudaGetErrorString(z));
  if (n == 0) return ABCD_OK;
  const SortPlan p = sort_plan(n, dtable->rows);
  const size_t smem = (size_t)kSortWarps * 2 * ((size_t)1 << p.bits);
  const cudaError_t room = allow_smem(ctx, (const void*)sort_place_kernel);
  if (room != cudaSuccess) return fail(ctx, ABCD_ERR_CUDA, "%s: %s", what, cudaGetErrorString(room));
  SortArgs q{index, nullptr, nullptr, s.key[0], s.id[0], s.count, s.total, n, p.tiles, p.per_tile, 0, p.bits,
             index_dtype == ABCD_I64, (unsigned)dtable->rows, (unsigned*)ctx->net_base};
  for (int pass = 0; pass < p.passes; ++pass) {
    q.shift = pass * p.bits;
    abcd_status st = check_launch(ctx, "sort_count_kernel", launch_pdl(sort_count_kernel, dim3(p.tiles), dim3(kSortThreads), 0, ctx->stream, q));
    if (st != ABCD_OK) return st;
    st = check_launch(ctx, "sort_scan_kernel", launch_pdl(sort_scan_kernel, dim3(((1 << p.bits) + 7) / 8), dim3(256), 0, ctx->stream, q));
    if (st != ABCD_OK) return st;
    st = check_launch(ctx, "sort_place_kernel", launch_pdl(sort_place_kernel, dim3(p.tiles), dim3(kSortThreads), smem, ctx->stream, q));
    if (st != ABCD_OK) return st;
    q.key = q.to_key;
    q.id = q.to_id;
    q.to_key = s.key[(pass + 1) & 1];
    q.to_id = s.id[(pass + 1) & 1];
  }
  const SumArgs a{dy->data, q.key, q.id, dtable->data, s.part, n, dy->stride, dtable->stride, (unsigned)dtable->rows,
                  (unsigned)dy->cols, scale, (n + kChunk - 1) / kChunk};
  return with_type(dy->dtype, [&](auto t) {
    using T = decltype(t);
    const dim3 grid((unsigned)a.chunks, (a.cols + 255) / 256);
    const abcd_status st = check_launch(ctx, "embed_sum_kernel", launch_pdl(embed_sum_kernel<T>, grid, dim3(256), 0, ctx->stream, a));
    if (st != ABCD_OK) return st;
    return check_launch(ctx, "embed_join_kernel", launch_pdl(embed_join_kernel<T>, grid, dim3(256), 0, ctx->stream, a));
  });
}
