// Lookups in a table of learned rows, and the table's gradient.
//   y[t] = add[t] + s table[i_t] (no row for i_t < 0),   dtable[v] = s sum of dy[t] over the t with i_t = v.
// Forward: bound by HBM (y, add; the table's rows come from L2 when it fits there).
// Backward: the tokens are sorted by the row that they name (a stable radix sort, up to 10 bits a pass), so
// that a row's tokens lie next to each other in their own order; runs of equal rows are then summed in
// registers, up to `kChunk` tokens a CTA, and runs that pass the end of a chunk are joined from the chunks'
// parts in order.  No atomic adds a gradient, so every run gives the same sums, whether all tokens name
// one row or each its own.
// 1,000,000 tokens of 100,000 rows of 64 fp32: forward 53 us (5.4 TB/s), backward 105: the sums 60 (4.7 TB/s: a
// token's row is 256 bytes somewhere), the sort 36 (two passes of nine bits: counts 6, places 12 each), joins 5.
#include <algorithm>
#include <type_traits>

#include "network.cuh"

namespace abcd {
namespace {

constexpr unsigned kBadIndex = 1u << ABCD_ERR_INVALID_ARG;    // the status bit of an index past the table

// The row that token t names as it is given, and as it is taken: `rows` for none.
__device__ __forceinline__ long long index_of(const void* index, int wide, long long t) {
  return wide ? __ldg((const long long*)index + t) : (long long)__ldg((const int*)index + t);
}
__device__ __forceinline__ unsigned row_of(long long i, unsigned rows, unsigned* status) {
  if (i >= (long long)rows) atomicOr(status, kBadIndex);
  return i >= 0 && i < (long long)rows ? (unsigned)i : rows;
}

struct LookupArgs {
  const void* table;
  const void* index;
  const void* add;
  void* y;
  long long rows, st, sa, sy;
  unsigned table_rows, cols, lanes;   // lanes: threads of a token, up to 256
  int slices;                         // of lanes x V columns
  int lookup;                         // tokens of a group of threads
  int add_vec;                        // add's rows start on V elements' boundaries (the table's and y's do)
  int wide;                           // 64-bit indices
  float scale;
  unsigned* status;
};

// V elements at p; of a row's last vector, which may pass its end, those that `left` counts.
template <typename T, int V> __device__ __forceinline__ Pack<T, V> load_part(const T* p, bool whole, int left) {
  Pack<T, V> v;
  if (whole) {
    v = *reinterpret_cast<const Pack<T, V>*>(p);
  } else {
#pragma unroll
    for (int e = 0; e < V; ++e) v.v[e] = e < left ? p[e] : T(0.f);
  }
  return v;
}

// V consecutive columns a thread (16 bytes, or one where rows start anywhere), `lanes` threads a token; a CTA
// takes up to kLookup tokens of each group of threads.  Bound by latency, unless many rows are on their way at once:
// the indices go to shared memory first, and a thread's loads are asked for U tokens at a time, without a
// condition (with one, the compiler moved each load to its use: 1,000,000 x 64 fp32 90 us instead of 53).
constexpr int kLookup = 16;           // at most: fewer where that leaves SMs idle
template <typename T, int V, bool ADD>
__global__ void __launch_bounds__(256) embed_kernel(const __grid_constant__ LookupArgs a) {
  pdl_wait();
  using P = Pack<T, V>;
  constexpr int U = ADD || V > 4 ? 4 : 8;
  __shared__ unsigned at[256 * kLookup];
  const unsigned groups = 256u / a.lanes, group = threadIdx.x / a.lanes;
  const long long first = blockIdx.x / a.slices * (long long)(groups * a.lookup);
  const int n = (int)min((long long)(groups * a.lookup), a.rows - first);
  for (int i = threadIdx.x; i < n; i += 4 * 256) {
    long long named[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) named[k] = index_of(a.index, a.wide, first + min(i + k * 256, n - 1));
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (i + k * 256 < n) at[i + k * 256] = row_of(named[k], a.table_rows, a.status);
  }
  __syncthreads();
  const unsigned c = (unsigned)(blockIdx.x % a.slices * a.lanes + threadIdx.x - group * a.lanes) * V;
  if (group >= groups || c >= a.cols || (int)group >= n) return;
  const bool whole = V == 1 || c + V <= a.cols, whole_add = whole && a.add_vec;
  const int left = (int)(a.cols - c);
  const T* table = (const T*)a.table + c;
  const T* add = ADD ? (const T*)a.add + first * a.sa + c : nullptr;
  T* y = (T*)a.y + first * a.sy + c;
  // the groups' tokens in turn
  for (int i0 = group; i0 < n; i0 += U * groups) {
    P v[U], w[ADD ? U : 1];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = min(i0 + u * (int)groups, n - 1);
      const unsigned row = at[i] < a.table_rows ? at[i] : 0u;
      v[u] = load_part<T, V>(table + row * a.st, whole, left);
      if (ADD) w[u] = load_part<T, V>(add + i * a.sa, whole_add, left);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + u * (int)groups;
      if (i >= n) break;
      const bool none = at[i] >= a.table_rows;
#pragma unroll
      for (int e = 0; e < V; ++e) {
        float x = none ? 0.f : a.scale * to_f32(v[u].v[e]);
        if (ADD) x += to_f32(w[u].v[e]);
        v[u].v[e] = from_f32<T>(x);
      }
      T* to = y + i * a.sy;
      if (whole) {
        *reinterpret_cast<P*>(to) = v[u];
      } else {
#pragma unroll
        for (int e = 0; e < V; ++e)
          if (e < left) to[e] = v[u].v[e];
      }
    }
  }
}

// ---- the sort

constexpr int kMaxDigits = 1024;      // bins of a pass
constexpr int kScanned = 8;           // tiles up to which each adds up the counts for itself
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
  // the first kernel of all clears the table's gradient with the CTAs behind its tiles' own
  char* zero;
  long long zero_rows, zero_bytes, zero_stride;       // of a row
};

// Clears the rows, a piece of E bytes at a time, with the CTAs from `first` on.
template <typename E> __device__ __forceinline__ void clear_rows(const SortArgs& a, int first) {
  const long long per_row = a.zero_bytes / (long long)sizeof(E), n = a.zero_rows * per_row;
  for (long long i = (blockIdx.x - first) * (long long)kSortThreads + threadIdx.x; i < n; i += (gridDim.x - first) * (long long)kSortThreads) {
    const long long row = a.zero_rows == 1 ? 0 : n < (1LL << 32) ? (unsigned)i / (unsigned)per_row : i / per_row;
    *reinterpret_cast<E*>(a.zero + row * a.zero_stride + (i - row * per_row) * (long long)sizeof(E)) = E{};
  }
}
__device__ __forceinline__ void clear_rows(const SortArgs& a, int first) {
  const unsigned long long all = (uintptr_t)a.zero | (unsigned long long)a.zero_bytes | (unsigned long long)(a.zero_rows > 1 ? a.zero_stride : 0);
  if (all % 16 == 0) clear_rows<uint4>(a, first);
  else if (all % 4 == 0) clear_rows<unsigned>(a, first);
  else clear_rows<unsigned short>(a, first);
}

// The keys of N tokens, `step` apart from the first on: all are on their way before one is looked at.  (Past
// `end`, that of the last one.)
template <int N> __device__ __forceinline__ void sort_keys(const SortArgs& a, long long first, int step, long long end, unsigned (&key)[N]) {
  if (a.key) {
#pragma unroll
    for (int k = 0; k < N; ++k) key[k] = a.key[min(first + k * step, end - 1)];
  } else {
    long long named[N];
#pragma unroll
    for (int k = 0; k < N; ++k) named[k] = index_of(a.index, a.wide, min(first + k * step, end - 1));
#pragma unroll
    for (int k = 0; k < N; ++k) key[k] = row_of(named[k], a.table_rows, a.status);
  }
}

// The tiles' tokens per digit.
__global__ void __launch_bounds__(kSortThreads) sort_count_kernel(const __grid_constant__ SortArgs a) {
  pdl_wait();
  if (blockIdx.x >= a.tiles) return clear_rows(a, a.tiles);
  __shared__ unsigned bins[kMaxDigits];
  const int digits = 1 << a.bits;
  for (int d = threadIdx.x; d < digits; d += kSortThreads) bins[d] = 0;
  __syncthreads();
  const long long first = (long long)blockIdx.x * a.per_tile, end = min(first + a.per_tile, a.n);
  constexpr int U = 4;
  for (long long i = first + threadIdx.x; i < end; i += U * kSortThreads) {
    unsigned key[U];
    sort_keys(a, i, kSortThreads, end, key);
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (i + u * kSortThreads < end) atomicAdd(&bins[key[u] >> a.shift & (digits - 1)], 1u);
  }
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

// Tokens to their places, equal digits in their order: a warp takes IT x 32 consecutive tokens of the tile, and
// knows how many of a digit its lanes and the warps before it have.  They go to shared memory in the order of
// their digits first, so that consecutive lanes write consecutive places.  One tile counts for itself.  Bound
// by latency: 1,000,000 tokens, nine bits, 12 us; with the match instruction instead of ballots 18, and with
// scattered writes 27.  (The 1,024 threads leave 64 registers each, and 88 to 172 bytes, by the tile's size, spill:
// the warps' counts of two digits are 32 registers.)
template <int IT>
__global__ void __launch_bounds__(kSortThreads) sort_place_kernel(const __grid_constant__ SortArgs a) {
  pdl_wait();
  if (blockIdx.x >= a.tiles) return clear_rows(a, a.tiles);
  extern __shared__ uint2 sorted[];                   // key and id of the tile's tokens
  __shared__ unsigned place[kMaxDigits], local[kMaxDigits], sums[32];
  const int digits = 1 << a.bits, lane = threadIdx.x & 31, warp = threadIdx.x / 32;
  const long long first = (long long)blockIdx.x * (IT * kSortThreads);
  const int n = (int)min((long long)(IT * kSortThreads), a.n - first), start = warp * 32 * IT + lane;
  // [warp][digit]: the warp's tokens, then those of the warps before it
  unsigned short* before = reinterpret_cast<unsigned short*>(sorted + IT * kSortThreads);
  unsigned short* own = before + warp * digits;
  unsigned key[IT];
  sort_keys(a, first + start, 32, a.n, key);
  unsigned all = 0, ahead = 0;                      // the digit's tokens, and those of the tiles before
  if (a.tiles > 1 && threadIdx.x < digits) {
    const unsigned* c = a.count + (long long)threadIdx.x * a.tiles;
    if (a.tiles > kScanned) {
      all = a.total[threadIdx.x];
      ahead = c[blockIdx.x];
    } else {
      unsigned v[kScanned];
#pragma unroll
      for (int t = 0; t < kScanned; ++t) v[t] = c[min(t, a.tiles - 1)];
#pragma unroll
      for (int t = 0; t < kScanned; ++t) {
        ahead += t < (int)blockIdx.x ? v[t] : 0u;
        all += t < a.tiles ? v[t] : 0u;
      }
    }
  }
  for (int i = threadIdx.x; i < kSortWarps * digits / 8; i += kSortThreads) reinterpret_cast<uint4*>(before)[i] = make_uint4(0u, 0u, 0u, 0u);
  __syncthreads();
  unsigned rank[IT];                                  // among the warp's tokens of the digit
#pragma unroll
  for (int k = 0; k < IT; ++k) {
    const bool in = start + 32 * k < n;
    const unsigned d = key[k] >> a.shift & (digits - 1);
    // the lanes with the same digit, bit by bit
    unsigned same = __ballot_sync(~0u, in);
    for (int b = 0; b < a.bits; ++b) {
      const bool one = d >> b & 1;
      const unsigned ones = __ballot_sync(~0u, one);
      same &= one ? ones : ~ones;
    }
    rank[k] = __popc(same & ((1u << lane) - 1));
    unsigned had = in ? own[d] : 0u;
    __syncwarp();
    if (in && rank[k] == 0) own[d] = (unsigned short)(had + __popc(same));
    rank[k] += had;
    __syncwarp();
  }
  __syncthreads();
  // the warps' tokens of a digit become those of the warps before; a thread takes two digits, a word
  if (threadIdx.x < digits / 2) {
    unsigned* word = reinterpret_cast<unsigned*>(before) + threadIdx.x;
    unsigned v[kSortWarps], sum = 0;
#pragma unroll
    for (int w = 0; w < kSortWarps; ++w) v[w] = word[w * (digits / 2)];
#pragma unroll
    for (int w = 0; w < kSortWarps; ++w) {
      word[w * (digits / 2)] = sum;
      sum += v[w];
    }
    local[2 * threadIdx.x] = sum & 0xffffu;
    local[2 * threadIdx.x + 1] = sum >> 16;
  }
  __syncthreads();
  const unsigned total = threadIdx.x < digits ? local[threadIdx.x] : 0u;
  // a digit's first place, in the tile and in all
  auto first_places = [&](unsigned count) {
    const unsigned up_to = warp_sums(count);
    __syncthreads();
    if (lane == 31) sums[warp] = up_to;
    __syncthreads();
    if (warp == 0) sums[lane] = warp_sums(sums[lane]);
    __syncthreads();
    return (warp ? sums[warp - 1] : 0u) + up_to - count;
  };
  const unsigned inside = first_places(total);
  unsigned outside = inside;
  if (a.tiles > 1) outside = first_places(all) + ahead;
  if (threadIdx.x < digits) {
    local[threadIdx.x] = inside;
    place[threadIdx.x] = outside - inside;
  }
  unsigned id[IT];
#pragma unroll
  for (int k = 0; k < IT; ++k) {
    const long long i = min(first + start + 32 * k, a.n - 1);
    id[k] = a.id ? a.id[i] : (unsigned)i;
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < IT; ++k) {
    if (start + 32 * k >= n) break;
    const unsigned d = key[k] >> a.shift & (digits - 1);
    sorted[local[d] + own[d] + rank[k]] = make_uint2(key[k], id[k]);
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < IT; ++k) {
    const int i = threadIdx.x + k * kSortThreads;
    if (i >= n) break;
    const uint2 t = sorted[i];
    const unsigned at = place[t.x >> a.shift & (digits - 1)] + i;
    a.to_key[at] = t.x;
    a.to_id[at] = t.y;
  }
}

// ---- the sums

constexpr int kChunk = 256;           // sorted tokens of a CTA at most

struct SumArgs {
  const void* dy;
  const unsigned* key;
  const unsigned* id;
  void* dtable;
  float* part;                        // [chunk][2][ld]: a run that began before the chunk; one that goes on after it
  long long n, sdy, st;
  unsigned table_rows, cols, ld;
  float scale;
  int lanes;                          // threads of a token's row, up to 256, V columns each
  int slices;                         // of lanes x V columns
  int chunk;                          // sorted tokens of a CTA
  int table_vec;                      // dtable's rows start on 16-byte boundaries
  long long chunks;
};

// V columns of a row of the table's gradient.
template <typename T, int V> __device__ __forceinline__ void put_row(const SumArgs& a, unsigned row, unsigned c, const float (&s)[V]) {
  T* to = (T*)a.dtable + (long long)row * a.st + c;
  if (V > 1 && a.table_vec && c + V <= a.cols) {
    Pack<T, V> q;
#pragma unroll
    for (int e = 0; e < V; ++e) q.v[e] = from_f32<T>(a.scale * s[e]);
    *reinterpret_cast<Pack<T, V>*>(to) = q;
  } else {
#pragma unroll
    for (int e = 0; e < V; ++e)
      if (c + e < a.cols) to[e] = from_f32<T>(a.scale * s[e]);
  }
}

// A chunk's tokens, in groups of threads that each walk a stretch of them, V columns a thread; eight (of
// eight columns four) tokens' rows are on their way at once.  A run of equal rows inside a stretch is a row of the result.  One that
// began before the stretch (its head) or goes on after it (its tail) is left in shared memory, and the
// group that a run begins in adds up what the next ones have of it; what passes the chunk goes to the
// workspace.
template <typename T, int V>
__global__ void __launch_bounds__(256) embed_sum_kernel(const __grid_constant__ SumArgs a) {
  pdl_wait();
  __shared__ unsigned key[kChunk + 2], id[kChunk];
  __shared__ float head[256 * V], tail[256 * V];
  const long long chunk = blockIdx.x / a.slices, first = chunk * a.chunk;
  const int n = (int)min((long long)a.chunk, a.n - first);
  const int lane = threadIdx.x % a.lanes, group = threadIdx.x / a.lanes, groups = 256 / a.lanes, stretch = (a.chunk + groups - 1) / groups;
  for (int i = threadIdx.x; i < a.chunk + 1; i += 256) {
    key[i + 1] = i < n || first + i < a.n ? a.key[first + i] : a.table_rows + 1;
    if (i < n) id[i] = a.id[first + i];
  }
  if (threadIdx.x == 0) key[0] = first > 0 ? a.key[first - 1] : a.table_rows + 1;
  __syncthreads();
  // key[i + 1] is token i's; rows past the table's are no rows, sorted to the end
  const unsigned c = ((unsigned)(blockIdx.x % a.slices) * a.lanes + lane) * V;
  const bool in = c < a.cols && group < groups;
  const int g0 = group < groups ? group * stretch : n, g1 = min(g0 + stretch, n);
  constexpr int U = V > 4 ? 4 : 8;
  float s[V] = {};
  bool began = g0 < g1 && key[g0] == key[g0 + 1];       // the run at hand began before the stretch
  bool has_tail = false;
  for (int i0 = g0; i0 < g1 && key[i0 + 1] < a.table_rows; i0 += U) {
    Pack<T, V> v[U];
    if (in) {
#pragma unroll
      for (int u = 0; u < U; ++u)     // without a condition, so that all are on their way before the first is used
        v[u] = load_part<T, V>((const T*)a.dy + (long long)id[min(i0 + u, g1 - 1)] * a.sdy + c, V == 1 || c + V <= a.cols, (int)(a.cols - c));
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + u;
      if (i >= g1 || key[i + 1] >= a.table_rows) break;
#pragma unroll
      for (int e = 0; e < V; ++e) s[e] += to_f32(v[u].v[e]);
      const bool ends = key[i + 2] != key[i + 1];
      if (!ends && i + 1 < g1) continue;
      if (began) {
#pragma unroll
        for (int e = 0; e < V; ++e) head[threadIdx.x * V + e] = s[e];
      } else if (!ends) {
        has_tail = true;
#pragma unroll
        for (int e = 0; e < V; ++e) tail[threadIdx.x * V + e] = s[e];
      } else if (in) {
        put_row<T, V>(a, key[i + 1], c, s);
      }
#pragma unroll
      for (int e = 0; e < V; ++e) s[e] = 0.f;
      began = false;
    }
  }
  __syncthreads();
  if (!in) return;
  // what the groups from `from` on have of the run of `row`, added to s; whether it goes on after the chunk
  auto follow = [&](unsigned row, int from) {
    for (int g = from; g * stretch < n && key[g * stretch + 1] == row; ++g) {
#pragma unroll
      for (int e = 0; e < V; ++e) s[e] += head[(g * a.lanes + lane) * V + e];
    }
    return key[n] == row && key[n + 1] == row;
  };
  auto leave = [&](int which) {
    float* to = a.part + (2 * chunk + which) * a.ld + c;
#pragma unroll
    for (int e = 0; e < V; ++e)
      if (c + e < a.cols) to[e] = s[e];
  };
  if (has_tail) {
#pragma unroll
    for (int e = 0; e < V; ++e) s[e] = tail[threadIdx.x * V + e];
    const unsigned row = key[g1];
    if (follow(row, group + 1)) leave(1);
    else put_row<T, V>(a, row, c, s);
  }
  if (group == 0 && key[0] == key[1] && key[1] < a.table_rows) {
#pragma unroll
    for (int e = 0; e < V; ++e) s[e] = 0.f;
    follow(key[1], 0);
    leave(0);
  }
}

// Runs that pass a chunk's end, by the chunk that they begin in.  A group of up to sixteen threads, four columns
// each, has a chunk; a run over few chunks it adds up by itself, for longer ones all groups of the CTA take
// consecutive parts side by side, whose sums are then added in their order.
constexpr int kJoinThreads = 1024, kJoinLanes = 16, kJoinAlone = 32;
template <typename T>
__global__ void __launch_bounds__(kJoinThreads) embed_join_kernel(const __grid_constant__ SumArgs a) {
  pdl_wait();
  __shared__ float4 run[kJoinThreads];
  __shared__ bool long_of[kJoinThreads];
  const int lane = threadIdx.x % a.lanes, group = threadIdx.x / a.lanes, groups = kJoinThreads / a.lanes;
  const long long base = blockIdx.x / a.slices * (long long)groups;
  const unsigned c = (blockIdx.x % a.slices * a.lanes + lane) * 4;
  const bool in = c < a.cols && group < groups;
  const auto has = [&](long long q, unsigned row) { return q < a.chunks && a.key[q * a.chunk] == row; };
  const auto part = [&](long long q, int which) { return __ldcg(reinterpret_cast<const float4*>(a.part + (2 * q + which) * a.ld + c)); };
  const auto sum = [](float4& s, const float4& v) { s = make_float4(s.x + v.x, s.y + v.y, s.z + v.z, s.w + v.w); };
  const auto put = [&](unsigned row, const float4& s) {
    const float v[4] = {s.x, s.y, s.z, s.w};
    put_row<T, 4>(a, row, c, v);
  };
  bool is_long = false;                                 // the group's run is too long for it
  if (group < groups) {
    const long long chunk = base + group, end = (chunk + 1) * a.chunk;
    if (end < a.n) {
      const unsigned row = a.key[end - 1], first = a.key[end - a.chunk], before = chunk > 0 ? a.key[end - a.chunk - 1] : a.table_rows;
      // the first rows of the next chunk and of those 1, 2, 4 ... after it: all asked for at once
      constexpr int LOOKS = 7;
      static_assert(kJoinAlone == 1 << (LOOKS - 2));
      unsigned then[LOOKS];
#pragma unroll
      for (int k = 0; k < LOOKS; ++k) then[k] = a.key[min(end + (long long)(k ? 1 << (k - 1) : 0) * a.chunk, a.n - 1)];
      if (row < a.table_rows && then[0] == row && !(first == row && before == row)) {
        int more = 0;                                   // chunks after the next one that begin with the row: as many as
#pragma unroll
        for (int k = 1; k < LOOKS; ++k) {               // the last look that saw it, or up to twice that
          const int q = 1 << (k - 1);
          if (then[k] == row && end + (long long)q * a.chunk < a.n) more = q;
        }
        is_long = more == kJoinAlone;
        if (!is_long) {
          for (int half = more / 2; half; half /= 2)
            if (has(chunk + 1 + more + half, row)) more += half;
          if (in) {
            float4 s = part(chunk, 1);
#pragma unroll 8
            for (int k = 0; k <= more; ++k) sum(s, part(chunk + 1 + k, 0));
            put(row, s);
          }
        }
      }
    }
    if (lane == 0) long_of[group] = is_long;
  }
  if (!__syncthreads_or(is_long)) return;
  for (int g = 0; g < groups; ++g) {
    if (!long_of[g]) continue;
    const long long chunk = base + g, left = a.chunks - 1 - chunk;    // chunks after the first, some of the run
    const unsigned row = a.key[(chunk + 1) * a.chunk];
    // how many begin with the row: all threads look, first `wide` apart, then at what lies between
    const long long wide = (left + kJoinThreads - 1) / kJoinThreads;
    const long long coarse = chunk + 1 + (__syncthreads_count(has(chunk + 1 + threadIdx.x * wide, row)) - 1) * wide;
    long long count = coarse - chunk - 1;
    for (long long q = 0; q < wide; q += kJoinThreads) count += __syncthreads_count(q + threadIdx.x < wide && has(coarse + q + threadIdx.x, row));
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
    if (in) {
      const long long q1 = chunk + 1 + count * (group + 1) / groups;
#pragma unroll 8
      for (long long q = chunk + 1 + count * group / groups; q < q1; ++q) sum(s, part(q, 0));
    }
    __syncthreads();
    run[threadIdx.x] = s;
    __syncthreads();
    if (group > 0 || !in) continue;
    s = part(chunk, 1);
    for (int h = 0; h < groups; ++h) sum(s, run[h * a.lanes + lane]);
    put(row, s);
  }
}

constexpr long long kMostTile = 16384;  // tokens of a tile at most: they lie in shared memory

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
  // one tile needs no counts; more of them share the SMs, within what a CTA's shared memory holds.  (One tile
  // of 16,384 took 25 us, four of 4,096 and their counts 15.)
  long long per = 4096;
  while (per < kMostTile && tokens > per * kNetSms) per *= 2;
  p.per_tile = (int)per;
  p.tiles = (int)((tokens + per - 1) / per);
  return p;
}

// How a chunk's threads lie over its tokens' columns: V of them each (16 bytes, or one where rows start
// anywhere), and the tokens of a chunk.  A group of threads walks 32 tokens, fewer where the chunks would not
// fill the SMs (of 4 tokens a group at least), and 64 at least go to a CTA of one or two groups, so that
// the parts that the chunks leave stay few.  (100,000 x 1,024 bf16: 220 us with 256 tokens a CTA, 109 so.)
struct Chunks { int lanes, slices, tokens; };
Chunks chunks_of(long long tokens, long long cols, int v) {
  Chunks c;
  c.lanes = lanes_of((cols + v - 1) / v);
  c.slices = (int)((cols + (long long)c.lanes * v - 1) / ((long long)c.lanes * v));
  const int groups = 256 / c.lanes;
  const long long fill = (tokens * c.slices + 2 * kNetSms * groups - 1) / (2LL * kNetSms * groups);
  const int stretch = (int)std::clamp<long long>(fill, 4, 32);
  c.tokens = std::min(kChunk, std::max(stretch * groups, stretch == 32 ? 64 : 1));
  return c;
}

// Chunks that up to `tokens` tokens of up to `cols` columns come in at most: of the tokens that a chunk has
// at least where they fill the SMs, or as many as fill them.
long long most_chunks(long long tokens, long long cols) {
  const int groups = 256 / (int)std::min<long long>(256, cols);
  const long long least = std::min(kChunk, std::max(32 * groups, 64));
  return std::min(tokens, std::max((tokens + least - 1) / least, 2LL * kNetSms + 2));
}

size_t part_ld(long long cols) { return (size_t)(cols + 3) / 4 * 4; }

// The workspace behind its header.
struct EmbedScratch {
  unsigned *key[2], *id[2], *count, *total;
  float* part;
  size_t bytes;
};
EmbedScratch scratch_of(char* base, long long tokens, long long cols) {
  size_t at = kNetHeader;
  const auto take = [&](size_t bytes) { char* q = base ? base + at : nullptr; at += net_align(bytes); return q; };
  EmbedScratch s;
  for (int k = 0; k < 2; ++k) {
    s.key[k] = (unsigned*)take(4 * (size_t)tokens);
    s.id[k] = (unsigned*)take(4 * (size_t)tokens);
  }
  // (tiles of up to as many tokens)
  const long long tiles = std::max(std::min<long long>((tokens + 4095) / 4096, kNetSms), (tokens + kMostTile - 1) / kMostTile);
  s.count = (unsigned*)take((size_t)4 * kMaxDigits * (size_t)tiles);
  s.total = (unsigned*)take((size_t)4 * kMaxDigits);
  s.part = (float*)take((size_t)8 * part_ld(cols) * (size_t)most_chunks(tokens, cols));
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
  *bytes = scratch_of(nullptr, tokens, cols).bytes;
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
  LookupArgs a{table->data, index, add ? add->data : nullptr, y->data, y->rows, table->stride, add ? add->stride : 0, y->stride,
                     (unsigned)table->rows, (unsigned)y->cols, 1, 1, 1, add && rows_aligned(add, 16), index_dtype == ABCD_I64, scale, (unsigned*)ctx->net_base};
  return with_type(y->dtype, [&](auto t) {
    using T = decltype(t);
    constexpr int V = 16 / sizeof(T);
    const bool vec = rows_aligned(y, 16) && rows_aligned(table, 16);
    if (!vec) a.add_vec = 1;                              // one element, wherever it lies
    const long long vectors = vec ? (y->cols + V - 1) / V : y->cols;
    a.lanes = (unsigned)lanes_of(vectors);
    a.slices = (int)((vectors + a.lanes - 1) / a.lanes);
    const long long groups = 256 / a.lanes;
    a.lookup = (int)std::clamp<long long>(y->rows * a.slices / (4LL * ctx->num_sms * groups), 1, kLookup);
    const long long per_cta = groups * a.lookup, grid = (y->rows + per_cta - 1) / per_cta * a.slices;
    auto* kernel = vec ? (add ? embed_kernel<T, V, true> : embed_kernel<T, V, false>) : (add ? embed_kernel<T, 1, true> : embed_kernel<T, 1, false>);
    return check_launch(ctx, "embed_kernel", launch_pdl(kernel, dim3((unsigned)grid), dim3(256), 0, ctx->stream, a));
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
  const EmbedScratch s = scratch_of(ctx->net_base, n, dy->cols);
  if (!ctx->net_base || s.bytes > ctx->net_bytes)
    return fail(ctx, ABCD_ERR_WORKSPACE, "%s: the network workspace has %zu bytes, needs %zu", what, ctx->net_bytes, s.bytes);
  const SortPlan p = sort_plan(n, dtable->rows);
  const size_t smem = 8 * (size_t)p.per_tile + (size_t)kSortWarps * 2 * ((size_t)1 << p.bits);
  auto* place = p.per_tile == 4096 ? sort_place_kernel<4> : p.per_tile == 8192 ? sort_place_kernel<8> : sort_place_kernel<16>;
  const cudaError_t room = allow_smem(ctx, (const void*)place);
  if (room != cudaSuccess) return fail(ctx, ABCD_ERR_CUDA, "%s: %s", what, cudaGetErrorString(room));
  const long long e = (long long)elem_size(dtable->dtype);
  const bool flat = dtable->stride == dtable->cols;
  SortArgs q{index, nullptr, nullptr, s.key[0], s.id[0], s.count, s.total, n, p.tiles, p.per_tile, 0, p.bits,
             index_dtype == ABCD_I64, (unsigned)dtable->rows, (unsigned*)ctx->net_base, (char*)dtable->data,
             flat ? 1 : dtable->rows, (flat ? dtable->rows : 1) * dtable->cols * e, dtable->stride * e};
  // CTAs that clear the gradient beside the first kernel's own
  const long long clear = std::min<long long>((dtable->rows * dtable->cols * e + 65535) / 65536, 2LL * ctx->num_sms);
  const auto sort = [&](const char* name, auto* kernel, long long grid, int threads, size_t bytes) {
    return check_launch(ctx, name, launch_pdl(kernel, dim3((unsigned)grid), dim3((unsigned)threads), bytes, ctx->stream, q));
  };
  if (n == 0) return sort("sort_count_kernel", sort_count_kernel, clear, kSortThreads, 0);
  for (int pass = 0; pass < p.passes; ++pass) {
    q.shift = pass * p.bits;
    const long long more = pass == 0 ? clear : 0;
    abcd_status st = ABCD_OK;
    if (p.tiles > 1) {
      st = sort("sort_count_kernel", sort_count_kernel, p.tiles + more, kSortThreads, 0);
      if (st == ABCD_OK && p.tiles > kScanned) st = sort("sort_scan_kernel", sort_scan_kernel, ((1 << p.bits) + 7) / 8, 256, 0);
    }
    if (st == ABCD_OK) st = sort("sort_place_kernel", place, p.tiles + (p.tiles > 1 ? 0 : more), kSortThreads, smem);
    if (st != ABCD_OK) return st;
    q.key = q.to_key;
    q.id = q.to_id;
    q.to_key = s.key[(pass + 1) & 1];
    q.to_id = s.id[(pass + 1) & 1];
  }
  const bool vec = rows_aligned(dy, 16);
  const Chunks c = chunks_of(n, dy->cols, vec ? 16 / (int)e : 1);
  SumArgs a{dy->data, q.key, q.id, dtable->data, s.part, n, dy->stride, dtable->stride, (unsigned)dtable->rows,
            (unsigned)dy->cols, (unsigned)part_ld(dy->cols), scale, c.lanes, c.slices, c.tokens, rows_aligned(dtable, 16), (n + c.tokens - 1) / c.tokens};
  return with_type(dy->dtype, [&](auto t) {
    using T = decltype(t);
    const auto sum = [&](auto width) {
      constexpr int V = decltype(width)::value;
      const abcd_status st = check_launch(ctx, "embed_sum_kernel", launch_pdl(embed_sum_kernel<T, V>, dim3((unsigned)(a.chunks * a.slices)), dim3(256), 0, ctx->stream, a));
      if (st != ABCD_OK || a.chunks == 1) return st;
      a.lanes = (int)std::min<unsigned>(kJoinLanes, a.ld / 4);
      const long long groups = kJoinThreads / a.lanes;
      a.slices = (int)((a.ld / 4 + a.lanes - 1) / a.lanes);
      const dim3 grid((unsigned)((a.chunks + groups - 1) / groups * a.slices));
      return check_launch(ctx, "embed_join_kernel", launch_pdl(embed_join_kernel<T>, grid, dim3(kJoinThreads), 0, ctx->stream, a));
    };
    return vec ? sum(std::integral_constant<int, 16 / sizeof(T)>()) : sum(std::integral_constant<int, 1>());
  });
}
