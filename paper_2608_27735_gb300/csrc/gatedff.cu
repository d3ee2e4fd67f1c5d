// Gated feed-forward layer, forward and backward:
//   G = x Wg^T, U = x Wu^T, H = act(G) U, y = H Wd^T
//   dH = dy Wd, dU = dH act(G), dG = dH U act'(G), dx = dG Wg + dU Wu,
//   dWg = dG^T x, dWu = dU^T x, dWd = dy^T H.
// Four launches of products: both projections with the activation and H; y; dH with dG, dU and H again
// (from the saved G and U, so that H need not be kept from the forward pass); dx (one sum over both
// weights) with dWg, dWu and dWd.
// What goes to memory between them (H, dG, dU; G and U for the caller) is rounded once to the matrices'
// type, which is what the next product's operands are.  In bf16 the result's own rounding leaves 1.7e-3 of
// its norm, H's makes that 2.4e-3 for y, and H's (or dG's and dU's) with G's and U's 3.5e-3 for the
// gradients.  As two 16-bit terms each they would double the products that read them, and G and U in 32
// bits take a fifth of the time of 100,000 x 256 x 1,024 more (820 MB); in fp16 the range is the type's too.
// 32-bit matrices keep 24 bits of each.  The kernel is in ffproduct.cuh; this file is the host's side:
// operands, tensor maps, the choice of tiles and splits, the workspace.
#include <algorithm>
#include <cmath>
#include <initializer_list>

#include "ffproduct.cuh"

namespace abcd {
namespace {

constexpr size_t kPartBytes = 2 * (size_t)kNetSms * 128 * 256 * 4;   // two large tiles' sums per SM

// A 16-bit operand of a product in device memory: planes of rows of cols values.
struct Operand {
  const void* p;
  long long rows, cols, pitch, plane;
  int planes;
};

int terms_of(int dtype) { return dtype == ABCD_F32 ? 3 : 1; }
long long pitch_of(long long cols) { return (cols + 63) / 64 * 64; }   // whole 128-byte lines

// Up to seven matrices that are laid out as operands by one launch.
struct PackArgs {
  struct One {
    const void* src;
    unsigned short* dst;
    long long rows, cols, stride, pitch, plane;
    long long first;                  // blocks of eight columns before this matrix's
  } m[7];
  int n;
  long long blocks;
};

// An operand from a matrix that TMA cannot read as it is: 32-bit values as three 16-bit terms, or
// 16-bit rows moved to 16-byte boundaries.  One thread per eight columns of a row.
template <typename T>
__global__ void __launch_bounds__(256) pack_kernel(const __grid_constant__ PackArgs a) {
  pdl_wait();
  for (long long i = blockIdx.x * 256LL + threadIdx.x; i < a.blocks; i += gridDim.x * 256LL) {
    int k = 0;
#pragma unroll
    for (int q = 1; q < 7; ++q) k += q < a.n && i >= a.m[q].first;
    const PackArgs::One& o = a.m[k];
    const long long groups = (o.cols + 7) / 8, at = i - o.first;
    const long long row = at < (1LL << 32) ? (unsigned)at / (unsigned)groups : at / groups;
    const int col = (int)(8 * (at - row * groups)), left = (int)(o.cols - col);
    const T* src = (const T*)o.src + row * o.stride + col;
    unsigned short* dst = o.dst + row * o.pitch + col;
    if constexpr (sizeof(T) == 4) {
      float v[8];
      if (left >= 8 && ((uintptr_t)src & 15) == 0) {
        const float4 lo = reinterpret_cast<const float4*>(src)[0], hi = reinterpret_cast<const float4*>(src)[1];
        v[0] = lo.x; v[1] = lo.y; v[2] = lo.z; v[3] = lo.w;
        v[4] = hi.x; v[5] = hi.y; v[6] = hi.z; v[7] = hi.w;
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = j < left ? src[j] : 0.f;
      }
#pragma unroll
      for (int t = 0; t < 3; ++t) {
        unsigned w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = take_terms(v[2 * j], v[2 * j + 1]);
        *reinterpret_cast<uint4*>(dst + t * o.plane) = make_uint4(w[0], w[1], w[2], w[3]);
      }
    } else {
      unsigned w[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const unsigned lo = 2 * j < left ? reinterpret_cast<const unsigned short*>(src)[2 * j] : 0u;
        const unsigned hi = 2 * j + 1 < left ? reinterpret_cast<const unsigned short*>(src)[2 * j + 1] : 0u;
        w[j] = lo | hi << 16;
      }
      *reinterpret_cast<uint4*>(dst) = make_uint4(w[0], w[1], w[2], w[3]);
    }
  }
}

// The results of products whose k was split: their parts added in their order, rounded to the type of
// the matrices; up to four results a launch.  A thread takes four columns of a row and a run of
// consecutive parts; where the parts are many, a CTA's threads share them in two to eight runs, which
// are added in their order.
struct JoinArgs {
  struct One {
    const float* part;
    long long ld, plane;              // elements between rows, between splits
    int rows, cols, splits, runs;
    Out c;
  } r[4];
};
template <typename T>
__global__ void __launch_bounds__(256) join_kernel(const __grid_constant__ JoinArgs a) {
  pdl_wait();
  __shared__ float4 run[256];
  const JoinArgs::One& q = a.r[blockIdx.y];
  const int lanes = 256 / q.runs, lane = threadIdx.x % lanes, w = threadIdx.x / lanes;
  const unsigned groups = (q.cols + 3) / 4;
  if (blockIdx.x * lanes >= groups * q.rows) return;
  const unsigned i = blockIdx.x * lanes + lane, row = i / groups, col = 4 * (i - row * groups);
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
  if (row < (unsigned)q.rows) {
    const float* p = q.part + row * q.ld + col;
    const int k1 = q.splits * (w + 1) / q.runs;
#pragma unroll 4
    for (int k = q.splits * w / q.runs; k < k1; ++k) {
      const float4 v = __ldcg(reinterpret_cast<const float4*>(p + k * q.plane));
      s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
    }
  }
  if (q.runs > 1) {
    run[threadIdx.x] = s;
    __syncthreads();
    if (w) return;
    for (int k = 1; k < q.runs; ++k) {
      const float4 v = run[k * lanes + lane];
      s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
    }
  }
  if (row >= (unsigned)q.rows) return;
  T* c = (T*)q.c.p + row * q.c.stride + col;
  if (q.c.vec && (int)col + 4 <= q.cols) {
    Pack<T, 4> v;
    v.v[0] = from_f32<T>(s.x); v.v[1] = from_f32<T>(s.y); v.v[2] = from_f32<T>(s.z); v.v[3] = from_f32<T>(s.w);
    *reinterpret_cast<Pack<T, 4>*>(c) = v;
  } else {
    const float v[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if ((int)col + e < q.cols) c[e] = from_f32<T>(v[e]);
  }
}

// Hands out the network workspace after its header; without a base it only counts.
struct Scratch {
  char* base;
  size_t at = kNetHeader;
  void* take(size_t bytes) {
    char* p = base ? base + at : nullptr;
    at += net_align(bytes);
    return p;
  }
  Operand operand(long long rows, long long cols, int dtype, int matrices = 1) {
    Operand o{nullptr, rows, cols, pitch_of(cols), 0, matrices * terms_of(dtype)};
    o.plane = rows * o.pitch;
    o.p = take((size_t)o.planes * (size_t)o.plane * 2);
    return o;
  }
};

bool needs_pack(const abcd_matrix* m) { return m->dtype == ABCD_F32 || !rows_aligned(m, 16); }

Operand in_place(const abcd_matrix* m) {
  return Operand{m->data, m->rows, m->cols, (m->stride + 7) / 8 * 8, 0, 1};
}

// The matrices of a call as operands: in place where TMA can read them, else as copies in the
// workspace, which one launch makes.
struct Operands {
  Scratch& s;
  PackArgs args{};
  Operand add(const abcd_matrix* m) {
    if (!needs_pack(m)) return in_place(m);
    const Operand o = s.operand(m->rows, m->cols, m->dtype);
    args.m[args.n++] = PackArgs::One{m->data, (unsigned short*)o.p, m->rows, m->cols, m->stride, o.pitch, o.plane, args.blocks};
    args.blocks += (m->cols + 7) / 8 * m->rows;
    return o;
  }
  abcd_status pack(abcd_ctx* ctx, int dtype) const {
    if (args.n == 0) return ABCD_OK;
    const long long grid = std::min<long long>((args.blocks + 255) / 256, 16LL * ctx->num_sms);
    return check_launch(ctx, "pack_kernel", launch_pdl(dtype == ABCD_F32 ? pack_kernel<float> : pack_kernel<unsigned short>,
                                                       dim3((unsigned)grid), dim3(256), 0, ctx->stream, args));
  }
};

using EncodeFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                              const cuuint64_t*, const cuuint32_t*, const cuuint32_t*,
                              CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion,
                              CUtensorMapFloatOOBfill);

EncodeFn encode_fn() {
  static const EncodeFn fn = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult r;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &r) != cudaSuccess ||
        r != cudaDriverEntryPointSuccess)
      p = nullptr;
    return (EncodeFn)p;
  }();
  return fn;
}

// The tensor map of an operand with boxes of 64 (or 32) consecutive columns and `box_rows` rows, their
// rows' 128 (64) bytes swizzled; what lies outside the matrix reads as zero.
bool make_map(CUtensorMap* map, const Operand& o, int dtype, int box_rows, int box_cols = 64) {
  const EncodeFn fn = encode_fn();
  if (!fn) return false;
  const cuuint64_t dims[3] = {(cuuint64_t)o.cols, (cuuint64_t)o.rows, (cuuint64_t)o.planes};
  const cuuint64_t strides[2] = {(cuuint64_t)o.pitch * 2, (cuuint64_t)std::max<long long>(o.plane, o.pitch) * 2};
  const cuuint32_t box[3] = {(cuuint32_t)box_cols, (cuuint32_t)box_rows, 1}, unit[3] = {1, 1, 1};
  return fn(map, dtype == ABCD_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3,
            const_cast<void*>(o.p), dims, strides, box, unit, CU_TENSOR_MAP_INTERLEAVE_NONE,
            box_cols == 64 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

Out out_of(const abcd_matrix* m) {
  return Out{m->data, m->stride, 0, rows_aligned(m, 16) ? 1 : 0};
}
Out out_of(const Operand& o, int matrix, int dtype) {
  return Out{(unsigned short*)const_cast<void*>(o.p) + matrix * terms_of(dtype) * o.plane, o.pitch, o.plane, 1};
}

// One product: A and up to two B operands (the sum of both products, or gate and up), and its results.
struct Job {
  Operand a, b[2];
  int nb;
  bool a_rows_last, b_rows_last;   // the operand lies with its own dimension contiguous instead of k
  long long m, n, k;
  int batches;
  Out c[2];
};
// What the epilogues of kUp and kDown read and write besides.
struct Hidden {
  int act;
  Operand c, g[2], in[2];          // as operands where TMA moves them
  Out out[2], saved[2];            // the same as g and in
};

int segments_of(const Job& j, int epi, int dtype) {
  return (epi == kUp ? 1 : j.nb) * (dtype == ABCD_F32 ? 6 : 1);
}

// Picks the shape and each product's splits with the least estimated time.  The items (tiles, or parts
// of them) cost their stages or, beside the next item's stages, their epilogue; they are dealt out to
// the CTAs in turn, so that the last wave is partly idle.  Splits bring the products' items near one
// size: the whole work's share of a CTA, or a part of it.  Their joining writes and reads the sums
// through L2.
struct Plan {
  int shape, splits[kMaxJobs];
};
Plan plan(int sms, int dtype, int epi, const Job* jobs, int n) {
  Plan found{0, {1, 1, 1}};
  sms = std::min(sms, kNetSms);
  const bool f32 = dtype == ABCD_F32;
  double best = 1e300;
  for (int s = 0; s < 3; ++s) {
    const Shape& q = kShapes[s];
    const long long units = (epi == kDown ? 1 : q.ctas) * sms / q.cg, cols = epi == kUp ? q.bn / 2 : q.bn;
    const double tile_bytes = 4.0 * 128 * q.cg * q.bn, epilogue = q.epilogue[epi][f32];
    long long tiles[kMaxJobs], kblocks[kMaxJobs];
    double work = 0;                                     // stages of all tiles
    long long whole = 0;                                 // items without splits
    for (int k = 0; k < n; ++k) {
      tiles[k] = jobs[k].batches * ((jobs[k].m + 128 * q.cg - 1) / (128 * q.cg)) * ((jobs[k].n + cols - 1) / cols);
      kblocks[k] = (jobs[k].k + kBlockK - 1) / kBlockK;
      work += (double)tiles[k] * (double)kblocks[k] * segments_of(jobs[k], epi, dtype);
    }
    for (const int waves : {0, 1, 2, 3, 4, 6, 8, 12, 16, 24, 32}) {   // 0: no splits
      double room = (double)kPartBytes, joined = 0, total = 0, longest = 0, items = 0;
      int p[kMaxJobs];
      for (int k = 0; k < n; ++k) {
        const double stages = (double)kblocks[k] * segments_of(jobs[k], epi, dtype);
        double want = waves == 0 ? 1 : stages / std::max(1.0, work / (double)(units * waves));
        // where the last part's warps add the parts up, all parts of a tile run at once; the large
        // tile's blocks of results are whole sums
        double most = epi == kPlain ? room / ((double)tiles[k] * tile_bytes) : s == 0 && !f32 ? 1 : (double)units / (double)tiles[k];
        most = std::min({most, (double)kblocks[k], 64.0});
        p[k] = std::max(1, (int)std::min(std::ceil(want - 0.05), std::floor(most)));
        if (p[k] > 1) {
          room -= (double)tiles[k] * p[k] * tile_bytes;
          joined += (double)tiles[k] * p[k] * tile_bytes / 4e6;
        }
        items += (double)tiles[k] * p[k];
      }
      if (waves > 0 && items == (double)whole) break;     // no splits again, nor with more waves
      if (waves == 0) whole = (long long)items;
      // a launch more, or the last warps' reading of part after part
      if (joined > 0) joined += epi == kPlain ? 2.5 : 1.5 + 0.4 * p[0];
      const double busy = std::min(1.0, items / (double)units), stage = q.idle + (q.busy - q.idle) * busy;
      double stages_last = 0;
      for (int k = 0; k < n; ++k) {
        const double stages = (double)((kblocks[k] + p[k] - 1) / p[k]) * segments_of(jobs[k], epi, dtype) * stage;
        const double cost = std::max(stages, epilogue);
        total += cost * (double)tiles[k] * p[k];
        longest = std::max(longest, cost);
        stages_last = std::max(stages_last, std::min(stages, epilogue));
      }
      // one product: whole waves; several: the last wave is filled to half on average
      double t = n == 1 ? longest * std::ceil(items / (double)units) : std::max(longest, total / (double)units + 0.5 * longest);
      t += q.fixed + stages_last + joined;
      if (t < best) {
        best = t;
        found.shape = s;
        for (int k = 0; k < n; ++k) found.splits[k] = p[k];
      }
    }
  }
  return found;
}

// Launches the products (and what joins their splits).
abcd_status run(abcd_ctx* ctx, int dtype, int epi, const Job* jobs, int n, const Plan& planned, const Hidden* hidden = nullptr) {
  ProductArgs a{};
  const int terms = terms_of(dtype);
  const int shape = planned.shape;
  const int* splits = planned.splits;
  const int cg = kShapes[shape].cg, bn = kShapes[shape].bn, cols = epi == kUp ? bn / 2 : bn;
  a.jobs = n;
  a.dtype = dtype;
  a.count = (unsigned*)(ctx->net_base + kNetCounters);
  a.status = (unsigned*)ctx->net_base;
  a.limit = ctx->wait_limit;
  float* part = (float*)(ctx->net_base + kNetHeader);
  JoinArgs join{};
  int results = 0;
  long long join_ctas = 0;
  bool ok = true;
  // the products of the longest items first: the short ones level the last wave
  int order_of[kMaxJobs] = {0, 1, 2};
  const auto length = [&](int k) { return (double)jobs[k].k * segments_of(jobs[k], epi, dtype) / splits[k]; };
  std::sort(order_of, order_of + n, [&](int x, int y) { return length(x) != length(y) ? length(x) > length(y) : x < y; });
  for (int slot = 0; slot < n; ++slot) {
    const int q = order_of[slot];
    const Job& j = jobs[q];
    ProductJob& o = a.job[slot];
    o.a_rows_last = j.a_rows_last;
    o.b_rows_last = j.b_rows_last;
    o.m = (int)j.m;
    o.n = (int)j.n;
    o.kblocks = (int)((j.k + kBlockK - 1) / kBlockK);
    // pairs of terms, the smallest products first
    for (int order = terms - 1; order >= 0; --order)
      for (int b = 0; b < (epi == kUp ? 1 : j.nb); ++b)
        for (int t = order; t >= 0; --t) {
          o.az[o.segments] = (unsigned char)(b * terms + t);
          o.bsel[o.segments] = (unsigned char)b;
          o.bz[o.segments++] = (unsigned char)(order - t);
        }
    o.batch_az = terms;
    o.batches = j.batches;
    o.tiles_m = (int)((j.m + 128 * cg - 1) / (128 * cg));
    o.tiles_n = (int)((j.n + cols - 1) / cols);
    o.splits = splits[q];
    o.first = a.items;
    a.items += o.batches * o.tiles_m * o.tiles_n * o.splits;
    o.c[0] = j.c[0];
    o.c[1] = j.c[1];
    o.part = part;
    o.part_ld = (j.n + 3) / 4 * 4;
    ok = ok && make_map(&o.a, j.a, dtype, j.a_rows_last ? 64 : 128);
    for (int b = 0; ok && b < j.nb; ++b) ok = make_map(&o.b[b], j.b[b], dtype, j.b_rows_last ? 64 : epi == kUp ? bn / 2 : bn / cg);
    if (j.nb < 2) o.b[1] = o.b[0];
    if (epi != kPlain || splits[q] == 1) continue;
    const long long plane = j.batches * j.m * o.part_ld;
    for (int b = 0; b < j.batches; ++b) {
      const int runs = splits[q] <= 8 ? 1 : splits[q] <= 16 ? 2 : splits[q] <= 32 ? 4 : 8, lanes = 256 / runs;
      join.r[results++] = JoinArgs::One{part + b * j.m * o.part_ld, o.part_ld, plane, (int)j.m, (int)j.n, splits[q], runs, j.c[b]};
      join_ctas = std::max(join_ctas, (j.m * ((j.n + 3) / 4) + lanes - 1) / lanes);
    }
    part += plane * splits[q];
  }
  if (hidden) {
    a.act = hidden->act;
    for (int k = 0; k < 2; ++k) {
      a.g[k] = hidden->out[k];
      a.in[k] = hidden->saved[k];
    }
    if (shape == 0 && dtype != ABCD_F32) {
      ok = ok && make_map(&a.c_map, hidden->c, dtype, 128, 32);
      for (int k = 0; k < 2; ++k) {
        if (ok && hidden->g[k].p) ok = make_map(&a.g_map[k], hidden->g[k], dtype, 128, 32);
        if (ok && hidden->in[k].p) ok = make_map(&a.in_map[k], hidden->in[k], dtype, 128, 32);
      }
    }
  }
  if (!ok) return fail(ctx, ABCD_ERR_CUDA, "tensor map of a product");
  const abcd_status st = dtype == ABCD_F32 ? launch_32(ctx, epi, shape, a) : launch_16(ctx, epi, shape, a);
  if (st != ABCD_OK || results == 0) return st;
  return with_type(dtype, [&](auto t) {
    return check_launch(ctx, "join_kernel", launch_pdl(join_kernel<decltype(t)>, dim3((unsigned)join_ctas, (unsigned)results),
                                                       dim3(256), 0, ctx->stream, join));
  });
}

bool shape_is(const abcd_matrix* m, int dtype, long long rows, long long cols) {
  return matrix_ok(m) && m->dtype == dtype && m->rows == rows && m->cols == cols;
}

// Whether a result overlaps an operand or another result; one that is not given lies nowhere.
bool same_place(std::initializer_list<const abcd_matrix*> results, std::initializer_list<const abcd_matrix*> operands) {
  for (auto r = results.begin(); r != results.end(); ++r) {
    if (!*r) continue;
    const auto at = [&](const abcd_matrix* m) { return m && overlap(m, *r); };
    if (std::any_of(operands.begin(), operands.end(), at) || std::any_of(results.begin(), r, at)) return true;
  }
  return false;
}

// The scratch of the calls when every matrix has to be copied: the most that they take.
size_t ff_scratch(long long rows, long long cols, long long ff, int dtype) {
  Scratch s{nullptr};
  s.take(kPartBytes);
  s.operand(rows, cols, dtype);           // x
  s.operand(rows, cols, dtype);           // dy
  s.operand(ff, cols, dtype);             // w_gate
  s.operand(ff, cols, dtype);             // w_up
  s.operand(cols, ff, dtype);             // w_down
  s.operand(rows, ff, dtype);             // hidden
  s.operand(rows, ff, dtype, 2);          // dG, dU
  for (int k = 0; k < 2 && dtype != ABCD_F32; ++k) s.operand(rows, ff, dtype);   // gate, up (backward)
  return s.at;
}

abcd_status room(abcd_ctx* ctx, const char* what, size_t need) {
  if (need <= ctx->net_bytes) return ABCD_OK;
  return fail(ctx, ABCD_ERR_WORKSPACE, "%s: the network workspace has %zu bytes, needs %zu", what, ctx->net_bytes, need);
}

}  // namespace

int norm_bwd_ctas(int num_sms);   // layernorm.cu
abcd_status few_tokens(abcd_ctx* ctx, const abcd_matrix* x, const abcd_matrix* w_gate, const abcd_matrix* w_up,
                       const abcd_matrix* w_down, int activation, const abcd_matrix* y, const abcd_matrix* gate,
                       const abcd_matrix* up, void* hidden);   // fffew.cu
// Tokens up to which the forward pass goes without tensor cores.
constexpr long long kFewRows = 8;

}  // namespace abcd

using namespace abcd;

extern "C" abcd_status abcd_network_workspace_size(long long rows, long long cols, long long ff,
                                                   int dtype, size_t* bytes) {
  if (!bytes || rows < 0 || rows > kMaxNetRows || cols < 1 || cols > kMaxNetCols || ff < 0 ||
      ff > kMaxNetCols || !dtype_ok(dtype))
    return ABCD_ERR_INVALID_ARG;
  const size_t norm = kNetHeader + (size_t)std::min<long long>(norm_bwd_ctas(kNetSms), rows) * 2 * (size_t)cols * sizeof(float);
  *bytes = ff > 0 ? std::max(norm, ff_scratch(rows, cols, ff, dtype)) : norm;
  return ABCD_OK;
}

extern "C" abcd_status abcd_set_network_workspace(abcd_ctx* ctx, void* ptr, size_t bytes) {
  if (!ctx) return ABCD_ERR_INVALID_ARG;
  if (!ptr || ((uintptr_t)ptr & 255) || bytes < kNetHeader)
    return fail(ctx, ABCD_ERR_INVALID_ARG, "the network workspace must be a 256-byte aligned device pointer to %zu bytes at least", kNetHeader);
  const cudaError_t e = cudaMemsetAsync(ptr, 0, kNetHeader, ctx->stream);
  if (e != cudaSuccess) return fail(ctx, ABCD_ERR_CUDA, "clearing the network workspace: %s", cudaGetErrorString(e));
  ctx->net_base = (char*)ptr;
  ctx->net_bytes = bytes;
  return ABCD_OK;
}

extern "C" abcd_status abcd_gated_ff(abcd_ctx* ctx, const abcd_matrix* x, const abcd_matrix* w_gate,
                                     const abcd_matrix* w_up, const abcd_matrix* w_down,
                                     int activation, const abcd_matrix* y, const abcd_matrix* gate,
                                     const abcd_matrix* up) {
  const char* what = "abcd_gated_ff";
  if (!ctx) return ABCD_ERR_INVALID_ARG;
  if (!matrix_ok(x) || !matrix_ok(w_gate)) return fail(ctx, ABCD_ERR_INVALID_ARG, "%s: bad x or w_gate", what);
  const long long m = x->rows, d = x->cols, f = w_gate->rows;
  const int t = x->dtype;
  if (f < 1 || f > kMaxNetCols || !shape_is(w_gate, t, f, d) || !shape_is(w_up, t, f, d) || !shape_is(w_down, t, d, f))
    return fail(ctx, ABCD_ERR_INVALID_ARG, "%s: the weights do not fit x", what);
  if (!shape_is(y, t, m, d) || (gate == nullptr) != (up == nullptr) ||
      (gate && (!shape_is(gate, t, m, f) || !shape_is(up, t, m, f))))
    return fail(ctx, ABCD_ERR_INVALID_ARG, "%s: the outputs do not fit x and the weights", what);
  if (activation < ABCD_SILU || activation > ABCD_RELU)
    return fail(ctx, ABCD_ERR_INVALID_ARG, "%s: unknown activation", what);
  if (m == 0) return ABCD_OK;
  if (same_place({gate, up}, {x, w_gate, w_up, w_down, y}) || same_place({y}, {w_gate, w_up, w_down}))
    return fail(ctx, ABCD_ERR_INVALID_ARG, "%s: an output overlaps an operand or another output", what);
  Scratch need{nullptr};
  if (m <= kFewRows) {
    need.operand(m, f, ABCD_F32);                  // room for the hidden matrix in any type
    const abcd_status st = room(ctx, what, need.at);
    return st != ABCD_OK ? st : few_tokens(ctx, x, w_gate, w_up, w_down, activation, y, gate, up, ctx->net_base + kNetHeader);
  }
  need.take(kPartBytes);
  if (needs_pack(x)) need.operand(m, d, t);
  if (needs_pack(w_gate)) need.operand(f, d, t);
  if (needs_pack(w_up)) need.operand(f, d, t);
  if (needs_pack(w_down)) need.operand(d, f, t);
  need.operand(m, f, t);
  abcd_status st = room(ctx, what, need.at);
  if (st != ABCD_OK) return st;
  Scratch s{ctx->net_base};
  s.take(kPartBytes);
  Operands in{s};
  const Operand ox = in.add(x), og = in.add(w_gate), ou = in.add(w_up), od = in.add(w_down);
  if ((st = in.pack(ctx, t)) != ABCD_OK) return st;
  const Operand h = s.operand(m, f, t);
  const Job up_job{ox, {og, ou}, 2, false, false, m, f, d, 1, {out_of(h, 0, t)}};
  Hidden hid{};
  hid.act = activation;
  hid.c = h;
  if (gate) {
    // TMA stores them where their rows allow it
    if (!needs_pack(gate) && !needs_pack(up)) {
      hid.g[0] = in_place(gate);
      hid.g[1] = in_place(up);
    }
    hid.out[0] = out_of(gate);
    hid.out[1] = out_of(up);
  }
  if ((st = run(ctx, t, kUp, &up_job, 1, plan(ctx->num_sms, t, kUp, &up_job, 1), &hid)) != ABCD_OK) return st;
  const Job y_job{h, {od}, 1, false, false, m, d, f, 1, {out_of(y)}};
  return run(ctx, t, kPlain, &y_job, 1, plan(ctx->num_sms, t, kPlain, &y_job, 1));
}

extern "C" abcd_status abcd_gated_ff_backward(abcd_ctx* ctx, const abcd_matrix* dy,
                                              const abcd_matrix* x, const abcd_matrix* w_gate,
                                              const abcd_matrix* w_up, const abcd_matrix* w_down,
                                              int activation, const abcd_matrix* gate,
                                              const abcd_matrix* up, const abcd_matrix* dx,
                                              const abcd_matrix* dw_gate, const abcd_matrix* dw_up,
                                              const abcd_matrix* dw_down) {
  const char* what = "abcd_gated_ff_backward";
  if (!ctx) return ABCD_ERR_INVALID_ARG;
  if (!matrix_ok(x) || !matrix_ok(w_gate)) return fail(ctx, ABCD_ERR_INVALID_ARG, "%s: bad x or w_gate", what);
  const long long m = x->rows, d = x->cols, f = w_gate->rows;
  const int t = x->dtype;
  if (f < 1 || f > kMaxNetCols || !shape_is(w_gate, t, f, d) || !shape_is(w_up, t, f, d) || !shape_is(w_down, t, d, f))
    return fail(ctx, ABCD_ERR_INVALID_ARG, "%s: the weights do not fit x", what);
  if (!shape_is(dy, t, m, d) || !shape_is(gate, t, m, f) || !shape_is(up, t, m, f))
    return fail(ctx, ABCD_ERR_INVALID_ARG, "%s: dy, gate or up do not fit x and the weights", what);
  if ((dx && !shape_is(dx, t, m, d)) || (dw_gate && !shape_is(dw_gate, t, f, d)) ||
      (dw_up && !shape_is(dw_up, t, f, d)) || (dw_down && !shape_is(dw_down, t, d, f)))
    return fail(ctx, ABCD_ERR_INVALID_ARG, "%s: the gradients do not fit x and the weights", what);
  if (activation < ABCD_SILU || activation > ABCD_RELU)
    return fail(ctx, ABCD_ERR_INVALID_ARG, "%s: unknown activation", what);
  if (m == 0) {                                   // sums over no rows
    for (const abcd_matrix* w : {dw_gate, dw_up, dw_down}) {
      if (!w) continue;
      const size_t e = elem_size(t);
      const cudaError_t c = cudaMemset2DAsync(w->data, (size_t)w->stride * e, 0, (size_t)w->cols * e, (size_t)w->rows, ctx->stream);
      if (c != cudaSuccess) return fail(ctx, ABCD_ERR_CUDA, "%s: %s", what, cudaGetErrorString(c));
    }
    return ABCD_OK;
  }
  if (same_place({dx, dw_gate, dw_up, dw_down}, {dy, x, w_gate, w_up, w_down, gate, up}))
    return fail(ctx, ABCD_ERR_INVALID_ARG, "%s: a gradient overlaps an operand or another gradient", what);
  Scratch need{nullptr};
  need.take(kPartBytes);
  if (needs_pack(dy)) need.operand(m, d, t);
  if (needs_pack(x)) need.operand(m, d, t);
  if (needs_pack(w_gate)) need.operand(f, d, t);
  if (needs_pack(w_up)) need.operand(f, d, t);
  if (needs_pack(w_down)) need.operand(d, f, t);
  const bool apart = t != ABCD_F32;                // gate and up are read as they are in 32 bits
  if (apart && needs_pack(gate)) need.operand(m, f, t);
  if (apart && needs_pack(up)) need.operand(m, f, t);
  need.operand(m, f, t);
  need.operand(m, f, t, 2);
  abcd_status st = room(ctx, what, need.at);
  if (st != ABCD_OK) return st;
  Scratch s{ctx->net_base};
  s.take(kPartBytes);
  Operands in{s};
  const Operand ody = in.add(dy), od = in.add(w_down);
  Operand ox{}, og{}, ou{}, ogate{}, oup{};
  if (apart) {
    ogate = in.add(gate);
    oup = in.add(up);
  }
  if (dw_gate || dw_up) ox = in.add(x);
  if (dx) {
    og = in.add(w_gate);
    ou = in.add(w_up);
  }
  if ((st = in.pack(ctx, t)) != ABCD_OK) return st;
  const Operand h = s.operand(m, f, t), dgu = s.operand(m, f, t, 2);
  const Job down{ody, {od}, 1, false, true, m, f, d, 1, {out_of(h, 0, t)}};
  Hidden hid{};
  hid.act = activation;
  hid.c = h;
  hid.g[0] = dgu;
  hid.in[0] = ogate;
  hid.in[1] = oup;
  hid.out[0] = out_of(dgu, 0, t);
  hid.out[1] = out_of(dgu, 1, t);
  hid.saved[0] = apart ? out_of(ogate, 0, t) : out_of(gate);
  hid.saved[1] = apart ? out_of(oup, 0, t) : out_of(up);
  if ((st = run(ctx, t, kDown, &down, 1, plan(ctx->num_sms, t, kDown, &down, 1), &hid)) != ABCD_OK) return st;
  // what is left does not depend on one another: one launch, planned as for all of it, so that no
  // gradient depends on which others are asked for
  const Job all[kMaxJobs] = {Job{dgu, {og, ou}, 2, false, true, m, d, f, 1, {}},
                             Job{dgu, {ox}, 1, true, true, f, d, m, 2, {}},      // dG^T x, dU^T x
                             Job{ody, {h}, 1, true, true, d, f, m, 1, {}}};
  const Plan whole = plan(ctx->num_sms, t, kPlain, all, kMaxJobs);
  Plan part{whole.shape, {1, 1, 1}};
  Job jobs[kMaxJobs];
  int n = 0;
  const auto take = [&](int k) -> Job& {
    part.splits[n] = whole.splits[k];
    jobs[n] = all[k];
    return jobs[n++];
  };
  if (dx) take(0).c[0] = out_of(dx);
  if (dw_gate || dw_up) {
    Job& j = take(1);
    j.c[0] = out_of(dw_gate ? dw_gate : dw_up);
    if (dw_gate && dw_up) {
      j.c[1] = out_of(dw_up);
    } else {                                       // one of them: dU's planes are the second half
      if (!dw_gate) j.a.p = (const unsigned short*)dgu.p + (long long)terms_of(t) * dgu.plane;
      j.a.planes = terms_of(t);
      j.batches = 1;
    }
  }
  if (dw_down) take(2).c[0] = out_of(dw_down);
  return n ? run(ctx, t, kPlain, jobs, n, part) : ABCD_OK;
}
