// The host's side of the matrix products: operands laid out, tiles and splits chosen, launches.
#include <algorithm>
#include <cmath>

#include "products.cuh"

namespace abcd {
namespace {

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

// The tensor map of a packed matrix's codes, with boxes of 128 rows of a group's 32 bytes, swizzled.
bool make_code_map(CUtensorMap* map, const abcd_packed8* q) {
  const EncodeFn fn = encode_fn();
  if (!fn) return false;
  const cuuint64_t dims[3] = {(cuuint64_t)q->cols, (cuuint64_t)q->rows, 1}, strides[2] = {(cuuint64_t)q->stride, (cuuint64_t)(q->rows * q->stride)};
  const cuuint32_t box[3] = {32, 128, 1}, unit[3] = {1, 1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, q->codes, dims, strides, box, unit, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_32B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

int segments_of(const Job& j, int epi, int dtype) {
  return (epi == kUp ? 1 : j.nb) * (dtype != ABCD_F32 ? 1 : j.b_terms == 1 ? 3 : 6);
}

}  // namespace

abcd_status Operands::pack(abcd_ctx* ctx, int dtype) const {
  if (args.n == 0) return ABCD_OK;
  const long long grid = std::min<long long>((args.blocks + 255) / 256, 16LL * ctx->num_sms);
  return check_launch(ctx, "pack_kernel", launch_pdl(dtype == ABCD_F32 ? pack_kernel<float> : pack_kernel<unsigned short>,
                                                     dim3((unsigned)grid), dim3(256), 0, ctx->stream, args));
}
// Picks the shape and each product's splits with the least estimated time.  The items (tiles, or parts
// of them) cost their stages or, beside the next item's stages, their epilogue; they are dealt out to
// the CTAs in turn, so that the last wave is partly idle.  Splits bring the products' items near one
// size: the whole work's share of a CTA, or a part of it.  Their joining writes and reads the sums
// through L2.
Plan plan(int sms, int dtype, int epi, const Job* jobs, int n) {
  Plan found{0, {1, 1, 1}};
  sms = std::min(sms, kNetSms);
  const bool f32 = dtype == ABCD_F32;
  double best = 1e300;
  for (int s = 0; s < 3; ++s) {
    const Shape& q = kShapes[s];
    const long long units = (epi == kDown ? 1 : q.ctas) * sms / q.cg, cols = epi == kUp ? q.bn / 2 : q.bn;
    const double tile_bytes = 4.0 * 128 * q.cg * q.bn;
    // the large tile's blocks are left (and its residual's, c[1], filled) element by element where rows start anywhere
    const bool apart = epi == kLinear && s == 0 && !f32 && (!jobs[0].c[0].vec || (jobs[0].c[1].p && !jobs[0].c[1].vec));
    const double epilogue = q.epilogue[epi][f32] * (apart ? 4.0 : 1.0);
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
abcd_status run(abcd_ctx* ctx, int dtype, int epi, const Job* jobs, int n, const Plan& planned, const Hidden* hidden) {
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
          if (j.b_terms && order - t >= j.b_terms) continue;
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
    a.bias = hidden->bias;
    a.wide_bias = hidden->wide_bias;
    for (int k = 0; k < 2; ++k) {
      a.g[k] = hidden->out[k];
      a.in[k] = hidden->saved[k];
    }
    if (shape == 0 && dtype != ABCD_F32) {
      if (hidden->c.p) ok = ok && make_map(&a.c_map, hidden->c, dtype, 128, 32);
      for (int k = 0; k < 2; ++k) {
        if (ok && hidden->g[k].p) ok = make_map(&a.g_map[k], hidden->g[k], dtype, 128, 32);
        if (ok && hidden->in[k].p) ok = make_map(&a.in_map[k], hidden->in[k], dtype, 128, 32);
        if (ok && epi == kDown8) {
          ok = make_code_map(&a.in_map[k], hidden->packed[k]);
          a.power[k] = hidden->packed[k]->powers;
          a.power_stride[k] = hidden->packed[k]->power_stride;
        }
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

}  // namespace abcd
