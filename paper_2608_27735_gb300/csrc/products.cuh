// The host's side of the matrix products (ffproduct.cuh), for the calls that are made of them (gatedff.cu,
// linear.cu): operands, results, the choice of tiles and splits, the workspace.
#pragma once

#include <algorithm>
#include <initializer_list>

#include "ffproduct.cuh"

namespace abcd {

constexpr size_t kPartBytes = 2 * (size_t)kNetSms * 128 * 256 * 4;   // two large tiles' sums per SM

// A 16-bit operand of a product in device memory: planes of rows of cols values.
struct Operand {
  const void* p;
  long long rows, cols, pitch, plane;
  int planes;
};

inline int terms_of(int dtype) { return dtype == ABCD_F32 ? 3 : 1; }
inline long long pitch_of(long long cols) { return (cols + 63) / 64 * 64; }   // whole 128-byte lines

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

inline bool needs_pack(const abcd_matrix* m) { return m->dtype == ABCD_F32 || !rows_aligned(m, 16); }

inline Operand in_place(const abcd_matrix* m) {
  return Operand{m->data, m->rows, m->cols, (m->stride + 7) / 8 * 8, 0, 1};
}

// A result that TMA stores: the whole 16-byte pieces of its rows.  (It writes the piece that a row ends in to that
// piece's end, over what lies behind the row, so what remains of a row goes by elements.)
inline Operand stored_in_place(const abcd_matrix* m) {
  Operand o = in_place(m);
  o.cols &= ~7LL;
  return o.cols ? o : Operand{};
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
  abcd_status pack(abcd_ctx* ctx, int dtype) const;
};

inline Out out_of(const abcd_matrix* m) {
  return Out{m->data, m->stride, 0, rows_aligned(m, 16) ? 1 : 0};
}
inline Out out_of(const Operand& o, int matrix, int dtype) {
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
  int b_terms;                     // planes of B that are not zero, where fewer than its type's; 0: all
};
// What the epilogues of kUp, kDown and kLinear read and write besides.
struct Hidden {
  int act;
  Operand c, g[2], in[2];          // as operands where TMA moves them
  Out out[2], saved[2];            // the same as g and in; kLinear: z and the residual
  const void* bias;
  int wide_bias;
  const abcd_packed8* packed[2];   // kDown8: gate and up
};

// The shape and the splits of a call's products.
struct Plan {
  int shape, splits[kMaxJobs];
};
Plan plan(int sms, int dtype, int epi, const Job* jobs, int n);
// Launches the products (and what joins their splits).
abcd_status run(abcd_ctx* ctx, int dtype, int epi, const Job* jobs, int n, const Plan& planned, const Hidden* hidden = nullptr);

inline bool shape_is(const abcd_matrix* m, int dtype, long long rows, long long cols) {
  return matrix_ok(m) && m->dtype == dtype && m->rows == rows && m->cols == cols;
}

// Whether a result overlaps an operand or another result; one that is not given lies nowhere.
inline bool same_place(std::initializer_list<const abcd_matrix*> results, std::initializer_list<const abcd_matrix*> operands) {
  for (auto r = results.begin(); r != results.end(); ++r) {
    if (!*r) continue;
    const auto at = [&](const abcd_matrix* m) { return m && overlap(m, *r); };
    if (std::any_of(operands.begin(), operands.end(), at) || std::any_of(results.begin(), r, at)) return true;
  }
  return false;
}

inline abcd_status room(abcd_ctx* ctx, const char* what, size_t need) {
  if (need <= ctx->net_bytes) return ABCD_OK;
  return fail(ctx, ABCD_ERR_WORKSPACE, "%s: the network workspace has %zu bytes, needs %zu", what, ctx->net_bytes, need);
}

}  // namespace abcd
