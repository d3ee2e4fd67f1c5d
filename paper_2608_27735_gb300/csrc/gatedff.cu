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
// 32-bit matrices keep 24 bits of each.  The kernel is in ffproduct.cuh, its launches in products.cu.
#include "packed8.cuh"
#include "products.cuh"

namespace abcd {
namespace {

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
      hid.g[0] = stored_in_place(gate);
      hid.g[1] = stored_in_place(up);
    }
    hid.out[0] = out_of(gate);
    hid.out[1] = out_of(up);
  }
  if ((st = run(ctx, t, kUp, &up_job, 1, plan(ctx->num_sms, t, kUp, &up_job, 1), &hid)) != ABCD_OK) return st;
  const Job y_job{h, {od}, 1, false, false, m, d, f, 1, {out_of(y)}};
  return run(ctx, t, kPlain, &y_job, 1, plan(ctx->num_sms, t, kPlain, &y_job, 1));
}

namespace abcd {
namespace {

// What the backward pass reads of the forward pass: a matrix, or one in 8 bits.
struct Saved {
  const abcd_matrix* full;
  const abcd_packed8* packed;
  bool ok() const { return full ? matrix_ok(full) : packed_ok(packed); }
  long long rows() const { return full ? full->rows : packed->rows; }
  long long cols() const { return full ? full->cols : packed->cols; }
  bool is(int dtype, long long rows, long long cols) const {
    return full ? shape_is(full, dtype, rows, cols) : packed_ok(packed) && packed->rows == rows && packed->cols == cols;
  }
  bool moved() const { return packed || needs_pack(full); }
  bool touched(std::initializer_list<const abcd_matrix*> results) const {
    return packed && std::any_of(results.begin(), results.end(), [&](const abcd_matrix* m) { return m && touches(packed, m); });
  }
};

abcd_status ff_backward(abcd_ctx* ctx, const char* what, const abcd_matrix* dy, const Saved& x, const abcd_matrix* w_gate,
                        const abcd_matrix* w_up, const abcd_matrix* w_down, int activation, const Saved& gate, const Saved& up,
                        const abcd_matrix* dx, const abcd_matrix* dw_gate, const abcd_matrix* dw_up, const abcd_matrix* dw_down) {
  if (!ctx) return ABCD_ERR_INVALID_ARG;
  if (!matrix_ok(dy) || !x.ok() || !matrix_ok(w_gate)) return fail(ctx, ABCD_ERR_INVALID_ARG, "%s: bad dy, x or w_gate", what);
  const long long m = x.rows(), d = x.cols(), f = w_gate->rows;
  const int t = dy->dtype;
  if (f < 1 || f > kMaxNetCols || !shape_is(w_gate, t, f, d) || !shape_is(w_up, t, f, d) || !shape_is(w_down, t, d, f))
    return fail(ctx, ABCD_ERR_INVALID_ARG, "%s: the weights do not fit x", what);
  if (!shape_is(dy, t, m, d) || !x.is(t, m, d) || !gate.is(t, m, f) || !up.is(t, m, f))
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
  if (same_place({dx, dw_gate, dw_up, dw_down}, {dy, x.full, w_gate, w_up, w_down, gate.full, up.full}) ||
      x.touched({dx, dw_gate, dw_up, dw_down}) || gate.touched({dx, dw_gate, dw_up, dw_down}) || up.touched({dx, dw_gate, dw_up, dw_down}))
    return fail(ctx, ABCD_ERR_INVALID_ARG, "%s: a gradient overlaps an operand or another gradient", what);
  Scratch need{nullptr};
  need.take(kPartBytes);
  if (needs_pack(dy)) need.operand(m, d, t);
  if (x.moved()) need.operand(m, d, x.packed && t == ABCD_F32 ? ABCD_BF16 : t);
  if (needs_pack(w_gate)) need.operand(f, d, t);
  if (needs_pack(w_up)) need.operand(f, d, t);
  if (needs_pack(w_down)) need.operand(d, f, t);
  const bool apart = t != ABCD_F32;                // gate and up are read as they are in 32 bits
  const Job shape_of{Operand{}, {Operand{}}, 1, false, true, m, f, d, 1, {}};
  const Plan down_plan = plan(ctx->num_sms, t, kDown, &shape_of, 1);
  // the large tile of 16-bit matrices takes 8-bit ones as they are
  const bool direct = apart && gate.packed && up.packed && down_plan.shape == 0;
  if (apart && !direct && gate.moved()) need.operand(m, f, t);
  if (apart && !direct && up.moved()) need.operand(m, f, t);
  if (!apart && gate.packed) need.take(2 * net_align((size_t)m * (size_t)pitch_of(f) * 4));
  need.operand(m, f, t);
  need.operand(m, f, t, 2);
  abcd_status st = room(ctx, what, need.at);
  if (st != ABCD_OK) return st;
  Scratch s{ctx->net_base};
  s.take(kPartBytes);
  Operands in{s};
  const Operand ody = in.add(dy), od = in.add(w_down);
  Operand ox{}, og{}, ou{}, ogate{}, oup{};
  Unpacked list[3];
  int unpacked = 0;
  // a saved matrix as an operand: one of 8 bits is unpacked to one, whose values are one 16-bit term
  const auto operand = [&](const Saved& q, int type) {
    if (q.full) return in.add(q.full);
    const Operand o = s.operand(m, q.cols(), type);
    list[unpacked++] = Unpacked{q.packed, const_cast<void*>(o.p), o.pitch, type};
    return o;
  };
  Out wide[2]{};                                   // gate and up in 32 bits
  Hidden hid{};
  if (direct) {
    hid.packed[0] = gate.packed;
    hid.packed[1] = up.packed;
  } else if (apart) {
    ogate = operand(gate, t);
    oup = operand(up, t);
  } else {
    const Saved* const both[2] = {&gate, &up};
    for (int k = 0; k < 2; ++k) {
      if (both[k]->full) {
        wide[k] = out_of(both[k]->full);
      } else {
        wide[k] = Out{s.take(net_align((size_t)m * (size_t)pitch_of(f) * 4)), pitch_of(f), 0, 1};
        list[unpacked++] = Unpacked{both[k]->packed, wide[k].p, wide[k].stride, ABCD_F32};
      }
    }
  }
  if (dw_gate || dw_up) ox = operand(x, x.packed && t == ABCD_F32 ? ABCD_BF16 : t);
  if (dx) {
    og = in.add(w_gate);
    ou = in.add(w_up);
  }
  if ((st = in.pack(ctx, t)) != ABCD_OK) return st;
  if (unpacked && (st = unpack(ctx, list, unpacked)) != ABCD_OK) return st;
  const Operand h = s.operand(m, f, t), dgu = s.operand(m, f, t, 2);
  const Job down{ody, {od}, 1, false, true, m, f, d, 1, {out_of(h, 0, t)}};
  hid.act = activation;
  hid.c = h;
  hid.g[0] = dgu;
  hid.in[0] = ogate;
  hid.in[1] = oup;
  hid.out[0] = out_of(dgu, 0, t);
  hid.out[1] = out_of(dgu, 1, t);
  hid.saved[0] = apart ? out_of(ogate, 0, t) : wide[0];   // (of direct ones nothing: the codes' maps say it)
  hid.saved[1] = apart ? out_of(oup, 0, t) : wide[1];
  if ((st = run(ctx, t, direct ? kDown8 : kDown, &down, 1, down_plan, &hid)) != ABCD_OK) return st;
  // what is left does not depend on one another: one launch, planned as for all of it, so that no
  // gradient depends on which others are asked for
  const Job all[kMaxJobs] = {Job{dgu, {og, ou}, 2, false, true, m, d, f, 1, {}},
                             Job{dgu, {ox}, 1, true, true, f, d, m, 2, {}, x.packed ? 1 : 0},      // dG^T x, dU^T x
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

}  // namespace
}  // namespace abcd

extern "C" abcd_status abcd_gated_ff_backward(abcd_ctx* ctx, const abcd_matrix* dy,
                                              const abcd_matrix* x, const abcd_matrix* w_gate,
                                              const abcd_matrix* w_up, const abcd_matrix* w_down,
                                              int activation, const abcd_matrix* gate,
                                              const abcd_matrix* up, const abcd_matrix* dx,
                                              const abcd_matrix* dw_gate, const abcd_matrix* dw_up,
                                              const abcd_matrix* dw_down) {
  return ff_backward(ctx, "abcd_gated_ff_backward", dy, Saved{x, nullptr}, w_gate, w_up, w_down, activation, Saved{gate, nullptr},
                     Saved{up, nullptr}, dx, dw_gate, dw_up, dw_down);
}

extern "C" abcd_status abcd_gated_ff_backward_packed8(abcd_ctx* ctx, const abcd_matrix* dy, const abcd_packed8* x,
                                                      const abcd_matrix* w_gate, const abcd_matrix* w_up,
                                                      const abcd_matrix* w_down, int activation, const abcd_packed8* gate,
                                                      const abcd_packed8* up, const abcd_matrix* dx, const abcd_matrix* dw_gate,
                                                      const abcd_matrix* dw_up, const abcd_matrix* dw_down) {
  return ff_backward(ctx, "abcd_gated_ff_backward_packed8", dy, Saved{nullptr, x}, w_gate, w_up, w_down, activation,
                     Saved{nullptr, gate}, Saved{nullptr, up}, dx, dw_gate, dw_up, dw_down);
}

extern "C" abcd_status abcd_packed8_workspace_size(long long rows, long long cols, long long ff, int dtype, size_t* bytes) {
  if (!bytes || rows < 0 || rows > kMaxNetRows || cols < 1 || cols > kMaxNetCols || ff < 1 || ff > kMaxNetCols || !dtype_ok(dtype))
    return ABCD_ERR_INVALID_ARG;
  Scratch s{nullptr, ff_scratch(rows, cols, ff, dtype)};
  if (dtype == ABCD_F32) s.take(2 * net_align((size_t)rows * (size_t)pitch_of(ff) * 4));   // gate, up
  *bytes = s.at;
  return ABCD_OK;
}
