// Matrices in 8 bits (packed8.cu), as the calls that read them see them.
#pragma once

#include "network.cuh"

namespace abcd {

// A packed matrix that a call may read or write: its shape within the limits, its codes on 32-byte boundaries and
// apart from its powers (which may lie between the rows of codes).
inline bool packed_ok(const abcd_packed8* q) {
  return q && q->rows >= 0 && q->rows <= kMaxNetRows && q->cols >= 1 && q->cols <= kMaxNetCols &&
         q->stride >= q->cols && q->stride <= (1LL << 31) && q->stride % 32 == 0 &&
         q->power_stride >= (q->cols + 31) / 32 && q->power_stride <= (1LL << 31) &&
         (q->rows == 0 || (q->codes && q->powers)) && ((uintptr_t)q->codes & 31) == 0 &&
         !overlap(ByteRows{(uintptr_t)q->codes, q->rows, q->cols, q->stride},
                  ByteRows{(uintptr_t)q->powers, q->rows, (q->cols + 31) / 32, q->power_stride});
}

// Whether a packed matrix and another may share a byte: the codes, or the powers, lie within the other's reach
// (or it within theirs), the gaps between rows counted in.
inline bool touches(const abcd_packed8* q, const abcd_matrix* m) {
  if (q->rows == 0 || m->rows == 0) return false;
  const auto end = [](const void* p, long long rows, long long step, long long width) { return (uintptr_t)p + (uintptr_t)((rows - 1) * step + width); };
  const long long e = (long long)elem_size(m->dtype);
  const uintptr_t first = (uintptr_t)m->data, last = end(m->data, m->rows, m->stride * e, m->cols * e);
  const auto apart = [&](const void* p, long long step, long long width) { return end(p, q->rows, step, width) <= first || last <= (uintptr_t)p; };
  return !apart(q->codes, q->stride, q->cols) || !apart(q->powers, q->power_stride, (q->cols + 31) / 32);
}

// A matrix that unpack() fills: a matrix of the call or an operand in the workspace.
struct Unpacked {
  const abcd_packed8* from;
  void* to;
  long long stride;
  int dtype;
};
// Up to three matrices unpacked, by one launch for each type.
abcd_status unpack(abcd_ctx* ctx, const Unpacked* list, int n);

}  // namespace abcd
