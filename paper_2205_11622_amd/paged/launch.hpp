// What the launches of the attention kernels have in common: the device and stream, how many pieces the
// work is cut into, and the workspace of their partial results.
#pragma once

#include "attend.hpp"
#include "runtime.hpp"
#include "sparselnr.h"

namespace slnr {
namespace paged {

// Pieces that the work is cut into, per compute unit.  Two blocks of attend_few are resident
// on one.  Pieces of a selection are all alike, so they go in one round (32 tokens over 32
// pages of 64: 69 us; at 3 a unit 87, at 4 77); contexts are ragged, and shorter pieces
// even them out (64 of 513 to 15096 keys: 259 us; at 2 a unit 291, at 4 262).  A block of attend_many fills a unit: at 2
// pieces a unit 2 of 2000 tokens behind 7000 738 us (at 1 706), 1 of 512 behind 8000 179 (133), 16 of 64 behind 4000 197
// (134), 64 of 1 to 200 behind up to 4000 417 (418).
constexpr int kFewPerCu = 3;
constexpr int kFewPerCuSparse = 2;
constexpr int kManyPerCu = 1;

struct Launch {
  int dev, cus;
  hipStream_t stream;
};

// A launch has fewer than 2^32 threads a dimension.
constexpr int64_t grid_limit(int block) { return (((int64_t)1 << 32) - 1) / block; }

template <class F>
int launch(F *fn, dim3 grid, int block, size_t lds, const Launch &l, const AttendArgs &a) {
  hipLaunchKernelGGL(fn, grid, dim3(block), lds, l.stream, a);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? SPARSELNR_OK : hip_error(e);
}

// Slots of split tiles that cutting the work into about `target` pieces takes (see split_scan):
// a tile of x caps makes at most x + 1 pieces and, if it is cut, at most 2 x.
constexpr int64_t few_slots(int64_t target) { return 2 * target; }
// With a tail: the work is `target` caps, three tenths of it (and what a tile reaches over) of
// a kTailCuts-th.
constexpr int64_t many_caps(int64_t target) { return target + target * kTailCuts * 3 / 10 + kTailCuts; }
constexpr int64_t many_slots(int64_t target) { return 2 * many_caps(target); }

// Partial results of `slots` pieces of `values` numbers, behind their records.
constexpr size_t records_bytes(int64_t slots) {
  return ((size_t)(1 + slots) * kMeta * sizeof(int32_t) + 255) / 256 * 256;
}
constexpr size_t partials_bytes(int64_t slots, int64_t values) {
  return records_bytes(slots) + (size_t)slots * values * sizeof(float);
}

// The workspace has one size for all calls on a device, the largest need there is (130 MB on 256
// units): a captured graph holds its address, so no later call of other tokens, heads, hint,
// type or dim may be one that has to grow it.
constexpr int64_t kFewValues = kFewRows * (kMaxDim + 2);
constexpr int64_t kManyValues = 256 * (128 + 2);  // eight waves of 32 rows up to 128 columns, four up to 256
inline size_t attend_bytes(int cus) {
  const size_t few = partials_bytes(few_slots((int64_t)cus * kFewPerCu), kFewValues);
  const size_t many = partials_bytes(many_slots((int64_t)cus * kManyPerCu), kManyValues);
  return few > many ? few : many;
}

inline int partials(const Launch &l, int64_t slots, AttendArgs &a, HeldWorkspace *ws) {
  const int rc = hold_workspace(l.dev, l.stream, attend_bytes(l.cus), kSlotAttend, ws);
  if (rc != SPARSELNR_OK) return rc;
  a.meta = (int32_t *)ws->ptr;
  a.part = (float *)((char *)ws->ptr + records_bytes(slots));
  return SPARSELNR_OK;
}

}  // namespace paged
}  // namespace slnr
