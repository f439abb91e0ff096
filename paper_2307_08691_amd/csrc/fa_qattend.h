// What the kernels of attention over a cache in 4 or 8 bits (fa_qattend.hip, fa_qattend_wide.hip) share: items and where their results go.
#pragma once
#include "fa_mx.h"

namespace fa {

// Packed rows (query * G + head of the group) row0 .. row0 + rows - 1 of sequence s and key/value head g, against the share [begin, end) of nk keys
struct QItem {
  int s, g, nk, begin, end;
  long tok0;                 // token of packed row 0
  int row0, rows, off, slot;
};
__device__ __forceinline__ long out_row(const QAttendArgs& a, const QItem& it, int r) {  // token * Hq + head of packed row r of the item
  const int row = it.row0 + r, q = row / a.G;
  return (it.tok0 + q) * a.Hq + it.g * a.G + (row - q * a.G);
}
__device__ __forceinline__ float* lse_at(const QAttendArgs& a, long at) {  // of out_row's row
  const long tok = at / a.Hq, s = tok / a.Nq;
  return a.LSE + (s * a.Hq + (at - tok * a.Hq)) * a.Nq + (tok - s * a.Nq);
}

// Block `blk` of the rows and share `share` of the keys of pair `pair` (sequences of uneven lengths: longest first)
__device__ __forceinline__ QItem make_item(const QAttendArgs& a, const QAttendPlan& plan, int pair, int blk, int share) {
  const int rank = pair / a.c.c.Hkv;
  const CacheSequence cs = cache_sequence(a.c.c.lens, a.c.c.Nk, a.nseq, rank);
  QItem it;
  it.s = cs.s;
  it.g = pair - rank * a.c.c.Hkv;
  it.slot = share;
  it.row0 = blk * plan.rows;
  it.rows = a.Nq * a.G - it.row0 < plan.rows ? a.Nq * a.G - it.row0 : plan.rows;
  it.tok0 = (long)it.s * a.Nq;
  it.nk = cs.len;
  it.off = it.nk - a.Nq;
  const long begin = (long)share * plan.keys;
  it.begin = begin < it.nk ? (int)begin : it.nk;
  it.end = it.nk - it.begin < plan.keys ? it.nk : it.begin + plan.keys;
  return it;
}
// An item without keys: L = -inf, and with one share O = 0
template <int D>
__device__ __forceinline__ void empty_item(const QAttendArgs& a, const QItem& it, bool direct) {
  const long all = (long)a.nseq * a.Nq * a.Hq;
  for (int i = threadIdx.x; i < it.rows * (D / 4); i += 256) {
    const int r = i / (D / 4), c = i % (D / 4);
    const long at = out_row(a, it, r);
    if (direct) *(u32x2*)(a.O + at * D + 4 * c) = (u32x2){0u, 0u};
    if (c == 0) *(direct ? lse_at(a, at) : a.Lpart + it.slot * all + at) = -INFINITY;
  }
}

// Items of 128 rows (fa_qattend_wide.hip)
hipError_t launch_qattend_wide(const QAttendArgs& a, const QAttendPlan& plan, hipStream_t st);

}  // namespace fa
