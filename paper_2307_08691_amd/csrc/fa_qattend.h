// What the kernels of attention over a cache in 4 or 8 bits (fa_qattend.hip, fa_qattend_wide.hip) share: how the work is cut, and where results go.
//
// Unit: the rows of one block (plan.rows packed rows, query * G + head of the group) of a (sequence, key/value head) against all keys that
// they may see. Its keys come in chunks of 2^plan.chunk_log2; the chunks of all units, sequence by sequence, head by head, block by block, are numbered through
// and dealt in equal runs to as many workgroups as fit on the chip at once, whatever the lengths are. A workgroup goes through its run
// segment by segment, a segment being the part of a unit that lies in it. A unit that is one workgroup's alone is finished there; of the others
// each workgroup leaves a normalised partial O and its logsumexp, and the merge joins them (fa_merge.h). A workgroup has two partial segments at
// most: the first, that begins inside a unit (slot 2 w), and the last, that begins a unit (slot 2 w + 1).
// (64 paged sequences of up to 8192 keys, 32 heads on 8 of 128, 4 bits: 69 us with equal shares of each sequence, the longest first, 64 so.)
#pragma once
#include "fa_mx.h"

namespace fa {

struct QSegment {
  int s, g, len, begin, end;  // keys of the sequence, and those of the segment
  long tok0;                  // token of packed row 0
  int row0, rows, off, slot;  // slot < 0: the whole unit
};
struct QRow {  // of packed row r of the block: token * Hq + head, and its place in LSE
  long at, lse;
};
__device__ __forceinline__ QRow out_row(const QAttendArgs& a, const QSegment& it, int r) {
  const int row = it.row0 + r, q = (int)((unsigned)row / (unsigned)a.G), h = it.g * a.G + (row - q * a.G);
  return {(it.tok0 + q) * a.Hq + h, ((long)it.s * a.Hq + h) * a.Nq + q};
}
__device__ __forceinline__ float* part_o(const QAttendArgs& a, const QAttendPlan& p, int slot, int r) {
  return a.Opart + ((long)slot * p.rows + r) * a.c.c.d;
}

// Chunks of the keys that the rows of block `blk` see of a sequence of `len`
__device__ __forceinline__ int block_chunks(const QAttendArgs& a, const QAttendPlan& p, int len, int blk, int& keys) {
  int n = len;
  if (a.causal && a.Nq > 1) {  // (what the block's last row sees)
    const int past = (blk + 1) * p.rows < a.Nq * a.G ? (blk + 1) * p.rows : a.Nq * a.G;
    n = len - a.Nq + (past - 1) / a.G + 1;
    n = n < 0 ? 0 : (n < len ? n : len);
  }
  keys = n;
  return (n + (1 << p.chunk_log2) - 1) >> p.chunk_log2;
}
__device__ __forceinline__ int head_chunks(const QAttendArgs& a, const QAttendPlan& p, int len) {  // of all blocks
  int keys;
  if (p.blocks == 1) return block_chunks(a, p, len, 0, keys);
  if (!a.causal) return block_chunks(a, p, len, 0, keys) * p.blocks;
  int n = 0;
  for (int b = 0; b < p.blocks; ++b) n += block_chunks(a, p, len, b, keys);
  return n;
}
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// The segments of this workgroup of 256 in turn: work(segment). LDS is the work's between its calls, which end with everyone done with it.
// (All counts fit 31 bits: the entry point sees to it.)
template <class F>
__device__ __forceinline__ void for_segments(const QAttendArgs& a, const QAttendPlan& p, char* smem, F work) {
  int* const room = (int*)smem;        // sums of the four wavefronts
  int* const found = (int*)(smem + 16);  // where this workgroup's run begins: sequence, its length, its chunks a head, the chunks before it
  const int Hkv = a.c.c.Hkv, b = blockIdx.x, tid = threadIdx.x;
  // each thread counts the chunks of as many sequences; a scan over threads
  const int each = (a.nseq + 255) / 256, s0 = tid * each < a.nseq ? tid * each : a.nseq, s1 = s0 + each < a.nseq ? s0 + each : a.nseq;
  int mine = 0, len0 = 0, chunks0 = 0;
  for (int s = s0; s < s1; ++s) {
    const int len = held_keys(a.c.c, s), n = head_chunks(a, p, len);
    if (s == s0) len0 = len, chunks0 = n;
    mine += n;
  }
  int sum = mine;
  sum += __builtin_amdgcn_update_dpp(0, sum, 0x111, 0xf, 0xf, true);  // (the steps of wave_sum: every lane has the sum up to itself)
  sum += __builtin_amdgcn_update_dpp(0, sum, 0x112, 0xf, 0xf, true);
  sum += __builtin_amdgcn_update_dpp(0, sum, 0x114, 0xf, 0xf, true);
  sum += __builtin_amdgcn_update_dpp(0, sum, 0x118, 0xf, 0xf, true);
  sum += __builtin_amdgcn_update_dpp(0, sum, 0x142, 0xa, 0xf, false);
  sum += __builtin_amdgcn_update_dpp(0, sum, 0x143, 0xc, 0xf, false);
  if ((tid & 63) == 63) room[tid >> 6] = sum;
  __syncthreads();
  int before = sum - mine, all = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int y = room[i];
    if (i < tid >> 6) before += y;
    all += y;
  }
  all = uniform(all) * Hkv;
  // As many workgroups as there are, or as there are chunks; a multiple of the XCDs where it can be. The first `more` of them have a
  // chunk more than the others.
  unsigned n = (unsigned)all < (unsigned)p.groups ? (unsigned)all : (unsigned)p.groups;
  if (n >= kXcds) n = n / kXcds * kXcds;
  n = (unsigned)uniform((int)n);
  if ((unsigned)b < n) {
    const int run = uniform((int)((unsigned)all / n)), more = all - run * (int)n;
    const int w = n >= kXcds ? b % kXcds * (int)(n / kXcds) + b / kXcds : b;  // (neighbours in the order of the chunks: on one XCD)
    int at = w * run + (w < more ? w : more);
    const int end = at + run + (w < more ? 1 : 0);
    if (before * Hkv <= at && at < (before + mine) * Hkv) {
      int s = s0, len = len0, m = chunks0, base = before * Hkv;
      while (at - base >= m * Hkv) {
        base += m * Hkv;
        len = held_keys(a.c.c, ++s);
        m = head_chunks(a, p, len);
      }
      found[0] = s, found[1] = len, found[2] = m, found[3] = base;
    }
    __syncthreads();
    int s = uniform(found[0]), len = uniform(found[1]), per_head = uniform(found[2]), base = uniform(found[3]);
    __syncthreads();
    while (at < end) {
      while (at - base >= per_head * Hkv) {  // the next sequence that has any
        base += per_head * Hkv;
        len = uniform(held_keys(a.c.c, ++s));
        per_head = uniform(head_chunks(a, p, len));
      }
      QSegment it;
      it.s = s;
      it.len = len;
      it.g = uniform((int)((unsigned)(at - base) / (unsigned)per_head));
      int in = at - base - it.g * per_head;
      int blk = 0, keys, chunks = block_chunks(a, p, len, 0, keys);
      while (in >= chunks) {
        in -= chunks;
        chunks = block_chunks(a, p, len, ++blk, keys);
      }
      const int take = end - at < chunks - in ? end - at : chunks - in;
      it.begin = in << p.chunk_log2;
      it.end = in + take < chunks ? (in + take) << p.chunk_log2 : keys;
      it.row0 = blk * p.rows;
      it.rows = a.Nq * a.G - it.row0 < p.rows ? a.Nq * a.G - it.row0 : p.rows;
      it.tok0 = (long)s * a.Nq;
      it.off = len - a.Nq;
      it.slot = take == chunks ? -1 : (in == 0 ? 2 * w + 1 : 2 * w);
      if (in == 0 && p.slots && tid == 0) {  // for the merge: who has parts of the unit that begins here
        int parts = 0;
        if (take < chunks) {  // its last chunk's workgroup: the first `more` have run + 1 each
          const int c = at + chunks - 1, long_ones = more * (run + 1);
          parts = (c < long_ones ? (int)((unsigned)c / (unsigned)(run + 1)) : more + (int)((unsigned)(c - long_ones) / (unsigned)run)) - w + 1;
        }
        a.units[((long)s * Hkv + it.g) * p.blocks + blk] = {w, parts};
      }
      at += take;
      work(it);
    }
  }
  // ---- blocks of rows that see no key: O = 0, L = -inf
  for (int s = b; s < a.nseq; s += gridDim.x) {
    const int len = uniform(held_keys(a.c.c, s));
    if (len >= a.Nq || (!a.causal && len > 0)) continue;
    for (int blk = 0; blk < p.blocks; ++blk) {
      int keys;
      if (block_chunks(a, p, len, blk, keys)) continue;
      const int row0 = blk * p.rows, rows = a.Nq * a.G - row0 < p.rows ? a.Nq * a.G - row0 : p.rows, d4 = a.c.c.d / 4;
      for (long i = tid; i < (long)Hkv * rows * d4; i += 256) {
        const int c4 = (int)(i % d4), r = (int)(i / d4 % rows);
        QSegment it;
        it.s = s, it.g = (int)(i / d4 / rows), it.tok0 = (long)s * a.Nq, it.row0 = row0;
        const QRow row = out_row(a, it, r);
        *(u32x2*)(a.O + row.at * a.c.c.d + 4 * c4) = (u32x2){0u, 0u};
        if (c4 == 0) a.LSE[row.lse] = -INFINITY;
        const int g = it.g;
        if (p.slots && c4 == 0 && r == 0) a.units[((long)s * Hkv + g) * p.blocks + blk] = {0, 0};
      }
    }
  }
}

// A wavefront's four elements of a finished row (slot < 0) or of a partial one
template <bool F16>
__device__ __forceinline__ void put_row(const QAttendArgs& a, const QAttendPlan& p, const QSegment& it, int r, int c4, f32x4 o, float lse) {
  if (it.slot < 0) {
    const QRow row = out_row(a, it, r);
    u32x2 x;
    x[0] = pack2<F16>(o[0], o[1]);
    x[1] = pack2<F16>(o[2], o[3]);
    *(u32x2*)(a.O + row.at * a.c.c.d + 4 * c4) = x;
    if (c4 == 0) a.LSE[row.lse] = lse;
  } else {
    *(f32x4*)(part_o(a, p, it.slot, r) + 4 * c4) = o;
    if (c4 == 0) a.Lpart[(long)it.slot * p.rows + r] = lse;
  }
}

// Items of 128 rows (fa_qattend_wide.hip)
hipError_t launch_qattend_wide(const QAttendArgs& a, const QAttendPlan& plan, hipStream_t st);

}  // namespace fa
