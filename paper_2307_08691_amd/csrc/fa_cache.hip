// A key/value cache that is written and kept small: new rows in (append), and the slots that drew least attention weight out (evict).
#include <hip/hip_runtime.h>

#include "fa_kernels.h"
#include "fa_lds.h"

namespace fa {

// ---- append: row i of sequence s goes to slot lens[s] - Nq + i. One thread moves 16 bytes of K and the same of V; the thread of
// a row's first piece sets the slot's weight and position. Bound by launch and latency at one row a sequence, by HBM above.
__global__ __launch_bounds__(256) void append_kernel(AppendArgs a) {
  const CacheView& c = a.c;
  const int cpr = c.d / 8;
  const long i = (long)blockIdx.x * 256 + threadIdx.x;
  const long row = i / cpr;  // (sequence, query, head)
  const int piece = (int)(i - row * cpr);
  const long tok = row / c.Hkv;
  const int g = (int)(row - tok * c.Hkv);
  const long s = tok / a.Nq;
  if (s >= a.nseq) return;
  const int q = (int)(tok - s * a.Nq);
  const long slot = (long)(c.lens ? c.lens[s] : c.Nk) - a.Nq + q;
  if (slot < 0 || slot >= c.Nk) return;  // (a length that is no length of this cache)
  const u32x4 k = *(const u32x4*)(a.Kn + 8 * i), v = *(const u32x4*)(a.Vn + 8 * i);
  const long at = (cache_row(c, (int)s, (int)slot) * c.Hkv + g) * c.d + 8 * piece;
  *(u32x4*)(a.K + at) = k;
  *(u32x4*)(a.V + at) = v;
  if (piece == 0) {
    const long w = (s * c.Hkv + g) * c.Nk + slot;
    if (a.weights) a.weights[w] = 0.f;
    if (a.positions) a.positions[w] = a.first ? a.first[s] + q : (int)slot;
  }
}
hipError_t launch_append(const AppendArgs& a, hipStream_t st) {
  const long pieces = (long)a.nseq * a.Nq * a.c.Hkv * (a.c.d / 8);
  hipLaunchKernelGGL(append_kernel, dim3((unsigned)((pieces + 255) / 256)), dim3(256), 0, st, a);
  return hipGetLastError();
}

// ---- evict
// Slots are ordered by a 32-bit key: the weight's bits made monotonic (-0 as 0, NaN below everything), all ones for a protected slot.
constexpr uint32_t kProtected = 0xffffffffu;
__device__ __forceinline__ uint32_t evict_key(float w, int pos, int sinks, long recent_from) {
  if (pos < sinks || pos >= recent_from) return kProtected;
  if (w != w) return 0u;
  const uint32_t x = __builtin_bit_cast(uint32_t, w + 0.f);
  return x & 0x80000000u ? ~x : x | 0x80000000u;
}
__device__ __forceinline__ int lane_before(unsigned long long m) {  // set bits below this lane
  return __builtin_amdgcn_mbcnt_hi((unsigned)(m >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)m, 0u));
}
constexpr int kEvictBins = 2048;

// Sum over the lanes up to this one (all active); the steps of wave_sum (fa_common.h).
__device__ __forceinline__ int lane_scan(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);
  return x;
}
typedef int i32x4 __attribute__((ext_vector_type(4)));
// Of the wavefronts' values in LDS: the sum of those before wavefront w, and of all. (Read together: one by one each is a latency.)
struct BeforeAndAll {
  int before, all;
};
template <int NW>
__device__ __forceinline__ BeforeAndAll over_waves(const int (&part)[NW], int w) {
  BeforeAndAll s = {0, 0};
  i32x4 x[NW / 4];
#pragma unroll
  for (int i = 0; i < NW / 4; ++i) x[i] = ((const i32x4*)part)[i];
#pragma unroll
  for (int i = 0; i < NW; ++i) {
    s.before += i < w ? x[i / 4][i % 4] : 0;
    s.all += x[i / 4][i % 4];
  }
  return s;
}

// One row of K and of V of a move, 16 bytes a thread
__device__ __forceinline__ void move_piece(const EvictArgs& a, int s, int g, int src, int dst, int piece) {
  const CacheView& c = a.c;
  const long from = (cache_row(c, s, src) * c.Hkv + g) * c.d + 8 * piece, to = (cache_row(c, s, dst) * c.Hkv + g) * c.d + 8 * piece;
  const u32x4 k = *(const u32x4*)(a.K + from), v = *(const u32x4*)(a.V + from);
  *(u32x4*)(a.K + to) = k;
  *(u32x4*)(a.V + to) = v;
}

// One workgroup per (sequence, key/value head). The last slot that stays, by key and then by slot, is found by counting the keys by
// their upper bits in LDS (11, 11 and 10 bits), and as soon as its counter has at most kFewKeys keys by comparing those with each other:
// after one round unless weights are much alike. A wavefront owns a contiguous range of slots, so that slot order is (wavefront,
// step, lane) and ranks are counts of ballots. Kept slots past the budget then move into free ones
// below it, both ascending: as many rows move as must, in place, and what stays keeps its slot. Bound by instructions where there are
// many pairs (so: few wavefronts, each with many slots) and by a chain of barriers and LDS latencies where there are few.
// ITEMS > 0: a lane's keys stay in registers (up to THREADS * ITEMS slots); 0: they are formed again from L2 in every round.
// Where no more than kFewMoves rows can have to move, they do so here, else by evict_move_kernel.
constexpr int kFewMoves = 64, kFewKeys = 64;
template <int THREADS, int ITEMS>
__global__ __launch_bounds__(THREADS) void evict_select_kernel(EvictArgs a) {
  constexpr int NW = THREADS / 64, BPT = kEvictBins / THREADS;  // counters of a thread
  __shared__ __attribute__((aligned(16))) int hist[kEvictBins];
  __shared__ __attribute__((aligned(16))) int part[4][NW];
  __shared__ int found[3][3];
  __shared__ __attribute__((aligned(16))) uint32_t few_keys[kFewKeys];
  __shared__ __attribute__((aligned(16))) int few_slots[kFewKeys];
  __shared__ int few_count, last_slot;
  __shared__ uint32_t last_key;
  __shared__ int few[2][kFewMoves];
  const int pair = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int s = pair / a.c.Hkv, g = pair - s * a.c.Hkv, budget = a.budget;
  const bool here = a.room <= kFewMoves;
  const long base = (long)pair * a.c.Nk;
  const float* W = a.weights + base;
  const int32_t* P = a.positions + base;
  float* Wo = a.weights_out + base;
  int32_t* Po = a.positions_out + base;
  // This lane: slots first + 64 i. They go by the slots that there are, not by those in use, so that the values are requested together
  // with the length.
  const int steps = (a.c.Nk + THREADS - 1) / THREADS, first = w * steps * 64 + lane;
  constexpr bool KEPT = ITEMS > 0 && ITEMS <= 8;  // weights and positions stay in registers too
  float wt[KEPT ? ITEMS : 1];
  int pos[KEPT ? ITEMS : 1];
  if constexpr (KEPT) {
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {  // (slots that are not there: the last one again)
      const int slot = i < steps && first + 64 * i < a.c.Nk ? first + 64 * i : a.c.Nk - 1;
      wt[i] = W[slot];
      pos[i] = P[slot];
    }
  }
  const int n = held_keys(a.c, s);
  if (a.lens_out != a.c.lens && g == 0 && tid == 0) a.lens_out[s] = n < budget ? n : budget;  // (else others still read it)
  if (n <= budget) {  // nothing goes
    if (!here && tid == 0) a.moves[pair] = 0;
    if (Wo != W)
      for (int i = tid; i < n; i += THREADS) Wo[i] = W[i];
    if (Po != P)
      for (int i = tid; i < n; i += THREADS) Po[i] = P[i];
    return;
  }
  auto clear = [&]() {
#pragma unroll
    for (int i = 0; i < BPT; ++i) hist[tid + i * THREADS] = 0;
  };
  int top = -0x7fffffff - 1;  // the newest position
  clear();
  if constexpr (KEPT) {
#pragma unroll
    for (int i = 0; i < ITEMS; ++i)
      if (i < steps && first + 64 * i < n) top = max(top, pos[i]);
  } else {
#pragma unroll 8
    for (int i = 0; i < steps; ++i) top = max(top, P[first + 64 * i < n ? first + 64 * i : n - 1]);
  }
  for (int o = 32; o; o >>= 1) top = max(top, __shfl_xor(top, o));
  if (lane == 0) part[0][w] = top;
  if (tid == 0) few_count = 0;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < NW / 4; ++i) {
    const i32x4 x = ((const i32x4*)part[0])[i];
    top = max(max(top, max(x[0], x[1])), max(x[2], x[3]));
  }
  const long recent_from = (long)top + 1 - a.recent;
  uint32_t held[ITEMS ? ITEMS : 1];
  if constexpr (KEPT) {
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) held[i] = evict_key(wt[i], pos[i], a.sinks, recent_from);
  } else if constexpr (ITEMS > 0) {
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      const int slot = first + 64 * i < n ? first + 64 * i : n - 1;
      held[i] = evict_key(W[slot], P[slot], a.sinks, recent_from);
    }
  }
  auto each = [&](auto f) {  // f(i, slot, key, whether the slot is held), for whole wavefronts
    if constexpr (ITEMS > 0) {
#pragma unroll
      for (int i = 0; i < ITEMS; ++i)
        if (i < steps) f(i, first + 64 * i, held[i], first + 64 * i < n);
    } else {
      for (int i = 0; i < steps; ++i) {
        const int slot = first + 64 * i, at = slot < n ? slot : n - 1;
        f(i, slot, evict_key(W[at], P[at], a.sinks, recent_from), slot < n);
      }
    }
  };
  // ---- the budget-th largest key
  uint32_t limit = 0, above = 0;  // bits of it known so far, and which they are
  int rest = budget;              // its rank among the keys that share them
  int alike = n;                  // how many do
#pragma unroll
  for (int round = 0; round < 3; ++round) {
    if (round > 0 && alike <= kFewKeys) break;
    const int shift = round == 0 ? 21 : round == 1 ? 10 : 0;
    const uint32_t bins = round < 2 ? 2047u : 1023u;
    if (round > 0) {
      clear();
      __syncthreads();
    }
    int safe = 0;  // protected slots come first of all: they are counted apart
    each([&](int, int, uint32_t key, bool in) {
      if (round == 0) safe += __builtin_popcountll(__builtin_amdgcn_ballot_w64(in && key == kProtected));
      in = in && key != kProtected && (key & above) == limit;
      const unsigned long long m = __builtin_amdgcn_ballot_w64(in);
      if (!m) return;
      const int bin = (key >> shift) & bins, one = __builtin_amdgcn_readlane(bin, __builtin_ctzll(m));
      if (__builtin_amdgcn_ballot_w64(in && bin != one) == 0) {  // (weights that are all alike would queue for one counter)
        if (lane == 0) atomicAdd(&hist[one], __builtin_popcountll(m));
      } else if (in) {
        atomicAdd(&hist[bin], 1);
      }
    });
    if (round == 0 && lane == 0) part[2][w] = safe;
    __syncthreads();
    if (round == 0) {
      const int all = over_waves(part[2], w).all;
      if (all >= budget) {
        limit = above = kProtected;
        alike = all;
        break;
      }
      rest -= all;
    }
    // thread t: BPT bins, thread 0 the topmost; how many keys lie in the bins down to its last
    int h[BPT], mine = 0;
#pragma unroll
    for (int i = 0; i < BPT; ++i) mine += h[i] = hist[kEvictBins - 1 - (BPT * tid + i)];
    int down = lane_scan(mine);
    if (lane == 63) part[1][w] = down;
    __syncthreads();
    down += over_waves(part[1], w).before;
    int up = down - mine;
    if (up < rest && down >= rest) {
      int hit = 0;
#pragma unroll
      for (int i = 0; i < BPT - 1; ++i)
        if (hit == i && up + h[i] < rest) up += h[i], ++hit;
      found[round][0] = kEvictBins - 1 - (BPT * tid + hit);
      found[round][1] = rest - up;
      found[round][2] = h[0];
#pragma unroll
      for (int i = 1; i < BPT; ++i)
        if (hit == i) found[round][2] = h[i];
    }
    __syncthreads();
    limit |= (uint32_t)found[round][0] << shift;
    above |= bins << shift;
    rest = found[round][1];
    alike = found[round][2];
  }
  if (alike <= kFewKeys) {  // they are written down and compared
    each([&](int, int slot, uint32_t key, bool in) {
      if (in && (key & above) == limit) {
        const int at = atomicAdd(&few_count, 1);
        few_keys[at] = key;
        few_slots[at] = slot;
      }
    });
    __syncthreads();
    if (tid < alike) {
      const uint32_t key = few_keys[tid];
      const int slot = few_slots[tid];
      int ahead = 0;
      for (int i = 0; i < alike; i += 4) {  // (what lies behind them is passed over)
        const u32x4 k = *(const u32x4*)(few_keys + i);
        const i32x4 x = *(const i32x4*)(few_slots + i);
#pragma unroll
        for (int u = 0; u < 4; ++u) ahead += i + u < alike && (k[u] > key || (k[u] == key && x[u] < slot));
      }
      if (ahead == rest - 1) {
        last_key = key;
        last_slot = slot;
      }
    }
  } else {  // (all of them equal: the rest-th in slot order)
    int equals = 0;
    each([&](int, int, uint32_t key, bool in) { equals += __builtin_popcountll(__builtin_amdgcn_ballot_w64(in && key == limit)); });
    if (lane == 0) part[0][w] = equals;
    __syncthreads();
    int rank = over_waves(part[0], w).before;
    each([&](int, int slot, uint32_t key, bool in) {
      const unsigned long long eq = __builtin_amdgcn_ballot_w64(in && key == limit);
      if (in && key == limit && rank + lane_before(eq) == rest - 1) {
        last_key = limit;
        last_slot = slot;
      }
      rank += __builtin_popcountll(eq);
    });
  }
  __syncthreads();
  // ---- who stays
  const uint32_t least = last_key;
  const int least_slot = last_slot;
  uint32_t kept = 0;  // (ITEMS > 0) of the lane's slots
  int nfree = 0, nmove = 0;
  auto keeps = [&](int slot, uint32_t key, bool in) { return in && (key > least || (key == least && slot <= least_slot)); };
  each([&](int i, int slot, uint32_t key, bool in) {
    const bool keep = keeps(slot, key, in);
    if (ITEMS > 0) kept |= (uint32_t)keep << i;
    nfree += __builtin_popcountll(__builtin_amdgcn_ballot_w64(in && !keep && slot < budget));
    nmove += __builtin_popcountll(__builtin_amdgcn_ballot_w64(keep && slot >= budget));
  });
  if (lane == 0) {
    part[2][w] = nfree;
    part[3][w] = nmove;
  }
  __syncthreads();
  int free_at = over_waves(part[2], w).before;
  const BeforeAndAll moved = over_waves(part[3], w);
  int move_at = moved.before;
  const int count = moved.all;
  int32_t* const dst = here ? few[0] : a.moves + gridDim.x + (long)pair * 2 * a.room;
  int32_t* const src = here ? few[1] : dst + a.room;
  each([&](int i, int slot, uint32_t key, bool in) {
    const bool keep = ITEMS > 0 ? kept >> i & 1 : keeps(slot, key, in);
    const bool fr = in && !keep && slot < budget, mv = keep && slot >= budget;
    const unsigned long long mf = __builtin_amdgcn_ballot_w64(fr), mm = __builtin_amdgcn_ballot_w64(mv);
    if (mf) {
      if (fr) dst[free_at + lane_before(mf)] = slot;
      free_at += __builtin_popcountll(mf);
    }
    if (mm) {
      if (mv) src[move_at + lane_before(mm)] = slot;
      move_at += __builtin_popcountll(mm);
    }
    if (keep && slot < budget) {
      if (Wo != W) Wo[slot] = KEPT ? wt[i] : W[slot];
      if (Po != P) Po[slot] = KEPT ? pos[i] : P[slot];
    }
  });
  if (!here && tid == 0) a.moves[pair] = count;
  if (here) lds_barrier();  // (the lists are in LDS: what has been stored to memory need not have arrived)
  else __syncthreads();
  for (int j = tid; j < count; j += THREADS) {  // (sources lie at or past the budget, where nothing is written)
    Wo[dst[j]] = W[src[j]];
    Po[dst[j]] = P[src[j]];
  }
  if (here) {
    const int cpr = a.c.d / 8;
    for (int i = tid; i < count * cpr; i += THREADS) move_piece(a, s, g, src[i / cpr], dst[i / cpr], i % cpr);
  }
}

__device__ __forceinline__ void cut_length(const EvictArgs& a, int s) {
  const int n = held_keys(a.c, s);
  a.lens_out[s] = n < a.budget ? n : a.budget;
}
// The moves of K and V rows; and the lengths, where they are cut in place and the kernel above still reads them.
__global__ __launch_bounds__(256) void evict_move_kernel(EvictArgs a) {
  const int pairs = a.nseq * a.c.Hkv, pair = blockIdx.x, s = pair / a.c.Hkv, g = pair - s * a.c.Hkv;
  if (a.lens_out == a.c.lens && blockIdx.y == 0 && g == 0 && threadIdx.x == 0) cut_length(a, s);
  const int count = a.moves[pair];
  const int32_t* dst = a.moves + pairs + (long)pair * 2 * a.room;
  const int32_t* src = dst + a.room;
  const int cpr = a.c.d / 8;
  const long pieces = (long)count * cpr;
  for (long i = (long)blockIdx.y * 256 + threadIdx.x; i < pieces; i += (long)gridDim.y * 256) {
    const int j = (int)(i / cpr);
    move_piece(a, s, g, src[j], dst[j], (int)(i - (long)j * cpr));
  }
}
__global__ __launch_bounds__(256) void evict_lengths_kernel(EvictArgs a) {
  const int s = blockIdx.x * 256 + threadIdx.x;
  if (s < a.nseq) cut_length(a, s);
}

hipError_t launch_evict(const EvictArgs& a, hipStream_t st) {
  const unsigned pairs = (unsigned)(a.nseq * a.c.Hkv);
  // (us at 256 / 512 / 1024 threads: 64 x 8 pairs of 2112 slots 12.4 / 10.8 / 16.6, 1 x 8 of 4096 19.8 / 14.3 / 14.5; 8 x 8 of 8192 at 512 / 1024:
  // 26.0 / 24.0; 2 x 8 of 32768: 110 with keys formed anew in every round, 76 with them in registers)
  if (a.c.Nk <= 4096) hipLaunchKernelGGL((evict_select_kernel<512, 8>), dim3(pairs), dim3(512), 0, st, a);
  else if (a.c.Nk <= 8192) hipLaunchKernelGGL((evict_select_kernel<1024, 8>), dim3(pairs), dim3(1024), 0, st, a);
  else if (a.c.Nk <= 32768) hipLaunchKernelGGL((evict_select_kernel<1024, 32>), dim3(pairs), dim3(1024), 0, st, a);
  else hipLaunchKernelGGL((evict_select_kernel<1024, 0>), dim3(pairs), dim3(1024), 0, st, a);
  if (hipError_t e = hipGetLastError()) return e;
  if (a.room <= kFewMoves) {
    if (a.lens_out != a.c.lens) return hipSuccess;
    hipLaunchKernelGGL(evict_lengths_kernel, dim3((a.nseq + 255) / 256), dim3(256), 0, st, a);
    return hipGetLastError();
  }
  const long most = (long)a.room * (a.c.d / 8);  // pieces of a pair
  long y = (most + 255) / 256;
  y = y < 1 ? 1 : (y > 64 ? 64 : y);
  hipLaunchKernelGGL(evict_move_kernel, dim3(pairs, (unsigned)y), dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace fa
