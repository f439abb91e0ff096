// A key/value cache that is written and kept small: new rows in (append), and the slots that drew least attention weight out (evict).
#include <hip/hip_runtime.h>

#include "fa_kernels.h"

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
__device__ __forceinline__ uint32_t evict_key(float w, int pos, int sinks, long recent_from) {
  if (pos < sinks || pos >= recent_from) return 0xffffffffu;
  if (w != w) return 0u;
  const uint32_t x = __builtin_bit_cast(uint32_t, w + 0.f);
  return x & 0x80000000u ? ~x : x | 0x80000000u;
}
__device__ __forceinline__ int lane_before(unsigned long long m) {  // set bits below this lane
  return __builtin_amdgcn_mbcnt_hi((unsigned)(m >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)m, 0u));
}
constexpr int kEvictThreads = 1024, kEvictWaves = 16, kEvictBins = 2048;

// One workgroup per (sequence, key/value head). The budget-th largest key is found by three rounds of counting (11, 11 and 10 bits)
// in LDS; what is above it stays, and of its equals the first ones in slot order. A wavefront owns a contiguous range of slots, so
// that slot order is (wavefront, step, lane) and ranks are counts of ballots. Kept slots past the budget then move into free ones
// below it, both ascending: as many rows move as must, in place, and what stays keeps its slot.
// ITEMS > 0: a lane's keys stay in registers (up to 1024 * ITEMS slots); 0: they are formed again from L2 in every round.
template <int ITEMS>
__global__ __launch_bounds__(kEvictThreads) void evict_select_kernel(EvictArgs a) {
  __shared__ int hist[kEvictBins];
  __shared__ int part[3][kEvictWaves];
  __shared__ int found[2];
  const int pair = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int s = pair / a.c.Hkv, n = held_keys(a.c, s), budget = a.budget;
  const long base = (long)pair * a.c.Nk;
  const float* W = a.weights + base;
  const int32_t* P = a.positions + base;
  float* Wo = a.weights_out + base;
  int32_t* Po = a.positions_out + base;
  if (n <= budget) {  // nothing goes
    if (tid == 0) a.moves[pair] = 0;
    if (Wo != W)
      for (int i = tid; i < n; i += kEvictThreads) Wo[i] = W[i];
    if (Po != P)
      for (int i = tid; i < n; i += kEvictThreads) Po[i] = P[i];
    return;
  }
  const int steps = (n + kEvictThreads - 1) / kEvictThreads, first = w * steps * 64 + lane;  // this lane: slots first + 64 i
  // the newest position
  int top = -0x7fffffff - 1;
  for (int i = 0; i < steps; ++i)
    if (first + 64 * i < n) top = max(top, P[first + 64 * i]);
  for (int o = 32; o; o >>= 1) top = max(top, __shfl_xor(top, o));
  if (lane == 0) part[0][w] = top;
  __syncthreads();
  for (int i = 0; i < kEvictWaves; ++i) top = max(top, part[0][i]);
  const long recent_from = (long)top + 1 - a.recent;
  auto form = [&](int slot) { return evict_key(W[slot], P[slot], a.sinks, recent_from); };
  uint32_t held[ITEMS ? ITEMS : 1];
  if constexpr (ITEMS > 0) {
#pragma unroll
    for (int i = 0; i < ITEMS; ++i)
      if (i < steps && first + 64 * i < n) held[i] = form(first + 64 * i);
  }
  auto each = [&](auto f) {  // f(slot, key, whether the slot is held), for whole wavefronts
    if constexpr (ITEMS > 0) {
#pragma unroll
      for (int i = 0; i < ITEMS; ++i)
        if (i < steps) f(first + 64 * i, held[i], first + 64 * i < n);
    } else {
      for (int i = 0; i < steps; ++i) {
        const int slot = first + 64 * i;
        f(slot, slot < n ? form(slot) : 0u, slot < n);
      }
    }
  };
  // ---- the budget-th largest key
  uint32_t limit = 0, above = 0;  // bits of it known so far, and which they are
  int rest = budget;              // its rank among the keys that share them
  for (int round = 0; round < 3; ++round) {
    const int shift = round == 0 ? 21 : round == 1 ? 10 : 0;
    const uint32_t bins = round < 2 ? 2047u : 1023u;
    hist[tid] = hist[tid + kEvictThreads] = 0;
    __syncthreads();
    each([&](int, uint32_t key, bool in) {
      in = in && (key & above) == limit;
      const unsigned long long m = __builtin_amdgcn_ballot_w64(in);
      if (!m) return;
      const int bin = (key >> shift) & bins;
      // (weights that are all alike would queue for one counter)
      const int one = __builtin_amdgcn_readlane(bin, __builtin_ctzll(m));
      if (__builtin_amdgcn_ballot_w64(in && bin != one) == 0) {
        if (lane == 0) atomicAdd(&hist[one], __builtin_popcountll(m));
      } else if (in) {
        atomicAdd(&hist[bin], 1);
      }
    });
    __syncthreads();
    // bins 2 t, 2 t + 1 of thread t; how many keys lie in the bins from there on
    const int h0 = hist[2 * tid], h1 = hist[2 * tid + 1];
    int from = h0 + h1;
    for (int o = 1; o < 64; o <<= 1) {
      const int x = __shfl_down(from, o);
      if (lane + o < 64) from += x;
    }
    if (lane == 0) part[1][w] = from;
    __syncthreads();
    for (int i = w + 1; i < kEvictWaves; ++i) from += part[1][i];
    if (from >= rest && from - h0 - h1 < rest) {
      const int after1 = from - h0 - h1, hit1 = after1 + h1 >= rest;
      found[0] = 2 * tid + hit1;
      found[1] = rest - (hit1 ? after1 : after1 + h1);
    }
    __syncthreads();
    limit |= (uint32_t)found[0] << shift;
    above |= bins << shift;
    rest = found[1];
  }
  // ---- who stays: larger keys, and the first `rest` equals
  int equals = 0;
  each([&](int, uint32_t key, bool in) { equals += __builtin_popcountll(__builtin_amdgcn_ballot_w64(in && key == limit)); });
  if (lane == 0) part[0][w] = equals;
  __syncthreads();
  int before = 0;
  for (int i = 0; i < w; ++i) before += part[0][i];
  auto each_kept = [&](auto f) {
    int rank = before;
    each([&](int slot, uint32_t key, bool in) {
      const unsigned long long eq = __builtin_amdgcn_ballot_w64(in && key == limit);
      const bool keep = in && (key > limit || (key == limit && rank + lane_before(eq) < rest));
      rank += __builtin_popcountll(eq);
      f(slot, in, keep);
    });
  };
  int nfree = 0, nmove = 0;
  each_kept([&](int slot, bool in, bool keep) {
    nfree += __builtin_popcountll(__builtin_amdgcn_ballot_w64(in && !keep && slot < budget));
    nmove += __builtin_popcountll(__builtin_amdgcn_ballot_w64(keep && slot >= budget));
  });
  if (lane == 0) {
    part[1][w] = nfree;
    part[2][w] = nmove;
  }
  __syncthreads();
  int free_at = 0, move_at = 0, count = 0;
  for (int i = 0; i < kEvictWaves; ++i) {
    if (i < w) {
      free_at += part[1][i];
      move_at += part[2][i];
    }
    count += part[2][i];
  }
  int32_t* dst = a.moves + gridDim.x + (long)pair * 2 * a.room;
  int32_t* src = dst + a.room;
  each_kept([&](int slot, bool in, bool keep) {
    const bool fr = in && !keep && slot < budget, mv = keep && slot >= budget;
    const unsigned long long mf = __builtin_amdgcn_ballot_w64(fr), mm = __builtin_amdgcn_ballot_w64(mv);
    if (fr) dst[free_at + lane_before(mf)] = slot;
    if (mv) src[move_at + lane_before(mm)] = slot;
    free_at += __builtin_popcountll(mf);
    move_at += __builtin_popcountll(mm);
    if (keep && slot < budget) {
      if (Wo != W) Wo[slot] = W[slot];
      if (Po != P) Po[slot] = P[slot];
    }
  });
  if (tid == 0) a.moves[pair] = count;
  __syncthreads();
  for (int j = tid; j < count; j += kEvictThreads) {  // (sources lie at or past the budget, where nothing is written)
    Wo[dst[j]] = W[src[j]];
    Po[dst[j]] = P[src[j]];
  }
}

// The moves of K and V rows, 16 bytes a thread; and the lengths, which the kernel above still reads.
__global__ __launch_bounds__(256) void evict_move_kernel(EvictArgs a) {
  const CacheView& c = a.c;
  const int pairs = a.nseq * c.Hkv, pair = blockIdx.x, s = pair / c.Hkv, g = pair - s * c.Hkv;
  if (blockIdx.y == 0 && g == 0 && threadIdx.x == 0) {
    const int n = held_keys(c, s);
    a.lens_out[s] = n < a.budget ? n : a.budget;
  }
  const int count = a.moves[pair];
  const int32_t* dst = a.moves + pairs + (long)pair * 2 * a.room;
  const int32_t* src = dst + a.room;
  const int cpr = c.d / 8;
  const long pieces = (long)count * cpr;
  for (long i = (long)blockIdx.y * 256 + threadIdx.x; i < pieces; i += (long)gridDim.y * 256) {
    const int j = (int)(i / cpr), piece = (int)(i - (long)j * cpr);
    const long from = (cache_row(c, s, src[j]) * c.Hkv + g) * c.d + 8 * piece, to = (cache_row(c, s, dst[j]) * c.Hkv + g) * c.d + 8 * piece;
    const u32x4 k = *(const u32x4*)(a.K + from), v = *(const u32x4*)(a.V + from);
    *(u32x4*)(a.K + to) = k;
    *(u32x4*)(a.V + to) = v;
  }
}

hipError_t launch_evict(const EvictArgs& a, hipStream_t st) {
  const unsigned pairs = (unsigned)(a.nseq * a.c.Hkv);
  const dim3 block(kEvictThreads);
  if (a.c.Nk <= 2 * kEvictThreads) hipLaunchKernelGGL(evict_select_kernel<2>, dim3(pairs), block, 0, st, a);
  else if (a.c.Nk <= 8 * kEvictThreads) hipLaunchKernelGGL(evict_select_kernel<8>, dim3(pairs), block, 0, st, a);
  else hipLaunchKernelGGL(evict_select_kernel<0>, dim3(pairs), block, 0, st, a);
  if (hipError_t e = hipGetLastError()) return e;
  const long most = (long)a.room * (a.c.d / 8);  // pieces of a pair
  long y = (most + 255) / 256;
  y = y < 1 ? 1 : (y > 64 ? 64 : y);
  hipLaunchKernelGGL(evict_move_kernel, dim3(pairs, (unsigned)y), dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace fa
