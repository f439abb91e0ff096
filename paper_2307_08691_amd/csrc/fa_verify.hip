// Drafted tokens against the target's probabilities. Draft i of a sequence is accepted iff all before it were and
// u_i q_i(x_i) < p_i(x_i). At the first that is not (or has no token) the sequence goes on with a token drawn from max(p_i - q_i, 0),
// behind k accepted ones with one drawn from p_k: the lowest token whose running sum exceeds u_k times the total.
//
// A running sum over 100 000 probabilities passes a random number at another token if it is off by 1e-7, so everything that is
// summed to draw is held in float64, whatever order it is summed in. The target's logits need their normaliser first: row maxima
// and float32 sums over all rows settle which drafts are accepted (one whose u q lies within 1e-6 of p may be taken the other way, which
// changes its odds by as little); the one row that is drawn from is then summed once more in float64.
//
//   stats   (logits) maximum and sum of every row, in segments of kSegment tokens, one a wavefront: bound by HBM
//   sums    per sequence: which drafts are accepted (every workgroup finds out for itself: cheaper than a launch); float64 sums of
//           the segments of the row that is drawn from
//   draw    per sequence: the segment in which the running sum passes, then the token in it: a chain of latencies
#include <hip/hip_runtime.h>

#include <cfloat>

#include "../../include/fa.h"
#include "fa_kernels.h"

namespace fa {

constexpr int kSegment = 2048, kVerifyThreads = 256, kVerifyWaves = kVerifyThreads / 64;
constexpr int kPieces = kSegment / 64 / 8;  // pieces of eight tokens of a lane: (64 i + lane) of the segment

struct SegmentSums {
  // p: sum of the segment's weights. above, drafts: sums of p and of q over its tokens with p > q. For logits p and above are sums
  // of exp(inv_t (l - maximum)), to be divided by the row's whole sum.
  double p, above, drafts;
};
struct RowPart {
  float max, sum;
};
__host__ __device__ inline int segments_of(int V) { return (V + kSegment - 1) / kSegment; }

// What the drafted token of a row has: the target's value, the draft model's probability (less than 0: there is no such token).
struct Picked {
  float target, draft;
};

size_t verify_workspace(int B, int k, int V) {
  return (size_t)B * (segments_of(V) * (sizeof(SegmentSums) + (size_t)(k + 1) * sizeof(RowPart)) + (size_t)(k + 1) * sizeof(Picked) + sizeof(float));
}
__device__ __forceinline__ SegmentSums* segment_sums(const VerifyArgs& a, long b) { return (SegmentSums*)a.ws + b * segments_of(a.V); }
__device__ __forceinline__ RowPart* row_parts(const VerifyArgs& a, long row) {
  const int n = segments_of(a.V);
  return (RowPart*)((SegmentSums*)a.ws + (long)a.nseq * n) + row * n;
}
__device__ __forceinline__ Picked* picked(const VerifyArgs& a) { return (Picked*)row_parts(a, (long)a.nseq * (a.k + 1)); }

__device__ __forceinline__ float* drawn_maxima(const VerifyArgs& a) { return (float*)(picked(a) + (long)a.nseq * (a.k + 1)); }  // of the rows that are drawn from

__device__ __forceinline__ float element(const void* p, int type, long i) {
  if (type == FA_TYPE_F32) return ((const float*)p)[i];
  if (type == FA_TYPE_BF16) return (float)((const __bf16*)p)[i];
  return (float)((const _Float16*)p)[i];
}
// Eight values from element i on, those from `n` on replaced by `none`. (16-byte loads at any element's address: rows may begin anywhere.)
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
typedef __bf16 bf16x8_any __attribute__((ext_vector_type(8), aligned(2)));
typedef _Float16 f16x8_any __attribute__((ext_vector_type(8), aligned(2)));
__device__ __forceinline__ void eight(const void* p, int type, long i, int n, float none, float (&x)[8]) {
  if (n >= 8) {
    if (type == FA_TYPE_F32) {
      const f32x4_any lo = *(const f32x4_any*)((const float*)p + i), hi = *(const f32x4_any*)((const float*)p + i + 4);
#pragma unroll
      for (int u = 0; u < 8; ++u) x[u] = u < 4 ? lo[u & 3] : hi[u & 3];
    } else if (type == FA_TYPE_BF16) {
      const bf16x8_any v = *(const bf16x8_any*)((const __bf16*)p + i);
#pragma unroll
      for (int u = 0; u < 8; ++u) x[u] = (float)v[u];
    } else {
      const f16x8_any v = *(const f16x8_any*)((const _Float16*)p + i);
#pragma unroll
      for (int u = 0; u < 8; ++u) x[u] = (float)v[u];
    }
  } else {
#pragma unroll
    for (int u = 0; u < 8; ++u) x[u] = u < n ? element(p, type, i + u) : none;
  }
}

// Over the lanes of a wavefront (all active) with data-parallel moves, which take a few cycles where a permutation through LDS takes a
// hundred: each step adds the lane 1, 2, 4, 8 below in its row of 16, then the last lane of the rows below.
template <int CTRL, int ROWS, class T>
__device__ __forceinline__ T from_below(T x, T none) {  // `none` where there is no such lane
  static_assert(sizeof(T) == 4 || sizeof(T) == 8, "");
  constexpr int W = sizeof(T) / 4;
  int v[W], o[W];
  __builtin_memcpy(v, &x, sizeof(T));
  __builtin_memcpy(o, &none, sizeof(T));
#pragma unroll
  for (int i = 0; i < W; ++i) v[i] = __builtin_amdgcn_update_dpp(o[i], v[i], CTRL, ROWS, 0xf, false);
  __builtin_memcpy(&x, v, sizeof(T));
  return x;
}
template <class T, class F>
__device__ __forceinline__ T wave_fold(T x, T none, F f) {  // of the lanes up to this one
  x = f(x, from_below<0x111, 0xf>(x, none));
  x = f(x, from_below<0x112, 0xf>(x, none));
  x = f(x, from_below<0x114, 0xf>(x, none));
  x = f(x, from_below<0x118, 0xf>(x, none));
  x = f(x, from_below<0x142, 0xa>(x, none));
  return f(x, from_below<0x143, 0xc>(x, none));
}
template <class T>
__device__ __forceinline__ T in_lane(T x, int lane) {
  constexpr int W = sizeof(T) / 4;
  int v[W];
  __builtin_memcpy(v, &x, sizeof(T));
#pragma unroll
  for (int i = 0; i < W; ++i) v[i] = __builtin_amdgcn_readlane(v[i], lane);
  __builtin_memcpy(&x, v, sizeof(T));
  return x;
}
template <class T>
__device__ __forceinline__ T wave_scan(T x) {  // sum of the lanes up to this one
  return wave_fold(x, (T)0, [](T u, T v) { return u + v; });
}
template <class T>
__device__ __forceinline__ T wave_add(T x) {
  return in_lane(wave_scan(x), 63);
}
__device__ __forceinline__ float wave_max(float x) {
  return in_lane(wave_fold(x, -INFINITY, [](float u, float v) { return fmaxf(u, v); }), 63);
}
__device__ __forceinline__ int wave_max(int x) {
  return in_lane(wave_fold(x, -0x7fffffff - 1, [](int u, int v) { return max(u, v); }), 63);
}

__device__ __forceinline__ int draft_token(const VerifyArgs& a, long b, int i) {  // -1: none
  const int x = i < a.k ? a.drafts[b * a.k + i] : -1;
  return x >= 0 && x < a.V ? x : -1;
}
__device__ __forceinline__ Picked pick(const VerifyArgs& a, long b, int i) {
  const int x = draft_token(a, b, i);
  if (x < 0) return {0.f, -1.f};
  return {element(a.target, a.target_type, (b * (a.k + 1) + i) * a.target_stride + x),
          a.q ? element(a.q, a.q_type, (b * a.k + i) * a.q_stride + x) : 1.f};
}

template <int TYPE>
__global__ __launch_bounds__(kVerifyThreads) void verify_stats_kernel(VerifyArgs a) {
  const long row = blockIdx.x;
  const int lane = threadIdx.x & 63, seg = blockIdx.y * kVerifyWaves + (threadIdx.x >> 6), c0 = seg * kSegment;
  if (seg >= segments_of(a.V)) return;
  const float t2 = fminf(a.inv_t * kLog2e, FLT_MAX);  // (finite: the maximum itself is 0 of it)
  float x[kPieces][8], m = -INFINITY;
  if (c0 + kSegment <= a.V) {  // (a branch of the whole wavefront: its loads are then requested together)
#pragma unroll
    for (int i = 0; i < kPieces; ++i) eight(a.target, TYPE, row * a.target_stride + c0 + (64 * i + lane) * 8, 8, -INFINITY, x[i]);
  } else {
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const int j = c0 + (64 * i + lane) * 8;
      eight(a.target, TYPE, row * a.target_stride + j, a.V - j, -INFINITY, x[i]);
    }
  }
#pragma unroll
  for (int i = 0; i < kPieces; ++i)
#pragma unroll
    for (int u = 0; u < 8; ++u) m = fmaxf(m, x[i][u]);
  m = wave_max(m);
  float z[2] = {0.f, 0.f};
#pragma unroll
  for (int i = 0; i < kPieces; ++i)
#pragma unroll
    for (int u = 0; u < 8; ++u) z[u & 1] += x[i][u] == -INFINITY ? 0.f : fast_exp2((x[i][u] - m) * t2);
  const float sum = wave_add(z[0] + z[1]);
  if (lane == 0) row_parts(a, row)[seg] = {m, sum};
  // (here they are a latency beside others, in the next kernel two in front of everything)
  if (seg == 0 && lane == 0) picked(a)[row] = pick(a, row / (a.k + 1), (int)(row % (a.k + 1)));
}

// Maximum of a row, and its sum against it (by a wavefront), from `mine`, this lane's segment of the first 64.
__device__ __forceinline__ RowPart first_part(const VerifyArgs& a, long row) {
  const int lane = threadIdx.x & 63;
  return lane < segments_of(a.V) ? row_parts(a, row)[lane] : RowPart{-INFINITY, 0.f};
}
__device__ __forceinline__ RowPart whole_row(const VerifyArgs& a, long row, RowPart mine) {
  const RowPart* part = row_parts(a, row);
  const int n = segments_of(a.V), lane = threadIdx.x & 63;
  float m = mine.max;
  for (int i = 64 + lane; i < n; i += 64) m = fmaxf(m, part[i].max);
  m = wave_max(m);
  float z = 0.f;
  auto take = [&](RowPart p) { z += p.max == -INFINITY ? 0.f : p.sum * fast_exp2((p.max - m) * a.inv_t * kLog2e); };
  take(mine);
  for (int i = 64 + lane; i < n; i += 64) take(part[i]);
  return {m, wave_add(z)};
}
// exp(inv_t (l - m)) in float64: with y = inv_t log2(e) (l - m), the difference first (the maximum's own weight is then 1 whatever inv_t
// is; the difference of two products would be off by 2^-53 of them, which counts from about 10^13 on), and n the whole number next to
// it (the low bits of y + 1.5 * 2^52), 2^n times the polynomial of degree 8 that meets 2^f at the nine Chebyshev points of [-1/2, 1/2], f = y - n: off by at most 1.1e-12 of
// its value, by which a draw over 10^5 tokens is decided otherwise once in some 10^6. n goes into the exponent's bits. Less than
// 2^-1000 is 0. (64 rows of 131072: 19.6 us with a Taylor series of eleven terms, rint and ldexp and reductions through LDS, 16.9 so.)
struct Exponential {
  double c, m;
  __device__ __forceinline__ Exponential(float inv_t, float max)
      : c((double)inv_t * 1.4426950408889634074), m(max == -INFINITY ? 0. : (double)max) {}  // (a row of -inf alone: all are 0)
  __device__ __forceinline__ double operator()(float l) const {
    constexpr double whole = 6755399441055744.;
    const double y = c * ((double)l - m), t = y + whole, f = y - (t - whole);
    double s = 0x1.63d1363a681b4p-20;
    s = __builtin_fma(s, f, 0x1.00dc4a5344ef5p-16);
    s = __builtin_fma(s, f, 0x1.4308ac85a69f8p-13);
    s = __builtin_fma(s, f, 0x1.5d8745a728209p-10);
    s = __builtin_fma(s, f, 0x1.3b2ab7181b77dp-7);
    s = __builtin_fma(s, f, 0x1.c6b08dd6fd236p-5);
    s = __builtin_fma(s, f, 0x1.ebfbdff823cedp-3);
    s = __builtin_fma(s, f, 0x1.62e42fef84cf0p-1);
    s = __builtin_fma(s, f, 1.);
    const uint64_t bits = __builtin_bit_cast(uint64_t, s) + (__builtin_bit_cast(uint64_t, t) << 52);
    return y < -1000. ? 0. : __builtin_bit_cast(double, bits);
  }
};
constexpr int kCertain = 3;  // in the place of a type: the drafts are certain
// What the draft model gave the tokens of row (b, i); 0 where nothing is to be taken off.
struct DraftRow {
  const void* q;
  int token;  // q == nullptr: all on `token` (-1: nothing)
  long at;
  template <int QTYPE>
  __device__ __forceinline__ void of(int j, int n, float (&d)[8]) const {
    if (QTYPE != kCertain && q) return eight(q, QTYPE, at + j, n, 0.f, d);
#pragma unroll
    for (int u = 0; u < 8; ++u) d[u] = j + u == token ? 1.f : 0.f;
  }
};
__device__ __forceinline__ DraftRow draft_row(const VerifyArgs& a, long b, int i) {
  const int x = draft_token(a, b, i);
  if (x < 0 || !a.q) return {nullptr, x, 0};
  return {a.q, x, (b * a.k + i) * a.q_stride};
}

template <int TYPE, int QTYPE>
__global__ __launch_bounds__(kVerifyThreads) void verify_sums_kernel(VerifyArgs a) {
  __shared__ int first;  // the first draft that is not accepted (k: none)
  __shared__ RowPart rows[kVerifyWaves];
  const long b = blockIdx.x;
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  // Four drafts at a time, a wavefront each, until one is not accepted. (What the last row needs is on its way meanwhile.)
  if (threadIdx.x == 0) first = a.k;
  const long row0 = b * (a.k + 1);
  RowPart r = {0.f, 1.f}, last = r;
  if (a.logits) last = first_part(a, row0 + a.k);
  __syncthreads();
  for (int i0 = 0; i0 < a.k; i0 += kVerifyWaves) {
    const int i = i0 + w;
    if (i < a.k) {
      const double u = (double)a.uniform[row0 + i];
      const Picked x = a.logits ? picked(a)[row0 + i] : pick(a, b, i);
      if (a.logits) r = whole_row(a, row0 + i, first_part(a, row0 + i));
      const double p = a.logits ? Exponential(a.inv_t, r.max)(x.target) / (double)r.sum : (double)x.target;
      if (lane == 0) {
        rows[w] = r;
        if (!(x.draft >= 0.f && u * (double)x.draft < p)) atomicMin(&first, i);
      }
    }
    __syncthreads();
    if (first < a.k) break;
    __syncthreads();  // (the rows' sums are written again)
  }
  const int i = first;
  if (i < a.k) r = rows[i % kVerifyWaves];
  else if (a.logits) r = whole_row(a, row0 + a.k, last);
  const int seg = blockIdx.y * kVerifyWaves + w, c0 = seg * kSegment;
  if (blockIdx.y == 0) {  // the tokens so far
    if (threadIdx.x == 0) {
      a.accepted[b] = i;
      drawn_maxima(a)[b] = r.max;
    }
    for (int j = threadIdx.x; j <= a.k; j += kVerifyThreads) a.tokens[b * (a.k + 1) + j] = j < i ? a.drafts[b * a.k + j] : -1;
  }
  if (c0 >= a.V) return;
  const DraftRow q = draft_row(a, b, i);
  const long at = (b * (a.k + 1) + i) * a.target_stride;
  const double inv = a.logits ? 1. / (double)r.sum : 1.;
  const Exponential weight(a.inv_t, r.max);
  double sp = 0., sa = 0., sq = 0.;
  // A loop, though it is short: in straight code the wavefronts wait for instructions, which each of them runs once (us of this launch,
  // unrolled and so: 5 rows of 9400 7.1 and 6.5; 59 x 3 of 43057 11.3 and 11.2; 64 x 5 of 131072 17.0 and 16.9).
  float l[8], d[8];
  auto request = [&](int piece) {
    const int j = c0 + (64 * piece + lane) * 8;
    eight(a.target, TYPE, at + j, a.V - j, a.logits ? -INFINITY : 0.f, l);
    q.of<QTYPE>(j, a.V - j, d);
  };
  request(0);
#pragma unroll 1
  for (int piece = 0; piece < kPieces; ++piece) {
    float x[8], y[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) x[u] = l[u], y[u] = d[u];
    if (piece + 1 < kPieces) request(piece + 1);
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const double p = a.logits ? weight(x[u]) : (double)x[u];
      sp += p;
      // (r.sum is good to 1e-7: a token at which that decides has p = q to within it, and adds as little either way)
      const double more = p * inv > (double)y[u] ? 1. : 0.;
      sa = __builtin_fma(p, more, sa);
      sq = __builtin_fma((double)y[u], more, sq);
    }
  }
  sp = wave_add(sp);
  sa = wave_add(sa);
  sq = wave_add(sq);
  if (lane == 0) segment_sums(a, b)[seg] = {sp, sa, sq};
}

template <int TYPE, int QTYPE>
__global__ __launch_bounds__(kVerifyThreads) void verify_draw_kernel(VerifyArgs a) {
  __shared__ double sums[kVerifyWaves];
  __shared__ int least[kVerifyWaves], most[kVerifyWaves];
  const long b = blockIdx.x;
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, n = segments_of(a.V), i = a.accepted[b];
  const long row = b * (a.k + 1) + i;
  const double u = (double)a.uniform[b * (a.k + 1) + a.k];
  const DraftRow q = draft_row(a, b, i);
  // (every wavefront for itself)
  const SegmentSums* part = segment_sums(a, b);
  const float row_max = drawn_maxima(a)[b];
  double z = 0., above = 0., off = 0.;
  for (int c = lane; c < n; c += 64) z += part[c].p, above += part[c].above, off += part[c].drafts;
  z = wave_add(z);
  above = wave_add(above);
  off = wave_add(off);
  const double inv = a.logits ? 1. / z : 1.;
  const bool residual = above * inv - off > 0.;  // whether p - q leaves anything
  const double want = u * (residual ? above * inv - off : z * inv);
  // the first segment whose end lies past `want`, or else the last one that adds anything; and what lies before it
  int seg = -1;
  double base = 0., done = 0.;
  for (int c0 = 0; c0 < n; c0 += 64) {
    const int c = c0 + lane;
    double x = c >= n ? 0. : residual ? part[c].above * inv - part[c].drafts : part[c].p * inv;
    x = x > 0. ? x : 0.;
    const double sum = done + wave_scan(x);
    const unsigned long long some = __builtin_amdgcn_ballot_w64(x > 0.), past = __builtin_amdgcn_ballot_w64(x > 0. && sum > want);
    if (some) {
      const int at = past ? __builtin_ctzll(past) : 63 - __builtin_clzll(some);
      seg = c0 + at;
      base = in_lane(sum - x, at);
    }
    if (past) break;
    done = in_lane(sum, 63);
  }
  if (seg < 0) return;  // (nothing to draw from: the token stays -1)
  // each thread: eight tokens that follow each other
  const Exponential weight(a.inv_t, row_max);
  const int j0 = seg * kSegment + tid * 8;
  float l[8], d[8];
  double x[8], mine = 0.;
  eight(a.target, TYPE, row * a.target_stride + j0, a.V - j0, a.logits ? -INFINITY : 0.f, l);
  q.of<QTYPE>(j0, a.V - j0, d);
  int last = -1, hit = 0x7fffffff;  // the last one that adds anything, the first one past `want`
#pragma unroll
  for (int v = 0; v < 8; ++v) {
    const double p = (a.logits ? weight(l[v]) : (double)l[v]) * inv, dv = residual ? (double)d[v] : 0.;
    x[v] = p > dv ? p - dv : 0.;
    mine += x[v];
    if (x[v] > 0.) last = j0 + v;
  }
  double run = wave_scan(mine);
  if (lane == 63) sums[w] = run;
  __syncthreads();
  run += base - mine;
  for (int v = 0; v < w; ++v) run += sums[v];
#pragma unroll
  for (int v = 0; v < 8; ++v) {
    run += x[v];
    if (x[v] > 0. && run > want && hit == 0x7fffffff) hit = j0 + v;
  }
  last = wave_max(last);
  hit = -wave_max(-hit);
  if (lane == 0) {
    least[w] = hit;
    most[w] = last;
  }
  __syncthreads();
  if (tid == 0) {
    for (int v = 1; v < kVerifyWaves; ++v) {
      hit = min(hit, least[v]);
      last = max(last, most[v]);
    }
    a.tokens[row] = hit != 0x7fffffff ? hit : last;
  }
}

template <int TYPE, int QTYPE>
static hipError_t launch_verify_as(const VerifyArgs& a, hipStream_t st) {
  const unsigned parts = (unsigned)((segments_of(a.V) + kVerifyWaves - 1) / kVerifyWaves);
  const dim3 block(kVerifyThreads);
  if (a.logits) {
    hipLaunchKernelGGL(verify_stats_kernel<TYPE>, dim3((unsigned)(a.nseq * (a.k + 1)), parts), block, 0, st, a);
    if (hipError_t e = hipGetLastError()) return e;
  }
  hipLaunchKernelGGL((verify_sums_kernel<TYPE, QTYPE>), dim3((unsigned)a.nseq, parts), block, 0, st, a);
  if (hipError_t e = hipGetLastError()) return e;
  hipLaunchKernelGGL((verify_draw_kernel<TYPE, QTYPE>), dim3((unsigned)a.nseq), block, 0, st, a);
  return hipGetLastError();
}
template <int TYPE>
static hipError_t launch_verify_t(const VerifyArgs& a, hipStream_t st) {
  if (!a.q) return launch_verify_as<TYPE, kCertain>(a, st);
  if (a.q_type == FA_TYPE_F32) return launch_verify_as<TYPE, FA_TYPE_F32>(a, st);
  return a.q_type == FA_TYPE_BF16 ? launch_verify_as<TYPE, FA_TYPE_BF16>(a, st) : launch_verify_as<TYPE, FA_TYPE_F16>(a, st);
}
hipError_t launch_verify(const VerifyArgs& a, hipStream_t st) {
  if (a.target_type == FA_TYPE_F32) return launch_verify_t<FA_TYPE_F32>(a, st);
  return a.target_type == FA_TYPE_BF16 ? launch_verify_t<FA_TYPE_BF16>(a, st) : launch_verify_t<FA_TYPE_F16>(a, st);
}

}  // namespace fa
