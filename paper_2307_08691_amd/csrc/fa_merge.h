// Partial results of shares of a row's keys (normalised partial O and logsumexp, float32), joined by the identity section 3.1.1 uses
// between blocks: O = sum_k exp(L_k - L) O_k, L = log sum_k exp(L_k).
#pragma once
#include "fa_common.h"

namespace fa {

// Workgroups of 256, one thread per four elements of a (token, head) row: Opart [slot][rows][D], Lpart [slot][rows], rows = tokens * Hq,
// tokens of one sequence after the other, Nq each. Few threads a row and a handful of slots: the time is the chain of loads, so
// the logsumexps and partial rows of FLY slots are requested together, and where there are no more than that none is read twice.
// (A slot without keys for this row has written no partial O: what is read in its place is not used.)
template <int D, bool F16, int FLY>
__device__ __forceinline__ void merge_slots(const float* Opart, const float* Lpart, __bf16* O, float* LSE, long all, int Hq, int Nq, int slots) {
  constexpr int TPR = D / 4;
  const long r = (long)blockIdx.x * (256 / TPR) + threadIdx.x / TPR;
  if (r >= all) return;
  const int c = threadIdx.x % TPR;
  float l[FLY], mx = -INFINITY;
  f32x4 o[FLY];
  auto request = [&](int k0) {
#pragma unroll
    for (int u = 0; u < FLY; ++u) l[u] = Lpart[(k0 + u < slots ? k0 + u : slots - 1) * all + r];
#pragma unroll
    for (int u = 0; u < FLY; ++u) o[u] = *(const f32x4*)(Opart + ((k0 + u < slots ? k0 + u : slots - 1) * all + r) * D + 4 * c);
  };
  request(0);
  for (int k = FLY; k < slots; ++k) mx = max_or_nan(mx, Lpart[k * all + r]);
#pragma unroll
  for (int u = 0; u < FLY; ++u) mx = max_or_nan(mx, l[u]);
  const long tok = r / Hq;
  const int h = (int)(r - tok * Hq);
  const long s = tok / Nq;
  float* lse = LSE + (s * Hq + h) * Nq + (tok - s * Nq);
  if (mx == -INFINITY) {  // no key anywhere
    *(u32x2*)(O + r * D + 4 * c) = (u32x2){0u, 0u};
    if (c == 0) *lse = -INFINITY;
    return;
  }
  float z = 0.f;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  for (int k0 = 0;;) {
#pragma unroll
    for (int u = 0; u < FLY; ++u) {
      if (k0 + u >= slots || l[u] == -INFINITY) continue;
      const float wgt = __expf(l[u] - mx);
      z += wgt;
      acc += o[u] * wgt;
    }
    if ((k0 += FLY) >= slots) break;
    request(k0);
  }
  const float inv = 1.f / z;
  u32x2 x;
  x[0] = pack2<F16>(acc[0] * inv, acc[1] * inv);
  x[1] = pack2<F16>(acc[2] * inv, acc[3] * inv);
  *(u32x2*)(O + r * D + 4 * c) = x;
  if (c == 0) *lse = mx + __logf(z);
}

// The same for one row whose partial results lie anywhere: partial(k) is where slot k's is, logsum(k) its logsumexp, done(c, o, lse) takes elements
// 4 c .. 4 c + 3. A thread has four elements (c: threadIdx.x modulo D / 4), and FLY slots on their way.
template <int D, int FLY, class P, class L, class F>
__device__ __forceinline__ void merge_few(int slots, P partial, L logsum, F done) {
  const int c = threadIdx.x % (D / 4);
  float mx = -INFINITY, z = 0.f;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  for (int k0 = 0; k0 < slots; k0 += FLY) {
    float l[FLY];
    f32x4 o[FLY];
#pragma unroll
    for (int u = 0; u < FLY; ++u) {
      const int k = k0 + u < slots ? k0 + u : slots - 1;
      l[u] = logsum(k);
      o[u] = *(const f32x4*)(partial(k) + 4 * c);
    }
    float m_new = mx;
#pragma unroll
    for (int u = 0; u < FLY; ++u) m_new = max_or_nan(m_new, l[u]);
    if (m_new == -INFINITY) continue;
    const float alpha = __expf(mx - m_new);  // (0 where nothing has come before)
    z *= alpha;
    acc *= alpha;
#pragma unroll
    for (int u = 0; u < FLY; ++u) {
      if (k0 + u >= slots || l[u] == -INFINITY) continue;
      const float wgt = __expf(l[u] - m_new);
      z += wgt;
      acc += o[u] * wgt;
    }
    mx = m_new;
  }
  if (mx == -INFINITY) done(c, (f32x4){0.f, 0.f, 0.f, 0.f}, -INFINITY);  // no key anywhere
  else done(c, acc * (1.f / z), mx + __logf(z));
}

// ... by a whole workgroup of 256, for many slots: groups of D / 4 threads take them in turn, each with a running maximum of its own, and
// join through LDS. (One sequence, 32 heads, 94 slots of 128 columns: 27 us by merge_slots, whose four workgroups go over the slots one
// after the other, 5.2 us so.)
template <int D>
constexpr int merge_split_lds() { return 256 * 16 + (1024 / D) * 4; }
template <int D, class P, class L, class F>
__device__ __forceinline__ void merge_split(char* smem, int slots, P partial, L logsum, F done) {
  constexpr int TPR = D / 4, NG = 256 / TPR;
  f32x4* const part = (f32x4*)smem;  // [NG][TPR]
  float* const top = (float*)(smem + 256 * 16);
  const int g = threadIdx.x / TPR;
  merge_few<D, 4>(slots > g ? (slots - g + NG - 1) / NG : 0, [&](int k) { return partial(g + NG * k); }, [&](int k) { return logsum(g + NG * k); },
                  [&](int c, f32x4 o, float lse) {
                    part[g * TPR + c] = o;
                    if (c == 0) top[g] = lse;
                  });
  __syncthreads();
  if (g != 0) return;
  const int c = threadIdx.x;
  float mx = -INFINITY, z = 0.f;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int u = 0; u < NG; ++u) mx = max_or_nan(mx, top[u]);
  if (mx == -INFINITY) return done(c, acc, -INFINITY);
#pragma unroll
  for (int u = 0; u < NG; ++u) {
    if (top[u] == -INFINITY) continue;
    const float wgt = __expf(top[u] - mx);
    z += wgt;
    acc += part[u * TPR + c] * wgt;
  }
  done(c, acc * (1.f / z), mx + __logf(z));
}

}  // namespace fa
