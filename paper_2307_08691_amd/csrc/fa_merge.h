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

}  // namespace fa
