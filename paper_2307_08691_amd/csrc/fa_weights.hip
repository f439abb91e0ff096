// Attention weight per cached key: weights[s, g, c] += sum over the query heads h of group g and the queries r that see key c of
// exp(scale * q_r . k_c - L_r), from the logsumexps L that the attention pass left: the column sums of P, which that pass never
// has whole. One product and one exponential per (row, key), no second product.
//
// A row is a (query, head of the group) pair, packed as query * G + head. S = Q K^T is formed with the KEYS as columns of the MFMA
// tile: a lane then holds 16 rows of ONE key, and the sum over rows is additions inside the lane and one exchange with the partner
// lane. Every key's sum is formed by one lane in a fixed order: no atomics, the same bits in every run.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "fa_kernels.h"
#include "fa_lds.h"

namespace fa {

// Up to 32 rows (decoding): the rows stay in registers and the keys stream past. Bound by reading K once; four wavefronts that
// share nothing, each with tiles of 32 keys, the next tile requested before the current one is used.
constexpr int kStepKeys = 512;  // keys of a workgroup
template <int D, bool F16>
__global__ __launch_bounds__(256) void weights_step_kernel(WeightsArgs a) {
  constexpr int KS = D / 16;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lq = lane & 31, hh = lane >> 5;
  const int pair = blockIdx.x, s = pair / a.c.Hkv, g = pair - s * a.c.Hkv;
  const int n = held_keys(a.c, s), c0 = blockIdx.y * kStepKeys;
  int nq = a.queries ? a.queries[s] : a.Nq;
  nq = nq < a.Nq ? nq : a.Nq;
  if (c0 >= n || nq <= 0) return;
  const int rows = nq * a.G, off = n - a.Nq;
  const float c2 = a.scale * kLog2e;
  const int end = n < c0 + kStepKeys ? n : c0 + kStepKeys;

  const long kstride = (long)a.c.Hkv * D;
  bf16x8 Kr[2][KS];
  auto request = [&](int t, auto BUF) {  // tile of 32 keys from t on; keys past the end repeat the last one
    const int row = t + lq < n ? t + lq : n - 1;
    const __bf16* kp = a.K + (cache_row(a.c, s, t) + (row - t)) * kstride + (long)g * D + 8 * hh;  // (a tile lies in one page)
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) Kr[decltype(BUF)::value][ks] = *(const bf16x8*)(kp + 16 * ks);
  };
  using B0 = std::integral_constant<int, 0>;
  using B1 = std::integral_constant<int, 1>;
  int t = c0 + 32 * w;
  if (t >= end) return;
  request(t, B0{});

  bf16x8 Qf[KS];
  {
    const int row = lq < rows ? lq : rows - 1;
    const __bf16* qp = a.Q + (((long)s * a.Nq + row / a.G) * a.Hq + g * a.G + row % a.G) * D + 8 * hh;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) Qf[ks] = *(const bf16x8*)(qp + 16 * ks);
  }
  float nl[16];  // -L in the exponent's base; -inf where the register's row adds nothing
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    const int row = acc_row(r, hh), rc = row < rows ? row : rows - 1;
    const float l = a.LSE[((long)s * a.Hq + g * a.G + rc % a.G) * a.Nq + rc / a.G];
    nl[r] = row < rows && l != -INFINITY ? -l * kLog2e : -INFINITY;
  }

  float* W = a.weights + ((long)s * a.c.Hkv + g) * a.c.Nk;
  auto compute = [&](int t, auto BUF) {
    f32x16 S = (f32x16){0};
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) S = mfma32<F16>(Qf[ks], Kr[decltype(BUF)::value][ks], S);
    const int key = t + lq;
    float sum[2] = {0.f, 0.f};
    if (a.causal && t + 31 > off) {
      asm volatile("; keep this a branch" ::);
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float e = fast_exp2(__builtin_fmaf(S[r], c2, nl[r]));
        sum[r & 1] += nl[r] != -INFINITY && key <= acc_row(r, hh) / a.G + off ? e : 0.f;
      }
    } else {
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float e = fast_exp2(__builtin_fmaf(S[r], c2, nl[r]));
        sum[r & 1] += nl[r] != -INFINITY ? e : 0.f;
      }
    }
    const float total = sum_with_partner32(sum[0] + sum[1]);
    if (hh == 0 && key < end) W[key] += total;
  };
  while (true) {
    if (t + 128 < end) request(t + 128, B1{});
    compute(t, B0{});
    if ((t += 128) >= end) break;
    if (t + 128 < end) request(t + 128, B0{});
    compute(t, B1{});
    if ((t += 128) >= end) break;
  }
}

// More rows: a wavefront holds 64 keys in registers and the rows stream past in tiles of 64, which the workgroup's four wavefronts
// (256 keys) share through LDS, one tile ahead. Bound by the exponentials. Under the causal rule tiles above the keys are not
// visited, and the blocks of keys with the most rows are handed out first.
constexpr int kPromptKeys = 256;
template <int D, bool F16>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2))) void weights_prompt_kernel(WeightsArgs a) {
  constexpr int KS = D / 16, ROWB = 2 * D, BR = 64, TILEB = BR * ROWB, CPR = ROWB / 16, RPI = 64 / CPR;
  __shared__ __attribute__((aligned(1024))) char smem[2 * TILEB + 2 * BR * 4];
  float* const stat = (float*)(smem + 2 * TILEB);
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), lq = lane & 31, hh = lane >> 5;
  const int pair = blockIdx.x, s = pair / a.c.Hkv, g = pair - s * a.c.Hkv;
  const int n = held_keys(a.c, s), c0 = blockIdx.y * kPromptKeys;
  int nq = a.queries ? a.queries[s] : a.Nq;
  nq = nq < a.Nq ? nq : a.Nq;
  if (c0 >= n || nq <= 0) return;
  const int rows = nq * a.G, off = n - a.Nq;
  const float c2 = a.scale * kLog2e;
  const int kb = c0 + 64 * w;  // this wavefront's keys
  bf16x8 Kr[2][KS];
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    int key = kb + 32 * u + lq;
    key = key < n ? key : n - 1;
    const __bf16* kp = a.K + (cache_row(a.c, s, key) * a.c.Hkv + g) * D + 8 * hh;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) Kr[u][ks] = *(const bf16x8*)(kp + 16 * ks);
  }
  const int q_first = a.causal && c0 > off ? c0 - off : 0;  // the first query that sees a key of the block
  const int tiles = (rows + BR - 1) / BR, t_first = (int)((long)q_first * a.G / BR);
  const __bf16* Qb = a.Q + ((long)s * a.Nq * a.Hq + g * a.G) * D;
  const float* Lb = a.LSE + ((long)s * a.Hq + g * a.G) * a.Nq;
  auto copy = [&](int t, int buf) {
#pragma unroll
    for (int u = 0; u < BR / RPI / 4; ++u) {
      const int rb = (w + 4 * u) * RPI, r = rb + lane / CPR, ch = (lane % CPR) ^ swz<ROWB>(r);
      int row = t * BR + r;
      row = row < rows ? row : rows - 1;
      const int q = row / a.G;
      dma16(Qb + ((long)q * a.Hq + (row - q * a.G)) * D + 8 * ch, smem + buf * TILEB + rb * ROWB);
    }
  };
  auto row_stat = [&](int t) {  // (threads 0 .. 63)
    const int row = t * BR + tid;
    if (tid >= BR || row >= rows) return -INFINITY;
    const int q = row / a.G;
    const float l = Lb[(long)(row - q * a.G) * a.Nq + q];
    return l != -INFINITY ? -l * kLog2e : -INFINITY;
  };
  float sum[2][2] = {{0.f, 0.f}, {0.f, 0.f}};
  const int zrow = lq * ROWB + 16 * (hh ^ swz<ROWB>(lq));
  if (t_first < tiles) {
    const float x = row_stat(t_first);
    if (tid < BR) stat[tid] = x;
    copy(t_first, 0);
  }
#pragma unroll
  for (int u = 0; u < 2; ++u)
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) touch(Kr[u][ks]);
  for (int t = t_first, buf = 0; t < tiles; ++t, buf ^= 1) {
    wait_vmem();
    lds_barrier();  // tile t has landed, everyone is done with the one before it
    float next = 0.f;
    if (t + 1 < tiles) {
      next = row_stat(t + 1);
      copy(t + 1, buf ^ 1);
    }
    const int q0 = t * BR / a.G, q1 = (t * BR + BR - 1) / a.G;
    if (!a.causal || q1 + off >= kb) {  // (else none of these rows sees any of these keys)
      const bool all = !a.causal || q0 + off >= kb + 63;
#pragma unroll
      for (int rt = 0; rt < 2; ++rt) {
        f32x16 S[2] = {(f32x16){0}, (f32x16){0}};
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          const bf16x8 q = lds_b128(smem, ((zrow + buf * TILEB) ^ (32 * ks)) + rt * 32 * ROWB);
          S[0] = mfma32<F16>(q, Kr[0][ks], S[0]);
          S[1] = mfma32<F16>(q, Kr[1][ks], S[1]);
        }
        f32x4 nl[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) nl[i] = *(const f32x4*)(stat + buf * BR + 32 * rt + 8 * i + 4 * hh);
        if (all) {
#pragma unroll
          for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int r = 0; r < 16; ++r) sum[u][r & 1] += fast_exp2(__builtin_fmaf(S[u][r], c2, nl[r / 4][r % 4]));
        } else {
          asm volatile("; keep this a branch" ::);
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int last = (t * BR + 32 * rt + acc_row(r, hh)) / a.G + off;  // the last key that the row sees
#pragma unroll
            for (int u = 0; u < 2; ++u) {
              const float e = fast_exp2(__builtin_fmaf(S[u][r], c2, nl[r / 4][r % 4]));
              sum[u][r & 1] += nl[r / 4][r % 4] != -INFINITY && kb + 32 * u + lq <= last ? e : 0.f;
            }
          }
        }
      }
    }
    if (t + 1 < tiles && tid < BR) stat[(buf ^ 1) * BR + tid] = next;
  }
  float* W = a.weights + ((long)s * a.c.Hkv + g) * a.c.Nk;
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const float total = sum_with_partner32(sum[u][0] + sum[u][1]);
    const int key = kb + 32 * u + lq;
    if (hh == 0 && key < n) W[key] += total;
  }
}

template <int D, bool F16>
static hipError_t launch_weights_d(const WeightsArgs& a, hipStream_t st) {
  const unsigned pairs = (unsigned)(a.nseq * a.c.Hkv);
  if ((long)a.Nq * a.G <= 32)
    hipLaunchKernelGGL((weights_step_kernel<D, F16>), dim3(pairs, (unsigned)((a.c.Nk + kStepKeys - 1) / kStepKeys)), dim3(256), 0, st, a);
  else
    hipLaunchKernelGGL((weights_prompt_kernel<D, F16>), dim3(pairs, (unsigned)((a.c.Nk + kPromptKeys - 1) / kPromptKeys)), dim3(256), 0, st, a);
  return hipGetLastError();
}
hipError_t launch_weights(const WeightsArgs& a, hipStream_t st) {
  if (a.c.d == 64) return a.f16 ? launch_weights_d<64, true>(a, st) : launch_weights_d<64, false>(a, st);
  return a.f16 ? launch_weights_d<128, true>(a, st) : launch_weights_d<128, false>(a, st);
}

}  // namespace fa
