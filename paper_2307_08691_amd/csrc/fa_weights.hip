// Attention weight per cached key: weights[s, g, c] += sum over the query heads h of group g and the queries r that see key c of
// exp(scale * q_r . k_c - L_r), from the logsumexps L that the attention pass left: the column sums of P, which that pass never
// has whole. One product and one exponential per (row, key), no second product.
//
// A row is a (query, head of the group) pair, packed as query * G + head. Every key's sum is formed in a fixed order: no atomics, the
// same bits in every run.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "fa_kernels.h"
#include "fa_lds.h"

namespace fa {

// A workgroup's (sequence, key/value head): the heads of a sequence follow each other on ONE XCD, and eight sequences are under way on
// the eight. Heads lie side by side in memory, a row of each after the other: (64 sequences of up to 8192 keys, 8 heads of 128: 99 us
// with a head to an XCD, 95 so; 96 of up to 2048, heads of 64: 26.7 and 25.3.) The sequences past the last eight: as they come.
__device__ __forceinline__ void pair_of(int i, int nseq, int heads, int& s, int& g) {
  const int set = kXcds * heads, whole = nseq / kXcds * set;
  if (i < whole) {
    const int in = i % set;
    s = i / set * kXcds + in % kXcds;
    g = in / kXcds;
  } else {
    s = i / heads;
    g = i % heads;
  }
}

// A workgroup's block of keys: grids hold 65535 of them along one axis, long caches have more.
constexpr long kBlocksY = 32768;
__device__ __forceinline__ int block_of_keys() { return (int)(blockIdx.z * gridDim.y + blockIdx.y); }
static dim3 grid_of(unsigned pairs, long blocks) {
  return dim3(pairs, (unsigned)(blocks < kBlocksY ? blocks : kBlocksY), (unsigned)((blocks + kBlocksY - 1) / kBlocksY));
}

// Few rows (decoding): the rows stay in registers and the keys stream past, in tiles of 32 that each of a workgroup's four wavefronts
// takes in turn: whole rows into a private piece of LDS, two tiles on their way. (A lane that loads its own key's row straight into
// registers makes every request touch 64 places: 107 us, 4.5 TB/s, for 64 sequences of up to 8192 keys, 32 heads on 8 of 128, where
// this takes 96, 5.0 TB/s; a kernel that only reads 4 GiB: 6.25.) S = Q K^T is formed with the KEYS as columns of the MFMA tile: a lane then holds 16
// rows of ONE key, and the sum over rows is additions inside the lane and one exchange with the partner lane. Bound by reading K once.
// What the rows and the slots have is requested beside the pages, before the first tile: memory answers in order, and what is
// requested behind a tile waits for it. For the same reason the sums are written when all tiles have come.
constexpr int kStepKeys = 512;  // of a workgroup at most
template <int D, bool F16>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(D == 64 ? 4 : 2))) void weights_step_kernel(WeightsArgs a, int keys) {  // keys: of a workgroup, a multiple of 128
  constexpr int KS = D / 16, NW = 4, ROWB = 2 * D, TILEB = 32 * ROWB, COPIES = TILEB / 1024, TILES = kStepKeys / (32 * NW);
  __shared__ __attribute__((aligned(1024))) char smem[NW * 2 * TILEB];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lq = lane & 31, hh = lane >> 5;
  int s, g;
  pair_of(blockIdx.x, a.nseq, a.c.Hkv, s, g);
  const int n = held_keys(a.c, s), c0 = block_of_keys() * keys;
  int nq = a.queries ? a.queries[s] : a.Nq;
  nq = nq < a.Nq ? nq : a.Nq;
  const int end = n - c0 < keys ? n : c0 + keys, t0 = c0 + 32 * w;
  if (t0 >= end || nq <= 0) return;
  const int rows = nq * a.G, off = n - a.Nq;
  const float c2 = a.scale * kLog2e;
  const long kstride = (long)a.c.Hkv * D;
  float* const W = a.weights + ((long)s * a.c.Hkv + g) * a.c.Nk;
  const int tiles = (end - t0 + 32 * NW - 1) / (32 * NW);  // this wavefront's: from t0, t0 + 128, ...
  int pages = 0;  // lane i: the page of tile i
  if (a.c.table) {
    const int x = t0 + lane * (32 * NW);
    pages = a.c.table[(long)s * a.c.table_stride + ((x < end ? x : t0) >> a.c.page_log2)];
  }
  // This lane's row
  const int rc = lq < rows ? lq : rows - 1, q = rc / a.G, h = g * a.G + (rc - q * a.G);
  const float l = a.LSE[s * a.lse_bs + h * a.lse_hs + q * a.lse_qs];
  bf16x8 Qf[KS];
  {
    const __bf16* qp = a.Q + (((long)s * a.Nq + q) * a.Hq + h) * D + 8 * hh;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) Qf[ks] = *(const bf16x8*)(qp + 16 * ks);
  }
  float sums[TILES];  // of the lane's key in every tile: what was there, and what is added
#pragma unroll
  for (int i = 0; i < TILES; ++i) sums[i] = W[t0 + 128 * i + lq < end ? t0 + 128 * i + lq : end - 1];
  touch(pages);
  touch(l);
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) touch(Qf[ks]);
#pragma unroll
  for (int i = 0; i < TILES; ++i) touch(sums[i]);
  char* const mine = smem + w * 2 * TILEB;
  auto request = [&](int i) {  // (keys past the end repeat the last one)
    const int t = t0 + 32 * NW * i;
    long row = (long)s * a.c.Nk + t;
    if (a.c.table) row = ((long)__builtin_amdgcn_readlane(pages, i) << a.c.page_log2) + (t & ((1 << a.c.page_log2) - 1));
    tile_load_async<D, 32, 1>(mine + (i & 1) * TILEB, a.K + row * kstride + (long)g * D, kstride, 0, n - 1 - t, 0, lane);
  };
  request(0);
  if (tiles > 1) request(1);
  f32x4 nl[4];  // of the rows of this lane's registers: -L in the exponent's base; -inf where the row adds nothing
  {
    const float x = lq < rows && l != -INFINITY ? -l * kLog2e : -INFINITY;
#pragma unroll
    for (int r = 0; r < 16; ++r) nl[r / 4][r % 4] = __shfl(x, acc_row(r, hh));
  }
  const int zrow = lq * ROWB + 16 * (hh ^ swz<ROWB>(lq));
  static_for<TILES>([&](auto I) {
    constexpr int i = decltype(I)::value;
    if (i >= tiles) return;
    const int t = t0 + 32 * NW * i;
    if (i + 1 < tiles) wait_vmem_upto<COPIES>();
    else wait_vmem();
    bf16x8 Kf[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) Kf[ks] = lds_b128(mine + (i & 1) * TILEB, zrow ^ (32 * ks));
    if (i + 2 < tiles) {
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // (read before its place is requested again)
      request(i + 2);
    }
    f32x16 S = (f32x16){0};
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) S = mfma32<F16>(Qf[ks], Kf[ks], S);
    float sum[2] = {0.f, 0.f};
    if (a.causal && t + 31 > off) {
      const int first = (t + lq - off) * a.G - 4 * hh;  // the first row that sees the lane's key, from the half's first
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float x = nl[r / 4][r % 4], e = fast_exp2(__builtin_fmaf(S[r], c2, x));
        sum[r & 1] += (x != -INFINITY) & (acc_row(r, 0) >= first) ? e : 0.f;
      }
    } else {
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float x = nl[r / 4][r % 4], e = fast_exp2(__builtin_fmaf(S[r], c2, x));
        sum[r & 1] += x != -INFINITY ? e : 0.f;
      }
    }
    sums[i] += sum_with_partner32(sum[0] + sum[1]);
  });
#pragma unroll
  for (int i = 0; i < TILES; ++i) {
    const int key = t0 + 32 * NW * i + lq;
    if (hh == 0 && key < end) W[key] = sums[i];
  }
}

// More rows, up to kStepRows, which lie in LDS. The keys of a tile come straight into registers, a row a lane, which the kernel above
// has left for whole rows through LDS: the rows take up to 68 KB of that here, and the other way has not been measured. 64 rows (G = 4) on
// 16 x 8 caches of up to 4096 keys of 128: 30 us, of which reading the keys at 6.25 TB/s would take about 11.
constexpr int kStepRows = 256;
template <int D, bool F16>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2))) void weights_rows_kernel(WeightsArgs a, int keys) {  // keys: of a workgroup, a multiple of 128
  constexpr int KS = D / 16, NW = 4, ROWB = 2 * D;
  __shared__ __attribute__((aligned(1024))) char smem[kStepRows * (ROWB + 4)];
  float* const stat = (float*)(smem + kStepRows * ROWB);  // nl of every row: -L in the exponent's base; -inf where the row adds nothing
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lq = lane & 31, hh = lane >> 5;
  int s, g;
  pair_of(blockIdx.x, a.nseq, a.c.Hkv, s, g);
  const int n = held_keys(a.c, s), c0 = block_of_keys() * keys;
  int nq = a.queries ? a.queries[s] : a.Nq;
  nq = nq < a.Nq ? nq : a.Nq;
  if (c0 >= n || nq <= 0) return;
  const int rows = nq * a.G, off = n - a.Nq;
  const float c2 = a.scale * kLog2e;
  const int end = n - c0 < keys ? n : c0 + keys;

  const long kstride = (long)a.c.Hkv * D;
  const int mask = (1 << a.c.page_log2) - 1;
  float* W = a.weights + ((long)s * a.c.Hkv + g) * a.c.Nk;
  bf16x8 Kr[2][KS];
  float old[2];   // (requested with the keys: loads come back in order, and one that is requested behind the next tile's waits for it)
  int pages = 0;  // lane i: the page of tile i of this wavefront's next 64
  auto request = [&](int t, auto BUF) {  // tile of 32 keys from t on; keys past the end repeat the last one
    long row = (long)s * a.c.Nk + t;
    if (a.c.table) {
      const int i = (t - c0) / (32 * NW) & 63;
      if (i == 0) {
        const int x = t + lane * (32 * NW);
        pages = a.c.table[(long)s * a.c.table_stride + ((x < end ? x : t) >> a.c.page_log2)];
      }
      row = ((long)__builtin_amdgcn_readlane(pages, i) << a.c.page_log2) + (t & mask);
    }
    const int in = t + lq < n ? lq : n - 1 - t;
    old[decltype(BUF)::value] = W[t + in];
    const __bf16* kp = a.K + (row + in) * kstride + (long)g * D + 8 * hh;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) Kr[decltype(BUF)::value][ks] = *(const bf16x8*)(kp + 16 * ks);
  };
  using B0 = std::integral_constant<int, 0>;
  using B1 = std::integral_constant<int, 1>;
  int t = c0 + 32 * w;
  if (t < end) request(t, B0{});
  if (t + 32 * NW < end) request(t + 32 * NW, B1{});

  auto row_stat = [&](int row) {
    const int rc = row < rows ? row : rows - 1, q = rc / a.G;
    const float l = a.LSE[s * a.lse_bs + (g * a.G + (rc - q * a.G)) * a.lse_hs + q * a.lse_qs];
    return row < rows && l != -INFINITY ? -l * kLog2e : -INFINITY;
  };
  auto row_at = [&](int row) {
    const int rc = row < rows ? row : rows - 1, q = rc / a.G;
    return a.Q + (((long)s * a.Nq + q) * a.Hq + g * a.G + (rc - q * a.G)) * D;
  };
  {
    constexpr int CPR = ROWB / 16;
    for (int i = threadIdx.x; i < (rows + 31) / 32 * 32 * CPR; i += 64 * NW) {
      const int r = i / CPR, ch = i % CPR;
      *(bf16x8*)(smem + swz_off<ROWB>(r, ch)) = *(const bf16x8*)(row_at(r) + 8 * ch);
    }
    if (threadIdx.x < (rows + 31) / 32 * 32) stat[threadIdx.x] = row_stat(threadIdx.x);
    __syncthreads();
    if (t >= end) return;
  }

  const int zrow = lq * ROWB + 16 * (hh ^ swz<ROWB>(lq));
  auto compute = [&](int t, auto BUF) {
    const int key = t + lq;
    float sum[2] = {0.f, 0.f};
    for (int rt = 0; rt < rows; rt += 32) {
      const long sees = a.causal ? (long)(t - off) * a.G : 0;  // the first row that sees the tile's first key
      if (sees > rt + 31) continue;
      f32x4 nl[4];  // of the rows of this lane's registers
#pragma unroll
      for (int i = 0; i < 4; ++i) nl[i] = *(const f32x4*)(stat + rt + 8 * i + 4 * hh);
      f32x16 S = (f32x16){0};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
        S = mfma32<F16>(lds_b128(smem, (zrow ^ (32 * ks)) + rt * ROWB), Kr[decltype(BUF)::value][ks], S);
      if (a.causal && sees + 31l * a.G > rt) {
        const int first = (key - off) * a.G - 4 * hh - rt;  // the first row that sees the lane's key, from the half's first
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const float x = nl[r / 4][r % 4], e = fast_exp2(__builtin_fmaf(S[r], c2, x));
          sum[r & 1] += (x != -INFINITY) & (acc_row(r, 0) >= first) ? e : 0.f;
        }
      } else {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const float x = nl[r / 4][r % 4], e = fast_exp2(__builtin_fmaf(S[r], c2, x));
          sum[r & 1] += x != -INFINITY ? e : 0.f;
        }
      }
    }
    const float total = sum_with_partner32(sum[0] + sum[1]);
    if (hh == 0 && key < end) W[key] = old[decltype(BUF)::value] + total;
  };
  bool here = true;
  while (true) {
    if (!here && t + 32 * NW < end) request(t + 32 * NW, B1{});
    here = false;
    compute(t, B0{});
    if ((t += 32 * NW) >= end) break;
    if (t + 32 * NW < end) request(t + 32 * NW, B0{});
    compute(t, B1{});
    if ((t += 32 * NW) >= end) break;
  }
}

// More rows: a workgroup has 64 keys, which each of its four wavefronts holds in registers, and the rows stream past, head by head, in
// tiles of 32 queries that the wavefronts take in turn: whole rows into a private piece of LDS, the next tile requested before the
// current one is used. The keys are the columns here too: a lane's sums are two keys' (with the keys as rows, 32 sums a lane and a
// transpose through LDS at the end, 2 prompts of 2048, 16 heads of 64, take 27.5 us instead of 23.7). Exponentials
// are 16 of the 24 cycles that a wavefront's 64 scores take, but the vector unit is busy 44% of that launch only: under the causal rule
// rows above the keys are not visited, a block of keys has from two to 64 row tiles there, and all blocks are resident at once, so that a
// compute unit has what its four happen to have. The blocks with the most are handed out first. No barrier in the loop.
constexpr int kPromptKeys = 64;
template <int D, bool F16>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(D == 64 ? 4 : 2))) void weights_prompt_kernel(WeightsArgs a) {
  constexpr int KS = D / 16, NW = 4, ROWB = 2 * D, CPR = ROWB / 16, RPI = 64 / CPR, COPIES = 32 / RPI;
  constexpr int STAGEB = 32 * ROWB + 256;  // a tile of rows, and the logsumexps (as many twice, a lane each)
  __shared__ __attribute__((aligned(1024))) char smem[NW * 2 * STAGEB];
  __shared__ float part[NW * kPromptKeys];
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), lq = lane & 31, hh = lane >> 5;
  const int pair = blockIdx.x, s = pair / a.c.Hkv, g = pair - s * a.c.Hkv;
  const int n = held_keys(a.c, s), c0 = block_of_keys() * kPromptKeys;
  int nq = a.queries ? a.queries[s] : a.Nq;
  nq = nq < a.Nq ? nq : a.Nq;
  if (c0 >= n || nq <= 0) return;
  const int off = n - a.Nq;
  const float c2 = a.scale * kLog2e;
  const int q_first = a.causal && c0 > off ? (c0 - off) & ~31 : 0;  // no query before it sees a key of the block
  const int per_head = nq > q_first ? (nq - q_first + 31) / 32 : 0, tiles = per_head * a.G;
  const __bf16* const Qb = a.Q + ((long)s * a.Nq * a.Hq + g * a.G) * D;
  const float* const Lb = a.LSE + s * a.lse_bs + g * a.G * a.lse_hs;
  const long qstride = (long)a.Hq * D;
  char* const ring = smem + w * 2 * STAGEB;
  // This wavefront's next tile to be requested: its head and first query (scalars, which advance by NW tiles)
  int next = w, next_h = 0, next_t = w;
  auto settle = [&]() {
    while (next_t >= per_head && next < tiles) next_t -= per_head, ++next_h;
  };
  auto request = [&](int stage) {
    settle();
    char* const to = ring + stage * STAGEB;
    const int q0 = q_first + 32 * next_t, last = nq - 1 - q0;  // (queries past the last one repeat it)
    const __bf16* const base = Qb + (long)next_h * D + (long)q0 * qstride;
    dma4(Lb + next_h * a.lse_hs + (q0 + (lq < last ? lq : last)) * a.lse_qs, to + 32 * ROWB);
#pragma unroll
    for (int u = 0; u < COPIES; ++u) {
      const int r = u * RPI + lane / CPR, ch = (lane % CPR) ^ swz<ROWB>(r);
      dma16(base + (long)(r < last ? r : last) * qstride + 8 * ch, to + u * 1024);
    }
    next += NW;
    next_t += NW;
  };
  bf16x8 Kr[2][KS];
  {
    const __bf16* kb = a.K + (cache_row(a.c, s, c0) * a.c.Hkv + g) * D + 8 * hh;  // (a block lies in one page)
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int row = 32 * u + lq, last = n - 1 - c0;  // (keys past the end repeat the last one)
      const __bf16* kp = kb + (long)(row < last ? row : last) * a.c.Hkv * D;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) Kr[u][ks] = *(const bf16x8*)(kp + 16 * ks);
    }
  }
  float sum[2][4] = {};  // of the lane's keys, over the rows so far
  const int zrow = lq * ROWB + 16 * (hh ^ swz<ROWB>(lq));
  auto compute = [&](int stage, int q0) {
    char* const at = ring + stage * STAGEB;
    float* const stat = (float*)(at + 32 * ROWB);
    // the rows' L becomes -L in the exponent's base (-inf where the row adds nothing), and goes to the lanes that hold its products
    const float l = stat[lane];
    const bool in = q0 + lq < nq && l != -INFINITY;
    stat[lane] = in ? -l * kLog2e : -INFINITY;
    bf16x8 q[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) q[ks] = lds_b128(at, zrow ^ (32 * ks));
    f32x4 nl[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) nl[i] = *(const f32x4*)(stat + 8 * i + 4 * hh);
    // (not all rows see all keys, or some are to add nothing: their scores may be NaN or +inf, and the exponential then is no 0)
    const bool some = (a.causal && q0 + off - c0 < kPromptKeys - 1) || __builtin_amdgcn_ballot_w64(!in);
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      f32x16 S = (f32x16){0};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) S = mfma32<F16>(q[ks], Kr[u][ks], S);
      if (some) {
        const int first = a.causal ? c0 + 32 * u + lq - off - q0 - 4 * hh : 0;  // the first row that sees the lane's key, from the half's first
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const float x = nl[r / 4][r % 4], e = fast_exp2(__builtin_fmaf(S[r], c2, x));
          sum[u][r & 3] += (x != -INFINITY) & (acc_row(r, 0) >= first) ? e : 0.f;
        }
      } else {
#pragma unroll
        for (int r = 0; r < 16; ++r) sum[u][r & 3] += fast_exp2(__builtin_fmaf(S[r], c2, nl[r / 4][r % 4]));
      }
    }
  };
  if (w < tiles) {
    int t = w, tq = w;
    request(0);
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) touch(Kr[u][ks]);
    for (int stage = 0; t < tiles; t += NW, tq += NW, stage ^= 1) {
      while (tq >= per_head) tq -= per_head;
      if (next < tiles) {
        request(stage ^ 1);
        wait_vmem_upto<COPIES + 1>();
      } else {
        wait_vmem();
      }
      compute(stage, q_first + 32 * tq);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // (read before its place is requested again)
    }
  }
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const float total = sum_with_partner32(sum[u][0] + sum[u][1] + (sum[u][2] + sum[u][3]));
    if (hh == 0) part[w * kPromptKeys + 32 * u + lq] = total;
  }
  __syncthreads();
  if (tid < kPromptKeys && c0 + tid < n) {
    float total = 0.f;
#pragma unroll
    for (int u = 0; u < NW; ++u) total += part[u * kPromptKeys + tid];
    a.weights[((long)s * a.c.Hkv + g) * a.c.Nk + c0 + tid] += total;
  }
}

template <int D, bool F16>
static hipError_t launch_weights_d(const WeightsArgs& a, hipStream_t st) {
  const unsigned pairs = (unsigned)(a.nseq * a.c.Hkv);
  // Rows that stay, or keys that do: a prompt among its own keys has as many of these as queries, and the blocks of 64 keys make more
  // workgroups (us, rows stay / keys stay: 256 rows among 256 keys, 2 x 8 pairs of 128: 10.8 / 6.5; 256 rows (G = 4) on up to
  // 2000 keys, 4 x 8 pairs of 64: 9.7 / 9.9; 64 rows (G = 4) on up to 4096, 16 x 8 of 128: 31 / 79; 40 rows (G = 8), 32 x 8: 57 / 153)
  if ((long)a.Nq * a.G <= kStepRows && ((long)a.Nq * a.G <= 32 || a.c.Nk > 2l * a.Nq)) {
    // Two workgroups a compute unit, or up to four tiles a wavefront (us at 128 / 256 / 512 / 1024 keys: 4 sequences of up to 2048, 8
    // heads of 128: 5.3 / 5.1 / 6.6 / 9.4; 8 of up to 4096: 14.5 / 11.3 / 10.0 / 10.0; 64 of up to 8192: 143 / 105 / 96 / 96; 96 of up to
    // 2048, heads of 64: 34 / 27 / 25 / 27)
    long keys = ((long)pairs * a.c.Nk / 512 + 127) / 128 * 128;
    keys = keys < 128 ? 128 : (keys > kStepKeys ? kStepKeys : keys);
    const dim3 grid = grid_of(pairs, (a.c.Nk + keys - 1) / keys);
    if (a.Nq * a.G <= 32) hipLaunchKernelGGL((weights_step_kernel<D, F16>), grid, dim3(256), 0, st, a, (int)keys);
    else hipLaunchKernelGGL((weights_rows_kernel<D, F16>), grid, dim3(256), 0, st, a, (int)keys);
  } else {
    hipLaunchKernelGGL((weights_prompt_kernel<D, F16>), grid_of(pairs, ((long)a.c.Nk + kPromptKeys - 1) / kPromptKeys), dim3(256), 0, st, a);
  }
  return hipGetLastError();
}
hipError_t launch_weights(const WeightsArgs& a, hipStream_t st) {
  if (a.c.d == 64) return a.f16 ? launch_weights_d<64, true>(a, st) : launch_weights_d<64, false>(a, st);
  return a.f16 ? launch_weights_d<128, true>(a, st) : launch_weights_d<128, false>(a, st);
}

}  // namespace fa
