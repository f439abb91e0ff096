// Attention of a batch whose sequences share a prefix: every query attends to the prefix, computed once for the whole batch, and to
// the keys that its own sequence holds. Softmax over the two together is the merge of its parts by their logsumexps (the identity of
// section 3.1.1 between blocks), so the work is cut into items that know nothing of each other:
//   * prefix items: rows of ALL sequences against a share of the prefix. A row is a (token, head of the group) pair, packed
//     token * G + head; K and V of the prefix are read once per block of rows, not once per sequence.
//   * own items: the rows of one sequence against a share of its own cache.
// One launch does the items of both kinds, since the first do many products with a key that they read and the second few: they ask
// different things of a compute unit. (Neither is at its limit: 64 sequences on 8192 shared keys, up to 1024 own ones, read 4.3 TB/s
// with the matrix units busy 12% of the launch; what is waited for is the longest share's chain of tiles.) Each leaves a normalised
// partial O and its logsumexp in float32, and a second launch merges them. P is rounded to the element type for the second product, as
// in every forward kernel here: O is then 1.3 to 1.4 times as far from the exact result as its own rounding alone would put it (bfloat16 0.0023
// and 0.0017 of it).
//
// Items of up to 32 rows (narrow) have one row tile, and the four wavefronts of a workgroup divide the keys; items of up to 128
// rows (wide) give each wavefront 32 rows, and the four share the tiles of K and V in LDS.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "fa_kernels.h"
#include "fa_lds.h"
#include "fa_merge.h"

namespace fa {

namespace {

struct Item {
  const __bf16 *K, *V;   // (already at the key/value head)
  const int32_t* table;  // of this item's keys; nullptr: rows follow each other
  int nk, begin, end;    // keys in all, and the share [begin, end), begin a multiple of 64
  long tok0;             // token of packed row 0
  int row0, rows;        // packed rows row0 .. row0 + rows - 1
  int off;               // causal: row r sees keys up to r / G + off; else a bound past every key
  bool causal;
  int g, slot;
};

__device__ __forceinline__ const __bf16* item_rows(const PrefixArgs& a, const Item& it, const __bf16* pool, int key, long kstride) {
  if (!it.table) return pool + (long)key * kstride;
  const int page = it.table[key >> a.own.page_log2];
  return pool + (((long)page << a.own.page_log2) + (key & ((1 << a.own.page_log2) - 1))) * kstride;
}

// Partial results of packed row r of an item
__device__ __forceinline__ long item_row(const PrefixArgs& a, const Item& it, int r) {
  const int row = it.row0 + r, q = row / a.G;
  return (long)it.slot * a.nseq * a.Nq * a.Hq + (it.tok0 + q) * a.Hq + it.g * a.G + (row - q * a.G);
}

// Tiles of K and of V that a wavefront of a narrow item has on their way (8 KB each of 64 columns, 16 of 128; eight wavefronts a unit)
template <int D>
constexpr int kNarrowStages = D == 64 ? 2 : 1;
template <int D>
constexpr int kPrefixLds = 4 * kNarrowStages<D> * 2 * 32 * 2 * D + 2 * 4 * 32 * 4;  // narrow: those, later partial O; m and l

template <int D, bool F16>
__device__ __forceinline__ void narrow_item(const PrefixArgs& a, const Item& it, char* smem) {
  constexpr int NW = 4, KT = 32, KS = D / 16, DT = D / 32, ROWB = 2 * D, TILEB = KT * ROWB, STAGES = kNarrowStages<D>, WAVEB = STAGES * 2 * TILEB, STAT_OFF = NW * WAVEB;
  static_assert(WAVEB >= D * 32 * 4 && STAT_OFF + 2 * NW * 32 * 4 <= kPrefixLds<D>, "the partial O^T of a wavefront takes the place of its tiles");
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), lq = lane & 31, hh = lane >> 5;
  const long kstride = (long)a.Hkv * D;
  const int prow = it.row0 + (lq < it.rows ? lq : it.rows - 1);  // (lanes past the end compute on a copy and store nothing)
  const int q = prow / a.G;
  bf16x8 Qf[KS];
  {
    const __bf16* qp = a.Q + ((it.tok0 + q) * a.Hq + it.g * a.G + (prow - q * a.G)) * D + 8 * hh;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) Qf[ks] = *(const bf16x8*)(qp + 16 * ks);
  }
  const int lim_row = it.causal && q + it.off < it.nk - 1 ? q + it.off : it.nk - 1;  // the last key of this lane's row
  // Pages of this wavefront's tiles: lane i has the one of tile i of the next 64 (looked up one by one each would be a memory latency
  // in front of its tile's requests).
  const int mask = (1 << a.own.page_log2) - 1;
  int pages = 0;
  auto issue = [&](int key0, int stage) {
    const int last = it.end - 1 - key0;  // (rows past the end repeat the last one)
    long row = key0;
    if (it.table) {
      const int i = (key0 - it.begin) / (NW * KT) & 63;
      if (i == 0) {
        const int t = key0 + lane * (NW * KT);
        pages = it.table[(t < it.end ? t : key0) >> a.own.page_log2];
      }
      row = ((long)__builtin_amdgcn_readlane(pages, i) << a.own.page_log2) + (key0 & mask);
    }
    char* const to = smem + w * WAVEB + stage * 2 * TILEB;
    tile_load_async<D, KT, 1>(to, it.K + row * kstride, kstride, 0, last, 0, lane);
    tile_load_async<D, KT, 1>(to + TILEB, it.V + row * kstride, kstride, 0, last, 0, lane);
  };
  f32x16 O[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) O[dt] = (f32x16){0};
  float m = -INFINITY, l = 0.f;
  const float c2 = a.scale_log2e;
  const int p16 = lane & 15, g16 = (lane >> 4) & 1;
  int zcol[2];
#pragma unroll
  for (int u = 0; u < 2; ++u) zcol[u] = swz_off<ROWB>(4 * hh + (p16 >> 2) + 8 * u, 2 * g16 + ((p16 & 3) >> 1)) + 8 * (p16 & 1);
  const int zrow = lq * ROWB + 16 * (hh ^ swz<ROWB>(lq));
  bf16x8 Kf[KS], Vf[2 * DT];  // of the tile in use: its place in LDS is the next one's at once
  auto take = [&](int stage) {
    const int kb = w * WAVEB + stage * 2 * TILEB, vb = kb + TILEB;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) Kf[ks] = lds_b128(smem, (zrow + kb) ^ (32 * ks));
#pragma unroll
    for (int i = 0; i < 2 * DT; ++i) {
      const int dt = i >> 1, ro = 16 * (i & 1) * ROWB;
      Vf[i] = lds_tr_pair(smem, ((zcol[0] + vb) ^ (64 * dt)) + ro, ((zcol[1] + vb) ^ (64 * dt)) + ro);
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  };
  auto compute = [&](int key0) {
    f32x16 S = (f32x16){0};
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) S = mfma32<F16>(Kf[ks], Qf[ks], S);
    if ((it.causal && key0 + KT - 1 > it.row0 / a.G + it.off) || key0 + KT > it.end) {
      const int lim = (lim_row < it.end - 1 ? lim_row : it.end - 1) - key0 - 4 * hh;
#pragma unroll
      for (int r = 0; r < 16; ++r) S[r] = acc_row(r, 0) > lim ? -INFINITY : S[r];
    }
    float mx = S[0];
#pragma unroll
    for (int r = 1; r < 16; ++r) mx = fmaxf(mx, S[r]);
    mx = max_with_partner32(mx);
    // (the reference of the softmax is only advanced where some row's maximum has outgrown it: fa_common.h)
    if (__builtin_amdgcn_ballot_w64((mx - m) * c2 > (float)kLazyLog2<F16> || (m == -INFINITY && mx != -INFINITY))) {
      const float m_new = fmaxf(m, mx);
      const float alpha = m_new == -INFINITY ? 1.f : fast_exp2((m - m_new) * c2);
      l *= alpha;
      m = m_new;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) O[dt][r] *= alpha;
    }
    const float ref = m == -INFINITY ? 0.f : m * c2;
    float rs = 0.f;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      S[r] = fast_exp2(__builtin_fmaf(S[r], c2, -ref));
      rs += S[r];
    }
    l += rs;
    bf16x8 Pf[2] = {pack8<F16>(S, 0), pack8<F16>(S, 1)};
#pragma unroll
    for (int i = 0; i < 2 * DT; ++i) O[i >> 1] = mfma32<F16>(Vf[i], Pf[i & 1], O[i >> 1]);
  };
  // (K too goes through LDS, as whole rows: a lane that loads its own row straight into registers makes every request touch 64 places.
  // 64 sequences on 8192 shared keys, up to 1024 own ones, 32 heads on 8 of 128: 41.8 -> 39.7 us; 4 on 2048, up to 256: 8.7 -> 7.4.)
  // One copy of the code of a tile: short shares run it twice, and wait for its instructions (2 KB) the first time.
  int t = it.begin + KT * w;
  if (t < it.end) {
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) touch(Qf[ks]);
    issue(t, 0);
    if (STAGES == 2 && t + NW * KT < it.end) issue(t + NW * KT, 1);
    for (int stage = 0;; stage ^= STAGES - 1) {
      if (STAGES == 2 && t + NW * KT < it.end) wait_vmem_upto<2 * TILEB / 1024>();
      else wait_vmem();
      take(stage);
      if (t + STAGES * NW * KT < it.end) issue(t + STAGES * NW * KT, stage);
      compute(t);
      if ((t += NW * KT) >= it.end) break;
    }
  }
  // ---- the wavefronts' partial results become the item's
  const float lsum = sum_with_partner32(l);
  __syncthreads();
  // rows of pieces of four columns, their places XOR-ed with the row
  constexpr int CPR = D / 4;
  char* const mine = smem + w * WAVEB + lq * (4 * D);
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int r4 = 0; r4 < 4; ++r4) {
      f32x4 o;
#pragma unroll
      for (int v = 0; v < 4; ++v) o[v] = O[dt][4 * r4 + v];
      *(f32x4*)(mine + 16 * ((8 * dt + 2 * r4 + hh) ^ (lq & (CPR - 1)))) = o;
    }
  float* stat = (float*)(smem + STAT_OFF);
  if (hh == 0) {
    stat[w * 32 + lq] = m;
    stat[32 * NW + w * 32 + lq] = lsum;
  }
  __syncthreads();
  for (int i = tid; i < it.rows * CPR; i += 64 * NW) {
    const int r = i / CPR, c = i % CPR;
    float mm = -INFINITY;
#pragma unroll
    for (int u = 0; u < NW; ++u) mm = fmaxf(mm, stat[u * 32 + r]);
    float den = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int u = 0; u < NW; ++u) {
      const float mw = stat[u * 32 + r], wgt = mw == -INFINITY ? 0.f : fast_exp2((mw - mm) * c2);
      den += wgt * stat[32 * NW + u * 32 + r];
      o += *(const f32x4*)(smem + u * WAVEB + r * (4 * D) + 16 * (c ^ (r & (CPR - 1)))) * wgt;
    }
    const float inv = den == 0.f ? 0.f : 1.f / den;  // (no visible key: L = -inf, and the merge does not look at O; a NaN stays one)
    const long at = item_row(a, it, r);
    *(f32x4*)(a.Opart + at * D + 4 * c) = o * inv;
    if (c == 0) a.Lpart[at] = den == 0.f ? -INFINITY : mm * a.scale + fast_log2(den) * kLn2;
  }
}

template <int D, bool F16>
__device__ __forceinline__ void wide_item(const PrefixArgs& a, const Item& it, char* smem) {
  constexpr int BC = 64, KS = D / 16, DT = D / 32, ROWB = 2 * D, TILEB = BC * ROWB, V_OFF = 2 * TILEB;
  static_assert(4 * TILEB <= kPrefixLds<D>, "two stages of K and of V");
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), lq = lane & 31, hh = lane >> 5;
  const long kstride = (long)a.Hkv * D;
  const int r0 = 32 * w, mine = r0 + lq;  // this lane's row of the item
  const int prow = it.row0 + (mine < it.rows ? mine : it.rows - 1), q = prow / a.G;
  TileCopier<BC, ROWB> copier;
  copier.init(kstride, w, lane);
  constexpr int CPT = TileCopier<BC, ROWB>::COPIES, AHEAD = 4;
  auto copy = [&](const __bf16* pool, int key0, int to) {
    const auto plan = copier.plan(item_rows(a, it, pool, key0, kstride), it.end - 1 - key0);
    static_for<CPT>([&](auto Q) { copier.template copy<Q.value>(plan, smem + to); });
  };
  copy(it.K, it.begin, 0);
  bf16x8 Qf[KS];
  {
    const __bf16* qp = a.Q + ((it.tok0 + q) * a.Hq + it.g * a.G + (prow - q * a.G)) * D + 8 * hh;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) Qf[ks] = *(const bf16x8*)(qp + 16 * ks);
  }
  copy(it.V, it.begin, V_OFF);
  if (it.begin + BC < it.end) copy(it.K, it.begin + BC, TILEB);
  const int lim_row = it.causal && q + it.off < it.nk - 1 ? q + it.off : it.nk - 1;
  const int lim_end = lim_row < it.end - 1 ? lim_row : it.end - 1;
  const int lim_least = it.causal ? (it.row0 + r0) / a.G + it.off : it.end;  // keys up to here: seen by all rows of the wavefront
  f32x16 O[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) O[dt] = (f32x16){0};
  float m = -INFINITY, l = 0.f;
  const float c2 = a.scale_log2e;
  const int zrow = lq * ROWB + 16 * (hh ^ swz<ROWB>(lq));
  const int p16 = lane & 15, g16 = (lane >> 4) & 1;
  int zcol[2];
#pragma unroll
  for (int u = 0; u < 2; ++u) zcol[u] = swz_off<ROWB>(4 * hh + (p16 >> 2) + 8 * u, 2 * g16 + ((p16 & 3) >> 1)) + 8 * (p16 & 1);
  auto scores = [&](f32x16 (&S)[2], int buf) {
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
      S[kt] = (f32x16){0};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
        S[kt] = mfma32<F16>(lds_b128(smem, ((zrow + buf * TILEB) ^ (32 * ks)) + kt * 32 * ROWB), Qf[ks], S[kt]);
    }
  };
  auto mask = [&](f32x16 (&S)[2], int key0) {
    if (key0 + BC - 1 > lim_least || key0 + BC > it.end) {
      asm volatile("; keep this a branch" ::);
      mask_past(S, lim_end - key0 - 4 * hh);
    }
  };
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) touch(Qf[ks]);
  if (it.begin + BC < it.end) wait_vmem_upto<2 * CPT>();
  else wait_vmem_upto<CPT>();
  lds_barrier();
  f32x16 Sa[2], Sb[2];
  scores(Sa, 0);
  mask(Sa, it.begin);
  m = row_maximum(Sa);
  // Iteration of the block at key0 (stage `buf`): the scores of the next block are formed beside the exponentials of this one, then O
  // is updated. K of the block after the next and V of the next are on their way meanwhile.
  auto iteration = [&](int key0, auto BUF, f32x16 (&S)[2], f32x16 (&Sn)[2]) {
    constexpr int buf = decltype(BUF)::value;
    const bool next = key0 + BC < it.end;
    wait_vmem();
    lds_barrier();
    if (next) {
      copy(it.V, key0 + BC, V_OFF + (buf ^ 1) * TILEB);
      if (key0 + 2 * BC < it.end) copy(it.K, key0 + 2 * BC, buf * TILEB);
    }
    bf16x8 P[2][2];
    float rs0, rs1;
    const float ref = m == -INFINITY ? 0.f : -m * c2;
    __builtin_amdgcn_sched_barrier(0);
    scores(Sn, buf ^ 1);  // (past the end: of whatever is there, and not used)
    block_exponentials<F16>(S, c2, ref, P, rs0, rs1);
    __builtin_amdgcn_sched_group_barrier(0x100, AHEAD, 0);
#pragma unroll
    for (int i = 0; i < 2 * KS; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x002, 8 * 16 / (2 * KS), 0);
    }
    __builtin_amdgcn_sched_barrier(0);
    if (reference_outgrown<F16>(rs0 + rs1) || __builtin_amdgcn_ballot_w64(m == -INFINITY)) {
      const float m_new = fmaxf(m, row_maximum(S));
      const float alpha = m_new == -INFINITY ? 1.f : fast_exp2((m - m_new) * c2);
      l *= alpha;
      m = m_new;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) O[dt][r] *= alpha;
      block_exponentials<F16>(S, c2, m == -INFINITY ? 0.f : -m * c2, P, rs0, rs1);
    }
    l += rs0 + rs1;
    __builtin_amdgcn_sched_barrier(0);
    mfma_stream<4 * DT, AHEAD, 2>(
        [&](int i) {
          const int dt = i >> 2, ro = 16 * (i & 3) * ROWB, vb = V_OFF + buf * TILEB;
          return lds_tr_pair(smem, ((zcol[0] + vb) ^ (64 * dt)) + ro, ((zcol[1] + vb) ^ (64 * dt)) + ro);
        },
        [&](int i, const bf16x8& v) { O[i >> 2] = mfma32<F16>(v, P[(i >> 1) & 1][i & 1], O[i >> 2]); });
    if (next) mask(Sn, key0 + BC);
  };
  using B0 = std::integral_constant<int, 0>;
  using B1 = std::integral_constant<int, 1>;
  for (int key0 = it.begin;;) {
    iteration(key0, B0{}, Sa, Sb);
    if ((key0 += BC) >= it.end) break;
    iteration(key0, B1{}, Sb, Sa);
    if ((key0 += BC) >= it.end) break;
  }
  // ---- through LDS, so that whole rows are stored (16 bytes a row and instruction straight from the accumulators took 1 us per MB)
  const float lsum = sum_with_partner32(l);
  const float inv = lsum == 0.f ? 0.f : 1.f / lsum;
  lds_barrier();  // everyone has read the last tiles
  constexpr int CPR = D / 4;  // 16-byte chunks of a row
  char* const stage = smem + w * (32 * 4 * D);
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int r4 = 0; r4 < 4; ++r4) {
      f32x4 o;
#pragma unroll
      for (int v = 0; v < 4; ++v) o[v] = O[dt][4 * r4 + v] * inv;
      *(f32x4*)(stage + lq * (4 * D) + 16 * ((8 * dt + 2 * r4 + hh) ^ (lq & (CPR - 1)))) = o;
    }
#pragma unroll 4
  for (int i = 0; i < CPR / 2; ++i) {
    const int r = (64 * i + lane) / CPR, c = lane & (CPR - 1);
    const f32x4 o = *(const f32x4*)(stage + r * (4 * D) + 16 * (c ^ (r & (CPR - 1))));
    if (r0 + r < it.rows) *(f32x4*)(a.Opart + item_row(a, it, r0 + r) * D + 4 * c) = o;
  }
  if (hh == 0 && mine < it.rows) a.Lpart[item_row(a, it, mine)] = lsum == 0.f ? -INFINITY : m * a.scale + fast_log2(lsum) * kLn2;
}

__device__ __forceinline__ void empty_item(const PrefixArgs& a, const Item& it) {
  for (int r = threadIdx.x; r < it.rows; r += 256) a.Lpart[item_row(a, it, r)] = -INFINITY;
}

// Share k of n keys cut into shares of `per` (a multiple of 64)
__device__ __forceinline__ void share_of(int n, int per, int k, int& begin, int& end) {
  const long b = (long)k * per;
  begin = b < n ? (int)b : n;
  end = n - begin < per ? n : begin + per;
}

template <int D, bool F16>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2))) void prefix_items_kernel(PrefixArgs a, PrefixPlan plan, int prefix_items) {
  __shared__ __attribute__((aligned(1024))) char smem[kPrefixLds<D>];
  Item it;
  const int i = blockIdx.x;
  int rows, wide;
  if (i < prefix_items) {
    const int all = a.nseq * a.Nq * a.G, blocks = (all + plan.prefix_rows - 1) / plan.prefix_rows;
    const int unit = i / blocks / kXcds * kXcds + i % kXcds, blk = i / kXcds % blocks;  // the blocks of rows of a share: on one XCD
    if (unit >= a.Hkv * plan.prefix_shares) return;
    it.g = unit / plan.prefix_shares;
    it.slot = unit - it.g * plan.prefix_shares;
    it.row0 = blk * plan.prefix_rows;
    rows = all;
    it.tok0 = 0;
    it.nk = a.Np;
    it.off = 0;
    it.causal = false;
    it.K = a.Kp + (long)it.g * D;
    it.V = a.Vp + (long)it.g * D;
    it.table = a.prefix_table;
    share_of(it.nk, plan.prefix_keys, it.slot, it.begin, it.end);
    wide = plan.prefix_rows;
  } else {
    const int j = i - prefix_items, blocks = (a.Nq * a.G + plan.own_rows - 1) / plan.own_rows, per = blocks * plan.own_shares;
    // (sequences of uneven lengths: longest first)
    const int pair = j / per, in = j - pair * per, rank = pair / a.Hkv;
    const CacheSequence cs = cache_sequence(a.own.lens, a.own.Nk, a.nseq, rank);
    const int s = cs.s;
    it.g = pair - rank * a.Hkv;
    it.slot = in % plan.own_shares;
    it.row0 = in / plan.own_shares * plan.own_rows;
    rows = a.Nq * a.G;
    it.tok0 = (long)s * a.Nq;
    it.nk = cs.len;
    it.off = it.nk - a.Nq;
    it.causal = a.causal != 0;
    const long first = a.own.table ? 0 : (long)s * a.own.Nk * a.Hkv;
    it.K = a.K + (first + it.g) * D;
    it.V = a.V + (first + it.g) * D;
    it.table = a.own.table ? a.own.table + (long)s * a.own.table_stride : nullptr;
    share_of(it.nk, plan.own_keys, it.slot, it.begin, it.end);
    it.slot += plan.prefix_shares;
    wide = plan.own_rows;
  }
  it.rows = rows - it.row0 < wide ? rows - it.row0 : wide;
  if (it.begin >= it.end) return empty_item(a, it);
  if (wide == 32) narrow_item<D, F16>(a, it, smem);
  else wide_item<D, F16>(a, it, smem);
}

template <int D, bool F16, int FLY>
__global__ __launch_bounds__(256) void prefix_merge_kernel(PrefixArgs a, int slots) {
  merge_slots<D, F16, FLY>(a.Opart, a.Lpart, a.O, a.LSE, (long)a.nseq * a.Nq * a.Hq, a.Hq, a.Nq, slots);
}

template <int D, bool F16>
hipError_t launch_prefix_d(const PrefixArgs& a, hipStream_t st) {
  const PrefixPlan plan = prefix_plan(a.nseq, a.Hq, a.Hkv, a.Nq, a.Np, a.own.Nk, D);
  const long all = (long)a.nseq * a.Nq * a.G, blocks = (all + plan.prefix_rows - 1) / plan.prefix_rows;
  const long units = (long)a.Hkv * plan.prefix_shares, prefix = (units + kXcds - 1) / kXcds * kXcds * blocks;
  const long own = (long)a.nseq * a.Hkv * (((long)a.Nq * a.G + plan.own_rows - 1) / plan.own_rows) * plan.own_shares;
  if (prefix + own > 0x7fffffffL) return hipErrorInvalidConfiguration;
  hipLaunchKernelGGL((prefix_items_kernel<D, F16>), dim3((unsigned)(prefix + own)), dim3(256), 0, st, a, plan, (int)prefix);
  if (hipError_t e = hipGetLastError()) return e;
  constexpr int RPB = 256 / (D / 4);
  const int slots = plan.prefix_shares + plan.own_shares;
  const dim3 grid((unsigned)(((long)a.nseq * a.Nq * a.Hq + RPB - 1) / RPB));
  if (slots <= 4) hipLaunchKernelGGL((prefix_merge_kernel<D, F16, 4>), grid, dim3(256), 0, st, a, slots);
  else if (slots <= 9) hipLaunchKernelGGL((prefix_merge_kernel<D, F16, 9>), grid, dim3(256), 0, st, a, slots);
  else hipLaunchKernelGGL((prefix_merge_kernel<D, F16, 17>), grid, dim3(256), 0, st, a, slots);
  return hipGetLastError();
}

}  // namespace

PrefixPlan prefix_plan(int B, int Hq, int Hkv, int Nq, int Np, int Nk, int d) {
  PrefixPlan p;
  const long G = Hq / Hkv, own_rows = Nq * G, all = B * own_rows;
  auto clamp = [](long x, long lo, long hi) { return x < lo ? lo : (x > hi ? hi : x); };
  auto up = [](long x, long y) { return (x + y - 1) / y; };
  // shares of `keys`, at most `most` of them and none below `least` keys
  auto cut = [&](long keys, long most, long least, int& share, int& shares) {
    const long per = clamp(up(up(keys, 64), most < 1 ? 1 : most), least / 64, 1l << 24);
    share = (int)(64 * per);
    shares = (int)up(keys, 64 * per);
  };
  p.prefix_rows = all <= 32 ? 32 : 128;
  const long units = Hkv * up(all, p.prefix_rows);
  // Half as many prefix items as compute units, in 16 shares at most, or shares of 1024 keys where that makes more of them, up to one
  // item a unit (64 sequences, 32 heads on 8 of 128, 8192 shared keys, 16 blocks of rows, us of the first launch at 6 / 8 / 12 / 16
  // shares: 45 / 40 / 43 / 43; 16 x 5 rows, 16 heads of 64, 12345 keys, 16 blocks, at 6 / 12 / 16: 40 / 31 / 31. Few blocks of rows,
  // the whole call with 16 shares and by the rule: one sequence, 4 heads on one of 128, 32768 and 65536 keys: 24.1 and 18.0, 42.7 and
  // 23.8; 8 on 2: 25.5 and 20.0, 43.7 and 27.7; 32 sequences, 4 heads on one of 64: 32.7 and 26.2, 57.2 and 36.6; 8 sequences, 16 on 4
  // of 128, 20480 and 32768 keys: 20.4 and 21.1, 26.7 and 25.0)
  const long most = std::max(std::min(up(128, units), 16l), clamp(Np / 1024, 1, up(256, units)));
  cut(Np, most, 256, p.prefix_keys, p.prefix_shares);
  // Up to 64 own rows are two narrow items: they read the keys twice, but divide them over four wavefronts each, where a wide one leaves
  // two idle (us, narrow and wide: 16 sequences of up to 1024 keys, 5 x 8 rows a head, 4 heads of 64: 13.9 and 15.6; one of up to 8192, 8
  // of 128: 18.9 and 25.9; 64 of 1024, 4 of 128, on 8192 shared: 70.4 and 72.3; but 16 of 2048, 8 of 128: 37.0 and 35.6; 32 of 2048, 9 x 4
  // rows, 8 of 64: 43.5 and 42.3; 64 of 512, 16 x 4 rows, 4 of 128: 38.9 and 35.4)
  p.own_rows = own_rows <= 64 ? 32 : 128;
  // Own items: with those of the prefix no more than fit on the chip at once, two a compute unit (16 x 16
  // pairs of up to 2048 keys of 64, beside 192 items of the prefix, one and two shares: 31 and 36 us; 24 x 8 of up to 4096 of 128, beside
  // 96, two, three and four: 43, 44 and 48)
  const long pairs = B * Hkv * up(own_rows, p.own_rows);
  cut(Nk, clamp((512 - units * p.prefix_shares) / pairs, 1, 8), 256, p.own_keys, p.own_shares);
  return p;
}

hipError_t launch_prefix(const PrefixArgs& a, int d, hipStream_t st) {
  if (d == 64) return a.f16 ? launch_prefix_d<64, true>(a, st) : launch_prefix_d<64, false>(a, st);
  return a.f16 ? launch_prefix_d<128, true>(a, st) : launch_prefix_d<128, false>(a, st);
}

}  // namespace fa
