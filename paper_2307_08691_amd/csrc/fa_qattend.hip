// Attention over a key/value cache held in 4 or 8 bits (fa_mx.h): Algorithm 1 over what the codes stand for, with the parallelism of
// decoding. The rows of one (sequence, key/value head), query * G + head of the group, are cut into items of up to 32 of them against a
// share of the keys; the four wavefronts of a workgroup take tiles of 32 keys in turn, each with a running softmax of its own, no barrier
// in the loop, and join through LDS at the end. Shares are joined by a second launch (fa_merge.h).
//
// Codes become 16-bit elements in registers, two an instruction, and every product is a 16x16x32 MFMA of those:
//   * S^T = K Q^T: a lane holds a quarter of a key's channels, D / 4 consecutive ones of one or two blocks, as they lie in memory. The
//     order in which channels are summed is free, so step s of the contraction takes eight of each lane's own, and Q is held alike.
//   * O^T += V^T P^T needs keys along a lane's operand, so V goes through LDS once: read in whole rows, converted, written as 16-bit rows and
//     read back transposed. P^T is in place already: the keys of a lane's eight operand elements are those whose scores it has.
// Bound by HBM, which hands a compute unit 24 bytes a ns: 136 bytes a key of 128 channels in 4 bits.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "fa_lds.h"
#include "fa_merge.h"
#include "fa_qattend.h"

namespace fa {

namespace {

template <bool F16>
__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) {
  if constexpr (F16) return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  else return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
// Over the four lanes l % 16 + 16 i
__device__ __forceinline__ float max_of_four(float x) {
  const int i = __builtin_bit_cast(int, x);
  auto sw = __builtin_amdgcn_permlane16_swap(i, i, false, false);
  return max_with_partner32(fmaxf(__builtin_bit_cast(float, (int)sw[0]), __builtin_bit_cast(float, (int)sw[1])));
}
__device__ __forceinline__ float sum_of_four(float x) {
  const int i = __builtin_bit_cast(int, x);
  auto sw = __builtin_amdgcn_permlane16_swap(i, i, false, false);
  return sum_with_partner32(__builtin_bit_cast(float, (int)sw[0]) + __builtin_bit_cast(float, (int)sw[1]));
}

// Where chunk c (16 bytes) of key k lies in a wavefront's V tile, 32 rows of 2 D bytes: XOR-ed with a function of the key chosen so that the
// transposing reads (8 keys x 32 bytes at a time) and the writes (16 lanes x 16 bytes: PIECE chunks a lane, 2 (VB = 8) or 4) are both free
// of bank conflicts.
template <int D, int VB>
__device__ __forceinline__ int v_swizzle(int k) {
  const int k0 = k & 1, k1 = (k >> 1) & 1, k2 = (k >> 2) & 1;
  if (D == 128) return VB == 4 ? (k0 << 1 | k1 | k1 << 2 | k2 << 3) : (k0 | k0 << 1 | k1 << 2 | k2 << 3);
  return VB == 4 ? (k2 | k1 << 1 | k2 << 2) : (k1 | k1 << 1 | k2 << 2);  // (two rows of 128 bytes share a line of the banks)
}

template <int D, int KB, int VB, int RT>
struct Narrow {
  static constexpr int NW = 4, KT = 32, ROWS = 16 * RT, ROWB = 2 * D, VTILE = KT * ROWB, PART = ROWS * 4 * D, WAVEB = VTILE > PART ? VTILE : PART;
  static constexpr int STAT_OFF = NW * WAVEB, LDS = STAT_OFF + 2 * NW * ROWS * 4;
};

template <int D, bool F16, int KB, int VB, int RT>
__device__ __forceinline__ void narrow_item(const QAttendArgs& a, const QItem& it, bool direct, char* smem) {
  typedef Narrow<D, KB, VB, RT> N;
  constexpr int NW = N::NW, KT = N::KT, ROWS = N::ROWS, ROWB = N::ROWB, WAVEB = N::WAVEB;
  constexpr int KS = D / 32, CT = D / 16;              // steps of the first product, tiles of channels of the second
  constexpr int KROW = D * KB / 8, VROW = D * VB / 8, SROW = D / 32;  // bytes of a row
  constexpr int KW = KROW / 16;                        // words of a key that a lane holds
  constexpr int VPR = VROW / 16, VN = KT * VPR / 64, VCH = D / VPR;  // pieces of 16 bytes of a row, of a lane, and channels of one
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), l16 = lane & 15, l4 = lane >> 4;
  const CacheView& cv = a.c.c;

  bf16x8 Qf[RT][KS];
  int lim_row[RT];  // the last key of this lane's row in the share
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int r = 16 * rt + l16 < it.rows ? 16 * rt + l16 : it.rows - 1;  // (lanes past the end compute on a copy and store nothing)
    const int q = (it.row0 + r) / a.G, lim = a.causal ? q + it.off : it.nk - 1;
    lim_row[rt] = lim < it.end - 1 ? lim : it.end - 1;
    const __bf16* qp = a.Q + out_row(a, it, r) * D + (D / 4) * l4;
#pragma unroll
    for (int s = 0; s < KS; ++s) Qf[rt][s] = *(const bf16x8*)(qp + 8 * s);
  }
  const int lim_least = a.causal ? it.row0 / a.G + it.off : it.nk - 1;  // keys up to here: seen by all rows

  struct Raw {
    uint32_t K[2][KW];
    u32x4 V[VN];
    uint32_t ks[2], vs[VN];
  };
  // Pages of this wavefront's tiles: lane i has the one of tile i of the next 64.
  const int mask = (1 << cv.page_log2) - 1;
  int pages = 0;
  auto load = [&](int key0, Raw& x) {
    long row = ((long)it.s * cv.Hkv + it.g) * cv.Nk + key0;
    if (cv.table) {
      const int i = (key0 - it.begin) / (NW * KT) & 63;
      if (i == 0) {
        const int t = key0 + lane * (NW * KT);
        pages = cv.table[(long)it.s * cv.table_stride + ((t < it.end ? t : key0) >> cv.page_log2)];
      }
      row = (((long)__builtin_amdgcn_readlane(pages, i) * cv.Hkv + it.g) << cv.page_log2) + (key0 & mask);
    }
    const int last = it.end - 1 - key0;  // (keys past the end repeat the last one)
    const uint8_t *kc = a.c.Kc + row * KROW, *ks = a.c.Ks + row * SROW, *vc = a.c.Vc + row * VROW, *vs = a.c.Vs + row * SROW;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int k = 16 * u + l16 < last ? 16 * u + l16 : last;
      const uint32_t* from = (const uint32_t*)(kc + k * KROW + 4 * KW * l4);
      if constexpr (KW == 2) {
        const u32x2 y = *(const u32x2*)from;
        x.K[u][0] = y[0], x.K[u][1] = y[1];
      } else {
#pragma unroll
        for (int j = 0; j < KW; j += 4) {
          const u32x4 y = *(const u32x4*)(from + j);
          x.K[u][j] = y[0], x.K[u][j + 1] = y[1], x.K[u][j + 2] = y[2], x.K[u][j + 3] = y[3];
        }
      }
      x.ks[u] = ks[k * SROW + l4 * SROW / 4];
    }
#pragma unroll
    for (int u = 0; u < VN; ++u) {
      const int i = 64 * u + lane, c = i % VPR, k = i / VPR < last ? i / VPR : last;
      x.V[u] = *(const u32x4*)(vc + k * VROW + 16 * c);
      x.vs[u] = vs[k * SROW + c * VCH / 32];
    }
  };

  f32x4 O[RT][CT];
  float m[RT], l[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) O[rt][ct] = (f32x4){0.f, 0.f, 0.f, 0.f};
    m[rt] = -INFINITY;
    l[rt] = 0.f;
  }
  const float c2 = a.scale_log2e;
  char* const vt = smem + w * WAVEB;
  // this lane's places: writes of V, transposing reads
  const int vread = 4 * l4 + (l16 >> 2), vcol = (l16 & 3) >> 1, vhalf = 8 * (l16 & 1);

  auto compute = [&](int key0, const Raw& x) {
    const bool edge = key0 + KT - 1 > lim_least || key0 + KT > it.end;
    // ---- V through LDS. (Where some rows do not see a key that is NaN, its blocks go in as zeros and the rows that do see it get their NaN below.)
    bool none[VN];
#pragma unroll
    for (int u = 0; u < VN; ++u) {
      const int i = 64 * u + lane, c = i % VPR, k = i / VPR, f = v_swizzle<D, VB>(k);
      none[u] = edge && x.vs[u] == 255u;
      const float s = mx_scale(none[u] ? 127u : x.vs[u]);
#pragma unroll
      for (int j = 0; j < VCH / 8; ++j) {
        const uint32_t w0 = VB == 4 ? x.V[u][j] : x.V[u][(2 * j) & 3], w1 = VB == 4 ? 0u : x.V[u][(2 * j + 1) & 3];
        *(bf16x8*)(vt + k * ROWB + 16 * ((c * (VCH / 8) + j) ^ f)) = mx_decode8<VB, F16>(none[u] ? 0u : w0, none[u] ? 0u : w1, s);
      }
    }
    // ---- S^T = K Q^T
    f32x4 S[RT][2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const float s = mx_scale(x.ks[u]);
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) S[rt][u] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int t = 0; t < KS; ++t) {
        const bf16x8 k = KB == 4 ? mx_decode8<KB, F16>(x.K[u][t], 0u, s) : mx_decode8<KB, F16>(x.K[u][(2 * t) % KW], x.K[u][(2 * t + 1) % KW], s);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) S[rt][u] = mfma16<F16>(k, Qf[rt][t], S[rt][u]);
      }
    }
    if (edge) {
#pragma unroll
      for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int r = 0; r < 4; ++r) S[rt][u][r] = key0 + 16 * u + 4 * l4 + r > lim_row[rt] ? -INFINITY : S[rt][u][r];
    }
    // ---- online softmax
    bf16x8 P[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      auto advance = [&]() {
        float mx = S[rt][0][0];
#pragma unroll
        for (int i = 1; i < 8; ++i) mx = fmaxf(mx, S[rt][i / 4][i % 4]);
        const float m_new = fmaxf(m[rt], max_of_four(mx));
        const float alpha = m_new == -INFINITY ? 1.f : fast_exp2((m[rt] - m_new) * c2);
        l[rt] *= alpha;
        m[rt] = m_new;
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) O[rt][ct] *= alpha;
      };
      f32x4 E[2];
      float rs;
      auto exponentials = [&]() {
        const float ref = m[rt] == -INFINITY ? 0.f : m[rt] * c2;
        rs = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          E[i / 4][i % 4] = fast_exp2(__builtin_fmaf(S[rt][i / 4][i % 4], c2, -ref));
          rs += E[i / 4][i % 4];
        }
      };
      if (__builtin_amdgcn_ballot_w64(m[rt] == -INFINITY)) advance();
      exponentials();
      if (reference_outgrown<F16>(rs)) {
        advance();
        exponentials();
      }
      l[rt] += rs;
      u32x4 p;
      p[0] = pack2<F16>(E[0][0], E[0][1]);
      p[1] = pack2<F16>(E[0][2], E[0][3]);
      p[2] = pack2<F16>(E[1][0], E[1][1]);
      p[3] = pack2<F16>(E[1][2], E[1][3]);
      P[rt] = __builtin_bit_cast(bf16x8, p);
    }
    // ---- O^T += V^T P^T
    asm volatile("" ::: "memory");
    const int f = v_swizzle<D, VB>(vread);  // (keys 16 further on have the same)
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
      const int at = vread * ROWB + 16 * ((2 * ct + vcol) ^ f) + vhalf;
      const bf16x8 v = lds_tr_pair(vt, at, at + 16 * ROWB);
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) O[rt][ct] = mfma16<F16>(v, P[rt], O[rt][ct]);
    }
    asm volatile("" ::: "memory");
    if (edge) {
#pragma unroll
      for (int u = 0; u < VN; ++u)
        for (unsigned long long b = __builtin_amdgcn_ballot_w64(none[u]); b; b &= b - 1) {
          const int i = 64 * u + __builtin_ctzll(b), k = key0 + i / VPR, blk = i % VPR * VCH / 32;
#pragma unroll
          for (int rt = 0; rt < RT; ++rt)
#pragma unroll
            for (int ct = 0; ct < CT; ++ct)
              if (ct / 2 == blk && k <= lim_row[rt]) O[rt][ct] = (f32x4){NAN, NAN, NAN, NAN};
        }
    }
  };

  Raw A, B;
  int t = it.begin + KT * w;
  if (t < it.end) {
    load(t, A);
    while (true) {
      if (t + NW * KT < it.end) load(t + NW * KT, B);
      compute(t, A);
      if ((t += NW * KT) >= it.end) break;
      if (t + NW * KT < it.end) load(t + NW * KT, A);
      compute(t, B);
      if ((t += NW * KT) >= it.end) break;
    }
  }

  // ---- the wavefronts' partial results become the item's: rows of pieces of four channels, their places XOR-ed with the row
  constexpr int CPR = D / 4;
  float lsum[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) lsum[rt] = sum_of_four(l[rt]);
  __syncthreads();
  float* stat = (float*)(smem + N::STAT_OFF);
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    char* const mine = smem + w * WAVEB + (16 * rt + l16) * (4 * D);
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) *(f32x4*)(mine + 16 * ((4 * ct + l4) ^ l16)) = O[rt][ct];
    if (l4 == 0) {
      stat[w * ROWS + 16 * rt + l16] = m[rt];
      stat[NW * ROWS + w * ROWS + 16 * rt + l16] = lsum[rt];
    }
  }
  __syncthreads();
  for (int i = tid; i < it.rows * CPR; i += 64 * NW) {
    const int r = i / CPR, c = i % CPR;
    float mm = -INFINITY;
#pragma unroll
    for (int u = 0; u < NW; ++u) mm = fmaxf(mm, stat[u * ROWS + r]);
    float den = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int u = 0; u < NW; ++u) {
      const float mw = stat[u * ROWS + r], wgt = mw == -INFINITY ? 0.f : fast_exp2((mw - mm) * c2);
      den += wgt * stat[NW * ROWS + u * ROWS + r];
      o += *(const f32x4*)(smem + u * WAVEB + r * (4 * D) + 16 * (c ^ (r & 15))) * wgt;
    }
    const float inv = den == 0.f ? 0.f : 1.f / den;  // (no visible key: L = -inf; a NaN stays one)
    const float lse = den == 0.f ? -INFINITY : mm * a.scale + fast_log2(den) * kLn2;
    const long at = out_row(a, it, r);
    if (direct) {
      if (den == 0.f) o = (f32x4){0.f, 0.f, 0.f, 0.f};
      u32x2 x;
      x[0] = pack2<F16>(o[0] * inv, o[1] * inv);
      x[1] = pack2<F16>(o[2] * inv, o[3] * inv);
      *(u32x2*)(a.O + at * D + 4 * c) = x;
      if (c == 0) *lse_at(a, at) = lse;
    } else {
      const long all = (long)a.nseq * a.Nq * a.Hq;
      *(f32x4*)(a.Opart + (it.slot * all + at) * D + 4 * c) = o * inv;
      if (c == 0) a.Lpart[it.slot * all + at] = lse;
    }
  }
}

// Wavefronts of a SIMD: what registers allow
constexpr int narrow_waves(int D, int bits, int RT) { return D == 64 ? (RT == 1 ? 4 : 3) : (RT == 1 && bits == 8 ? 3 : 2); }
template <int D, bool F16, int KB, int VB, int RT>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(narrow_waves(D, KB + VB, RT), narrow_waves(D, KB + VB, RT)))) void qattend_narrow_kernel(QAttendArgs a, QAttendPlan plan) {
  __shared__ __attribute__((aligned(1024))) char smem[Narrow<D, KB, VB, RT>::LDS];
  const int blocks = (a.Nq * a.G + plan.rows - 1) / plan.rows, per = blocks * plan.shares;
  const int pair = blockIdx.x / (unsigned)per, in = blockIdx.x - (unsigned)pair * per;
  const QItem it = make_item(a, plan, pair, in / plan.shares, in % plan.shares);
  const bool direct = plan.shares == 1;
  if (it.begin >= it.end) return empty_item<D>(a, it, direct);
  narrow_item<D, F16, KB, VB, RT>(a, it, direct, smem);
}

template <int D, bool F16, int FLY>
__global__ __launch_bounds__(256) void qattend_merge_kernel(QAttendArgs a, int slots) {
  merge_slots<D, F16, FLY>(a.Opart, a.Lpart, a.O, a.LSE, (long)a.nseq * a.Nq * a.Hq, a.Hq, a.Nq, slots);
}

template <int D, bool F16, int KB, int VB>
hipError_t launch_bits(const QAttendArgs& a, const QAttendPlan& plan, hipStream_t st) {
  const long items = (long)a.nseq * a.c.c.Hkv * (((long)a.Nq * a.G + plan.rows - 1) / plan.rows) * plan.shares;
  if (items > 0x7fffffffL) return hipErrorInvalidConfiguration;
  const dim3 grid((unsigned)items), block(256);
  if (plan.rows == 16) hipLaunchKernelGGL((qattend_narrow_kernel<D, F16, KB, VB, 1>), grid, block, 0, st, a, plan);
  else hipLaunchKernelGGL((qattend_narrow_kernel<D, F16, KB, VB, 2>), grid, block, 0, st, a, plan);
  return hipGetLastError();
}
template <int D, bool F16>
hipError_t launch_type(const QAttendArgs& a, hipStream_t st) {
  const QAttendPlan plan = qattend_plan(a.nseq, a.Hq, a.c.c.Hkv, a.Nq, a.c.c.Nk, D);
  const hipError_t e = plan.rows == 128 ? launch_qattend_wide(a, plan, st) : a.c.k_bits == 4 ? (a.c.v_bits == 4 ? launch_bits<D, F16, 4, 4>(a, plan, st) : launch_bits<D, F16, 4, 8>(a, plan, st))
                                       : (a.c.v_bits == 4 ? launch_bits<D, F16, 8, 4>(a, plan, st) : launch_bits<D, F16, 8, 8>(a, plan, st));
  const int slots = plan.shares;
  if (e || slots == 1) return e;
  constexpr int RPB = 256 / (D / 4);
  const dim3 grid((unsigned)(((long)a.nseq * a.Nq * a.Hq + RPB - 1) / RPB));
  if (slots <= 4) hipLaunchKernelGGL((qattend_merge_kernel<D, F16, 4>), grid, dim3(256), 0, st, a, slots);
  else hipLaunchKernelGGL((qattend_merge_kernel<D, F16, 16>), grid, dim3(256), 0, st, a, slots);
  return hipGetLastError();
}

}  // namespace

QAttendPlan qattend_plan(int B, int Hq, int Hkv, int Nq, int Nk, int d) {
  QAttendPlan p;
  const long rows = (long)Nq * (Hq / Hkv);
  p.rows = rows <= 16 ? 16 : (rows <= 64 ? 32 : 128);
  const long items = (long)B * Hkv * ((rows + p.rows - 1) / p.rows), blocks = ((long)Nk + 63) / 64;
  long shares = (p.rows == 128 ? 512 : 768) / items;
  shares = std::max(1l, std::min(std::min(shares, 128l), blocks / 4));
  const long per = (blocks + shares - 1) / shares;
  p.keys = (int)(64 * per);
  p.shares = (int)((blocks + per - 1) / per);
  return p;
}

hipError_t launch_qattend(const QAttendArgs& a, hipStream_t st) {
  if (a.c.c.d == 64) return a.f16 ? launch_type<64, true>(a, st) : launch_type<64, false>(a, st);
  return a.f16 ? launch_type<128, true>(a, st) : launch_type<128, false>(a, st);
}

}  // namespace fa
