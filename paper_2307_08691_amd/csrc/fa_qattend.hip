// Attention over a key/value cache held in 4 or 8 bits (fa_mx.h): Algorithm 1 over what the codes stand for, with the parallelism of
// decoding. The rows of one (sequence, key/value head), query * G + head of the group, come in blocks of up to 32; the four wavefronts of
// a workgroup take tiles of 32 keys (64 where 32 would be 2 KB) of a segment (fa_qattend.h) in turn, each with a running softmax of its own, no barrier in the loop, and
// join through LDS at the segment's end.
//
// Codes become 16-bit elements in registers, two an instruction, and every product is a 16x16x32 MFMA of those:
//   * S^T = K Q^T: a lane holds a quarter of a key's channels, D / 4 consecutive ones of one block. The order in which channels are summed is
//     free, so step s of the contraction takes eight of each lane's own, and Q is held alike.
//   * O^T += V^T P^T needs keys along a lane's operand, so V goes through LDS again as 16-bit elements, 64 channels at a time, and is
//     read back transposed. P^T is in place already: the keys of a lane's eight operand elements are those whose scores it has.
// Tiles come by direct copies to LDS, whole rows a request, several tiles ahead, and go to registers at once when they are
// there, so that their place is requested again. Bound by HBM, which hands a compute unit 24 bytes a ns: 136 bytes a key of 128 channels in 4 bits.
// (64 paged sequences of up to 8192 keys, 32 heads on 8 of 128, 4 bits: 71 us with rows loaded to registers a lane's part at a time, 64 so, of 49
// for the bytes at 6.25 TB/s. One sequence of 131072 keys, 8 and 4 bits: 42 us with the merge, of 34.)
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

// Tiles of codes in LDS, 32 rows of ROW bytes in pieces of 16: piece c of key k lies at place c ^ mix(k) of its row, so that 16 keys' pieces c
// lie in different banks.
template <int ROW>
__device__ __forceinline__ int code_mix(int k) {
  return ROW == 128 ? (k >> 1) & 7 : (ROW == 64 ? (k >> 2) & 3 : (k >> 3) & 1);
}
// What lane `lane` fetches with request u of a tile: from its first row on, keys past `last` repeating that one
template <int ROW>
__device__ __forceinline__ unsigned code_offset(int u, int lane, int last) {
  const int k = (64 * u + lane) / (ROW / 16), c = (lane % (ROW / 16)) ^ code_mix<ROW>(k);
  return (unsigned)((k < last ? k : last) * ROW + 16 * c);
}
// V as 16-bit elements: 32 rows of 64 channels (128 bytes). Free of conflicts for the writes (16 keys at one piece) and the transposing reads
// (8 keys x 32 bytes; two rows share a line of the banks).
__device__ __forceinline__ int v_mix(int k) { return (k & 6) | ((k >> 3) & 1); }

// 2 bytes a lane from global memory into LDS, a word each (see dma16)
__device__ __forceinline__ void dma2(const void* gaddr, const void* lds) {
  asm volatile("s_mov_b32 m0, %1\n\tglobal_load_lds_ushort %0, off" ::"v"(gaddr), "s"(__builtin_amdgcn_readfirstlane(lds_address(lds))) : "memory");
}

// Keys of a tile: 64 where 32 would be 2 KB (their instructions beside the elements' own: 64 sequences of up to 4096 keys of 64, 4 bits, 29.4 us with
// tiles of 32, 28.0 so; with 8 bits 16 x 16 heads of up to 4096: 17.2 and 18.9)
constexpr int narrow_keys(int d, int bits) { return d == 64 && bits == 8 ? 64 : 32; }
template <int D, int KB, int VB, int RT>
struct Narrow {
  static constexpr int NW = 4, KT = narrow_keys(D, KB + VB), ROWS = 16 * RT, KROW = D * KB / 8, VROW = D * VB / 8, SROW = D / 32;  // bytes of a row of codes, of scales
  static constexpr int KN = KT * KROW / 1024, VN = KT * VROW / 1024, SN = KT / 32, REQUESTS = KN + VN + SN;  // of a tile
  static_assert(KT == 32 || D == 64, "the scales of a tile: 64 words a request");
  static constexpr int STAGEB = KT * (KROW + VROW + 8), VTILE = 32 * 128, PART = ROWS * 4 * D;
  // wavefronts of a SIMD by the registers, and what LDS a wavefront then has
  static constexpr int WAVES = RT == 1 ? 3 : 2, ROOM = 160 * 1024 / (4 * WAVES) - 2 * ROWS * 4 - 64;
  static constexpr int STAGES = (ROOM - VTILE) / STAGEB < 1 ? 1 : ((ROOM - VTILE) / STAGEB > 4 ? 4 : (ROOM - VTILE) / STAGEB);
  static constexpr int WAVEB = STAGES * STAGEB + VTILE > PART ? STAGES * STAGEB + VTILE : PART;
  static constexpr int STAT_OFF = NW * WAVEB, LDS = STAT_OFF + 2 * NW * ROWS * 4;
};

template <int D, bool F16, int KB, int VB, int RT>
__device__ __forceinline__ void narrow_segment(const QAttendArgs& a, const QAttendPlan& plan, const QSegment& it, char* smem) {
  typedef Narrow<D, KB, VB, RT> N;
  constexpr int NW = N::NW, KT = N::KT, ROWS = N::ROWS, WAVEB = N::WAVEB, STAGES = N::STAGES, KROW = N::KROW, VROW = N::VROW, SROW = N::SROW;
  constexpr int KS = D / 32, CT = D / 16, KU = KT / 16;  // steps of the first product, tiles of 16 channels, of 16 keys
  constexpr int HG = D / 64, PK = KT / 32, GROUPS = HG * PK;  // V: groups of 64 channels, of 32 keys, and of both
  constexpr int KW = KROW / 16, VW = VB;                // words that a lane holds of a key's quarter, of 32 channels of V
  constexpr int V_OFF = KT * KROW, S_OFF = V_OFF + KT * VROW;  // in a stage: codes of K, of V, a word of scales a key of each
  int tid = threadIdx.x;  // (hidden from the compiler: nothing that follows from it is to live across segments)
  asm volatile("" : "+v"(tid));
  const int lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), l16 = lane & 15, l4 = lane >> 4;
  const CacheView& cv = a.c.c;
  char* const ring = smem + w * WAVEB;
  char* const vt = ring + STAGES * N::STAGEB;

  bf16x8 Qf[RT][KS];
  int lim_row[RT];  // the last key of this lane's row in the segment
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int r = 16 * rt + l16 < it.rows ? 16 * rt + l16 : it.rows - 1;  // (lanes past the end compute on a copy and store nothing)
    const int q = (it.row0 + r) / a.G, lim = a.causal ? q + it.off : it.len - 1;
    lim_row[rt] = lim < it.end - 1 ? lim : it.end - 1;
    const __bf16* qp = a.Q + out_row(a, it, r).at * D + (D / 4) * l4;
#pragma unroll
    for (int s = 0; s < KS; ++s) Qf[rt][s] = *(const bf16x8*)(qp + 8 * s);
  }
  const int lim_least = a.causal ? it.row0 / a.G + it.off : it.len - 1;  // keys up to here: seen by all rows

  // ---- requests of a tile
  const int t0 = it.begin + KT * w, tiles = t0 < it.end ? (it.end - t0 + NW * KT - 1) / (NW * KT) : 0;
  const int mask = (1 << cv.page_log2) - 1;
  int pages = 0;  // of this wavefront's tiles: lane i has the one of tile i of the next 64
  unsigned koff[N::KN], voff[N::VN];  // where this lane's pieces of a whole tile are
#pragma unroll
  for (int u = 0; u < N::KN; ++u) koff[u] = code_offset<KROW>(u, lane, KT - 1);
#pragma unroll
  for (int u = 0; u < N::VN; ++u) voff[u] = code_offset<VROW>(u, lane, KT - 1);
  auto request = [&](int i, int stage) {
    const int key0 = t0 + i * (NW * KT);
    long row = ((long)it.s * cv.Hkv + it.g) * cv.Nk + key0;
    if (cv.table) {
      if ((i & 63) == 0) {
        const int t = key0 + lane * (NW * KT);
        pages = cv.table[(long)it.s * cv.table_stride + ((t < it.end ? t : key0) >> cv.page_log2)];
        touch(pages);
      }
      row = (((long)__builtin_amdgcn_readlane(pages, i & 63) * cv.Hkv + it.g) << cv.page_log2) + (key0 & mask);
    }
    const int last = it.end - 1 - key0;  // (keys past the end repeat the last one)
    char* const to = ring + stage * N::STAGEB;
    unsigned ko[N::KN], vo[N::VN];
    int k = lane & (KT - 1);
#pragma unroll
    for (int u = 0; u < N::KN; ++u) ko[u] = koff[u];
#pragma unroll
    for (int u = 0; u < N::VN; ++u) vo[u] = voff[u];
    if (last < KT - 1) {
      asm volatile("; keep this a branch" ::);
#pragma unroll
      for (int u = 0; u < N::KN; ++u) ko[u] = code_offset<KROW>(u, lane, last);
#pragma unroll
      for (int u = 0; u < N::VN; ++u) vo[u] = code_offset<VROW>(u, lane, last);
      k = k < last ? k : last;
    }
    const uint8_t *kc = a.c.Kc + row * KROW, *vc = a.c.Vc + row * VROW;
#pragma unroll
    for (int u = 0; u < N::KN; ++u) dma16_uniform_once(kc, ko[u], to + 1024 * u);
#pragma unroll
    for (int u = 0; u < N::VN; ++u) dma16_uniform_once(vc, vo[u], to + V_OFF + 1024 * u);
    // (scales: a word a key of K, then of V)
    const uint8_t* const sc = (KT == 32 && lane >= 32 ? a.c.Vs : a.c.Ks) + row * SROW + k * SROW;
    if constexpr (SROW == 4) dma4(sc, to + S_OFF);
    else dma2(sc, to + S_OFF);
    if constexpr (KT == 64) dma2(a.c.Vs + row * SROW + k * SROW, to + S_OFF + 4 * KT);
  };

  // ---- a tile in registers: of keys 16 u + l16 quarter l4 of the channels of K; of V, group (b, h), of key 32 b + lane % 32 the channels
  // 64 h + 32 (lane / 32) ..
  uint32_t Kr[KU][KW], Vr[GROUPS][VW], ks[KU], vs[PK];
  auto take = [&](int stage) {
    const char* st = ring + stage * N::STAGEB;
#pragma unroll
    for (int u = 0; u < KU; ++u) {
      const int k = 16 * u + l16;
      if constexpr (KW == 2) {
        const u32x2 y = *(const u32x2*)(st + k * KROW + 16 * ((l4 >> 1) ^ code_mix<KROW>(k)) + 8 * (l4 & 1));
        Kr[u][0] = y[0], Kr[u][1] = y[1];
      } else {
#pragma unroll
        for (int j = 0; j < KW / 4; ++j) {
          const u32x4 y = *(const u32x4*)(st + k * KROW + 16 * ((l4 * (KW / 4) + j) ^ code_mix<KROW>(k)));
          Kr[u][4 * j] = y[0], Kr[u][4 * j + 1] = y[1], Kr[u][4 * j + 2] = y[2], Kr[u][4 * j + 3] = y[3];
        }
      }
      ks[u] = *(const uint32_t*)(st + S_OFF + 4 * k);
    }
    const int sub = lane >> 5;
#pragma unroll
    for (int v = 0; v < GROUPS; ++v) {
      const int k = 32 * (v / HG) + (lane & 31);
#pragma unroll
      for (int j = 0; j < VW / 4; ++j) {
        const u32x4 y = *(const u32x4*)(st + V_OFF + k * VROW + 16 * (((2 * (v % HG) + sub) * (VW / 4) + j) ^ code_mix<VROW>(k)));
        Vr[v][4 * j] = y[0], Vr[v][4 * j + 1] = y[1], Vr[v][4 * j + 2] = y[2], Vr[v][4 * j + 3] = y[3];
      }
      if (v % HG == 0) vs[v / HG] = *(const uint32_t*)(st + S_OFF + 4 * (KT + k));
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
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
  const int vread = 4 * l4 + (l16 >> 2), vcol = (l16 & 3) >> 1, vhalf = 8 * (l16 & 1);

  auto compute = [&](int key0) {
    const bool edge = key0 + KT - 1 > lim_least || key0 + KT > it.end;
    // (Where some rows do not see a key, elements of V that are not finite go in as zeros, and the rows that do see it get them below.)
    unsigned long long past[GROUPS];
    uint32_t e[GROUPS];
#pragma unroll
    for (int v = 0; v < GROUPS; ++v) {
      past[v] = 0ull;
      e[v] = (vs[v / HG] >> (8 * (2 * (v % HG) + (lane >> 5)))) & 0xffu;
    }
    if (edge) {
#pragma unroll
      for (int v = 0; v < GROUPS; ++v) {
        past[v] = __builtin_amdgcn_ballot_w64(mx_past_type<VB, F16>(Vr[v], e[v]));
        if (past[v]) mx_drop_past_type<VB, F16>(Vr[v], e[v]);
      }
    }
    auto put_v = [&](int v) {
      const int k = lane & 31, sub = lane >> 5;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t w0 = VB == 4 ? Vr[v][j] : Vr[v][(2 * j) % VW], w1 = VB == 4 ? 0u : Vr[v][(2 * j + 1) % VW];
        *(bf16x8*)(vt + k * 128 + 16 * ((4 * sub + j) ^ v_mix(k))) = mx_decode8<VB, F16>(w0, w1, mx_scale(e[v]));
      }
    };
    put_v(0);
    // ---- S^T = K Q^T
    f32x4 S[RT][KU];
#pragma unroll
    for (int u = 0; u < KU; ++u) {
      const float s = mx_scale((ks[u] >> (8 * (D == 128 ? l4 : l4 >> 1))) & 0xffu);
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) S[rt][u] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int t = 0; t < KS; ++t) {
        const bf16x8 k = KB == 4 ? mx_decode8<KB, F16>(Kr[u][t], 0u, s) : mx_decode8<KB, F16>(Kr[u][(2 * t) % KW], Kr[u][(2 * t + 1) % KW], s);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) S[rt][u] = mfma16<F16>(k, Qf[rt][t], S[rt][u]);
      }
    }
    if (edge) {
#pragma unroll
      for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int u = 0; u < KU; ++u)
#pragma unroll
          for (int r = 0; r < 4; ++r) S[rt][u][r] = key0 + 16 * u + 4 * l4 + r > lim_row[rt] ? -INFINITY : S[rt][u][r];
    }
    // ---- online softmax
    bf16x8 P[RT][PK];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      auto advance = [&]() {
        float mx = S[rt][0][0];
#pragma unroll
        for (int i = 1; i < 4 * KU; ++i) mx = fmaxf(mx, S[rt][i / 4][i % 4]);
        const float m_new = fmaxf(m[rt], max_of_four(mx));
        const float alpha = m_new == -INFINITY ? 1.f : fast_exp2((m[rt] - m_new) * c2);
        l[rt] *= alpha;
        m[rt] = m_new;
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) O[rt][ct] *= alpha;
      };
      f32x4 E[KU];
      float rs;
      auto exponentials = [&]() {
        const float ref = m[rt] == -INFINITY ? 0.f : m[rt] * c2;
        rs = 0.f;
#pragma unroll
        for (int i = 0; i < 4 * KU; ++i) {
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
#pragma unroll
      for (int b = 0; b < PK; ++b) {
        u32x4 p;
        p[0] = pack2<F16>(E[2 * b][0], E[2 * b][1]);
        p[1] = pack2<F16>(E[2 * b][2], E[2 * b][3]);
        p[2] = pack2<F16>(E[2 * b + 1][0], E[2 * b + 1][1]);
        p[3] = pack2<F16>(E[2 * b + 1][2], E[2 * b + 1][3]);
        P[rt][b] = __builtin_bit_cast(bf16x8, p);
      }
    }
    // ---- O^T += V^T P^T, 64 channels of 32 keys at a time (LDS keeps a wavefront's order: the next ones are written behind the reads)
    const int f = v_mix(vread);  // (keys 16 further on have the same)
#pragma unroll
    for (int v = 0; v < GROUPS; ++v) {
      asm volatile("" ::: "memory");
      bf16x8 x[4];
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const int at = vread * 128 + 16 * ((2 * c + vcol) ^ f) + vhalf;
        x[c] = lds_tr_pair(vt, at, at + 16 * 128);
      }
      asm volatile("" ::: "memory");
      if (v + 1 < GROUPS) put_v(v + 1);
#pragma unroll
      for (int c = 0; c < 4; ++c)
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) O[rt][4 * (v % HG) + c] = mfma16<F16>(x[c], P[rt][v / HG], O[rt][4 * (v % HG) + c]);
    }
    asm volatile("" ::: "memory");
    if (edge) {
#pragma unroll
      for (int v = 0; v < GROUPS; ++v)
        for (unsigned long long b = past[v]; b; b &= b - 1) {
          const int i = __builtin_ctzll(b), k = key0 + 32 * (v / HG) + (i & 31), blk = 2 * (v % HG) + (i >> 5);
          if (k >= it.end) continue;  // (the last key once more)
          const long row = mx_row(cv, it.s, it.g, k);  // (from the cache again: the tile's place is another's by now)
          const uint32_t ee = a.c.Vs[row * SROW + blk];
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            const f32x4 x = mx_past_type4<VB, F16>(a.c.Vc + row * VROW + (32 * blk + 16 * c + 4 * l4) * VB / 8, ee);
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
#pragma unroll
              for (int ct = 0; ct < CT; ++ct)
                if (ct == 2 * blk + c && k <= lim_row[rt]) O[rt][ct] += x;
          }
        }
    }
  };

  if (tiles > 0) {
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
      for (int s = 0; s < KS; ++s) touch(Qf[rt][s]);
#pragma unroll
    for (int i = 0; i < STAGES; ++i)
      if (i < tiles) request(i, i);
    for (int i = 0, stage = 0; i < tiles; ++i) {
      if (STAGES > 1 && i + STAGES <= tiles) wait_vmem_upto<(STAGES - 1) * N::REQUESTS>();  // (all that are on their way but this one's)
      else wait_vmem();
      take(stage);
      if (i + STAGES < tiles) request(i + STAGES, stage);
      compute(t0 + i * (NW * KT));
      stage = stage + 1 < STAGES ? stage + 1 : 0;
    }
  }

  // ---- the wavefronts' partial results become the segment's: rows of pieces of four channels, their places XOR-ed with the row
  constexpr int CPR = D / 4;
  float lsum[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) lsum[rt] = sum_of_four(l[rt]);
  float* stat = (float*)(smem + N::STAT_OFF);
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    char* const mine = ring + (16 * rt + l16) * (4 * D);
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
    const float inv = den == 0.f ? 0.f : 1.f / den;  // (no visible key: O = 0, L = -inf; a NaN stays one)
    put_row<F16>(a, plan, it, r, c, o * inv, den == 0.f ? -INFINITY : mm * a.scale + fast_log2(den) * kLn2);
  }
  __syncthreads();
}

template <int D, bool F16, int KB, int VB, int RT>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(Narrow<D, KB, VB, RT>::WAVES, Narrow<D, KB, VB, RT>::WAVES))) void qattend_narrow_kernel(
    QAttendArgs a, QAttendPlan plan) {
  __shared__ __attribute__((aligned(1024))) char smem[Narrow<D, KB, VB, RT>::LDS];
  for_segments(a, plan, smem, [&](const QSegment& it) { narrow_segment<D, F16, KB, VB, RT>(a, plan, it, smem); });
}

// Units that several workgroups have parts of. ONE: a workgroup a row, for few units with many parts; else one for as many rows as it has
// threads for.
template <int D, bool F16, bool ONE>
__global__ __launch_bounds__(256) void qattend_merge_kernel(QAttendArgs a, QAttendPlan p) {
  __shared__ __attribute__((aligned(16))) char parts[ONE ? merge_split_lds<D>() : 16];
  constexpr int AT_ONCE = 256 / (D / 4);
  const int here = ONE ? p.rows : p.rows / AT_ONCE, unit = blockIdx.x / (unsigned)here, part = blockIdx.x % (unsigned)here;
  const int pair = unit / p.blocks, row0 = (unit - pair * p.blocks) * p.rows;
  const int rows = a.Nq * a.G - row0 < p.rows ? a.Nq * a.G - row0 : p.rows;
  const QAttendArgs::Unit u = a.units[unit];
  if (u.parts == 0) return;
  auto slot = [&](int k) { return k == 0 ? 2 * u.first + 1 : 2 * (u.first + k); };
  auto o_at = [&](int k, int r) { return (const float*)part_o(a, p, slot(k), r); };
  auto l_at = [&](int k, int r) { return a.Lpart[(long)slot(k) * p.rows + r]; };
  auto done = [&](int r, int c4, f32x4 o, float lse) {
    QSegment it;
    const int s = pair / a.c.c.Hkv;
    it.s = s, it.g = pair - s * a.c.c.Hkv, it.tok0 = (long)s * a.Nq, it.row0 = row0, it.slot = -1;
    put_row<F16>(a, p, it, r, c4, o, lse);
  };
  const int r = ONE ? part : part * AT_ONCE + (int)threadIdx.x / (D / 4);
  if (r >= rows) return;
  auto partial = [&](int k) { return o_at(k, r); };
  auto logsum = [&](int k) { return l_at(k, r); };
  auto finish = [&](int c4, f32x4 o, float lse) { done(r, c4, o, lse); };
  if constexpr (ONE) merge_split<D>(parts, u.parts, partial, logsum, finish);
  else merge_few<D, 4>(u.parts, partial, logsum, finish);
}

template <int D, bool F16, int KB, int VB>
hipError_t launch_bits(const QAttendArgs& a, const QAttendPlan& plan, hipStream_t st) {
  const dim3 grid((unsigned)plan.groups), block(256);
  if (plan.rows == 16) hipLaunchKernelGGL((qattend_narrow_kernel<D, F16, KB, VB, 1>), grid, block, 0, st, a, plan);
  else hipLaunchKernelGGL((qattend_narrow_kernel<D, F16, KB, VB, 2>), grid, block, 0, st, a, plan);
  return hipGetLastError();
}
template <int D, bool F16>
hipError_t launch_type(const QAttendArgs& a, hipStream_t st) {
  const QAttendPlan plan = qattend_plan(a.nseq, a.Hq, a.c.c.Hkv, a.Nq, a.c.c.Nk, D, a.c.k_bits + a.c.v_bits);
  const hipError_t e = plan.rows == 128 ? launch_qattend_wide(a, plan, st)
                       : a.c.k_bits == 4 ? (a.c.v_bits == 4 ? launch_bits<D, F16, 4, 4>(a, plan, st) : launch_bits<D, F16, 4, 8>(a, plan, st))
                                         : (a.c.v_bits == 4 ? launch_bits<D, F16, 8, 4>(a, plan, st) : launch_bits<D, F16, 8, 8>(a, plan, st));
  if (e || plan.slots == 0) return e;
  const long units = (long)a.nseq * a.c.c.Hkv * plan.blocks;
  if (units * plan.rows <= 4 * plan.groups) hipLaunchKernelGGL((qattend_merge_kernel<D, F16, true>), dim3((unsigned)(units * plan.rows)), dim3(256), 0, st, a, plan);
  else hipLaunchKernelGGL((qattend_merge_kernel<D, F16, false>), dim3((unsigned)(units * (plan.rows / (1024 / D)))), dim3(256), 0, st, a, plan);
  return hipGetLastError();
}

}  // namespace

// Short caches whose units all have a workgroup: nothing is cut, and no merge is launched (us, cut and whole: 96 sequences of up to 1024
// keys, 16 heads on 4 of 64: 15.1 and 11.1; 8 of up to 1024, 8 on 2: 11.1 and 8.2; but 4 of up to 2048, 32 on 8 of 128: 10.9 and 17.2)
constexpr int kWhole = 1024;
QAttendPlan qattend_plan(int B, int Hq, int Hkv, int Nq, int Nk, int d, int bits) {
  QAttendPlan p;
  const long rows = (long)Nq * (Hq / Hkv);
  // Rows of a block. us of a pass, 32 heads on 8 of 128, 4 bits, pages of 64, by blocks of 16, 32 and 128:
  //   rows                             16                  20                   32                   36                  48                   64             128
  //   16 sequences of up to 4096   27  32  41          35  35  40           39  39  42           50  58  42          53  64  43           65  74  44     -  133  49
  //   64 of up to 8192             80 104 196         144 110 197          149 120 197          210 195 197         217 206 199          285 219 202     -  416 216
  // (8 and 8 bits, and 64 channels, rank alike.) Up to 16 rows and from 17 to 32 the choice is the fastest. From 33 to 64 two blocks of 32 read the cache
  // twice and are mostly slower than one of 128, by up to 1.7 times on few sequences and 9% on many.
  p.rows = rows <= 16 ? 16 : (rows <= 64 ? 32 : 128);
  p.blocks = (int)((rows + p.rows - 1) / p.rows);
  // As many workgroups as fit: three a compute unit, or two. Two stream as fast as three where a tile has 6 KB and more, and leave fewer
  // parts to the merge (us at 512 and 768: 131072 keys of 128, 8 and 4 bits, one sequence, 32 heads on 8: 42.2 and 45.3; 16 sequences of up to
  // 8192, 8 and 8: 35.0 and 35.5; but 64 of up to 8192, 4 and 4: 76.5 and 66.0; 64 of up to 4096 of 64 channels, 8 and 8: 39.3 and 34.7). Both sides
  // with LDS and registers for three (Narrow::WAVES), where more than 8 bits of 128 channels have one tile on its way: what two could do with
  // the room that they have is not measured.
  p.groups = p.rows == 16 && !(d == 128 && bits > 8) ? 768 : 512;
  p.chunk_log2 = p.rows != 128 && bits && narrow_keys(d, bits) == 64 ? 8 : 7;  // (narrow: a tile for each of four wavefronts)
  const double units = (double)B * Hkv * p.blocks;
  if (p.rows != 128 && units <= 512 && Nk <= kWhole)  // (whatever the bits: the workspace is sized without them)
    while ((1 << p.chunk_log2) < Nk) ++p.chunk_log2;
  const double chunks = units * (((Nk - 1) >> p.chunk_log2) + 1);
  if (chunks < p.groups) p.groups = (int)chunks;
  p.slots = Nk <= 1 << p.chunk_log2 ? 0 : 2 * p.groups;  // (a unit of one chunk is never shared)
  return p;
}

hipError_t launch_qattend(const QAttendArgs& a, hipStream_t st) {
  if (a.c.c.d == 64) return a.f16 ? launch_type<64, true>(a, st) : launch_type<64, false>(a, st);
  return a.f16 ? launch_type<128, true>(a, st) : launch_type<128, false>(a, st);
}

}  // namespace fa
