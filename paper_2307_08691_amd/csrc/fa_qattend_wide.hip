// Attention over a key/value cache held in 4 or 8 bits (fa_mx.h) for many rows a key/value head: chunks of prompts. A block is 128 packed rows,
// against a segment of the keys (fa_qattend.h); each of the four wavefronts has 32 rows, and they share tiles of 64 keys in LDS, which hold 16-bit elements:
// every thread converts a quarter of a key's channels of K and of V on the way from memory (one block of 32, or half of one), requested an
// iteration earlier. The loop is that of the shared prefix's wide items (fa_prefix.hip): scores of the next tile beside the exponentials of
// this one, then O^T += V^T P^T, operands requested a few products ahead. Two workgroups share a compute unit. Bound by the matrix units
// and the vector instructions beside them. (4 chunks of 512 queries, 32 heads on 8 of 128, over 4 bits of up to 8192 keys: 428 us by the kernel of
// few rows, 245 by this one with pages looked up by every thread, 193 with the merge now; the products are 131 us of the largest matrix product's rate.)
#include <hip/hip_runtime.h>

#include <type_traits>

#include "fa_lds.h"
#include "fa_qattend.h"

namespace fa {

namespace {

template <int D>
struct Wide {
  static constexpr int BC = 64, ROWB = 2 * D, TILEB = BC * ROWB, V_OFF = 2 * TILEB, FLAGS_OFF = 4 * TILEB, LDS = FLAGS_OFF + 2 * 4 * BC;
};

template <int D, bool F16, int KB, int VB>
__device__ __forceinline__ void wide_segment(const QAttendArgs& a, const QAttendPlan& plan, const QSegment& it, char* smem) {
  typedef Wide<D> W;
  constexpr int BC = W::BC, ROWB = W::ROWB, TILEB = W::TILEB, V_OFF = W::V_OFF, KS = D / 16, DT = D / 32, AHEAD = 4;
  constexpr int CH = D / 4, CHUNKS = CH / 8, KW = CH * KB / 32, VW = CH * VB / 32;  // of a thread and tile: channels, 16-byte pieces of 16-bit ones, words
  const CacheView& cv = a.c.c;
  int tid = threadIdx.x;  // (hidden from the compiler: nothing that follows from it is to live across segments)
  asm volatile("" : "+v"(tid));
  const int lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), lq = lane & 31, hh = lane >> 5;
  const int r0 = 32 * w, mine = r0 + lq;  // this lane's row of the item
  const int prow = mine < it.rows ? mine : it.rows - 1, q = (it.row0 + prow) / a.G;
  // this thread's part of a tile: 16 keys beside each other in 16 lanes, whose pieces then lie in different banks
  struct Part {
    int key, quarter;
  };
  auto part = [&]() {
    int ln = lane;  // (hidden from the compiler, which would keep what follows from it in registers across the loop)
    asm volatile("" : "+v"(ln));
    return Part{16 * w + (ln & 15), ln >> 4};
  };
  const int lim = a.causal ? q + it.off : it.len - 1, lim_end = lim < it.end - 1 ? lim : it.end - 1;
  const int lim_least = a.causal ? (it.row0 + r0) / a.G + it.off : it.len - 1;  // keys up to here: seen by all rows of the wavefront
  const int lim_item = a.causal ? it.row0 / a.G + it.off : it.len - 1;          // ... of the item

  const Part at = part();
  struct Raw {
    uint32_t k[KW], v[VW], ks, vs;
  };
  const int mask = (1 << cv.page_log2) - 1;
  // Row in which the tile that K was last requested of begins; V of it is requested next. Pages: lane i has that of tile i of the next 64.
  long row_k = 0;
  int pages = 0;
  auto next_row = [&](int key0) {
    if (!cv.table) {
      row_k = ((long)it.s * cv.Hkv + it.g) * cv.Nk + key0;
      return;
    }
    const int i = (key0 - it.begin) / BC & 63;
    if (i == 0) {
      const int t = key0 + lane * BC;
      pages = cv.table[(long)it.s * cv.table_stride + ((t < it.end ? t : key0) >> cv.page_log2)];
      touch(pages);
    }
    row_k = (((long)__builtin_amdgcn_readlane(pages, i) * cv.Hkv + it.g) << cv.page_log2) + (key0 & mask);
  };
  auto words = [&](auto N, const uint8_t* from, uint32_t* to) {
    if constexpr (decltype(N)::value == 2) {
      const u32x2 y = *(const u32x2*)from;
      to[0] = y[0], to[1] = y[1];
    } else {
#pragma unroll
      for (int j = 0; j < decltype(N)::value; j += 4) {
        const u32x4 y = *(const u32x4*)(from + 4 * j);
        to[j] = y[0], to[j + 1] = y[1], to[j + 2] = y[2], to[j + 3] = y[3];
      }
    }
  };
  auto request_k = [&](int key0, Raw& x) {  // (keys past the end repeat the last one)
    const auto [tk, quarter] = part();
    next_row(key0);
    const long row = row_k + (tk < it.end - 1 - key0 ? tk : it.end - 1 - key0);
    words(std::integral_constant<int, KW>{}, a.c.Kc + row * (D * KB / 8) + quarter * (4 * KW), x.k);
    x.ks = a.c.Ks[row * (D / 32) + quarter * D / 128];
  };
  auto request_v = [&](int key0, Raw& x) {
    const auto [tk, quarter] = part();
    const long row = row_k + (tk < it.end - 1 - key0 ? tk : it.end - 1 - key0);
    words(std::integral_constant<int, VW>{}, a.c.Vc + row * (D * VB / 8) + quarter * (4 * VW), x.v);
    x.vs = a.c.Vs[row * (D / 32) + quarter * D / 128];
  };
  auto put_k = [&](const Raw& x, int to) {
    const int tk = at.key, quarter = at.quarter;
    const float s = mx_scale(x.ks);
#pragma unroll
    for (int j = 0; j < CHUNKS; ++j) {
      const bf16x8 y = KB == 4 ? mx_decode8<KB, F16>(x.k[j % KW], 0u, s) : mx_decode8<KB, F16>(x.k[(2 * j) % KW], x.k[(2 * j + 1) % KW], s);
      *(bf16x8*)(smem + to + swz_off<ROWB>(tk, quarter * CHUNKS + j)) = y;
    }
  };
  // (Where some row does not see a key of the tile, elements that are not finite go in as zeros, and the rows that see them get them after the product.)
  auto put_v = [&](Raw& x, int key0, int stage) {
    const int tk = at.key, quarter = at.quarter;
    if (key0 + BC - 1 > lim_item || key0 + BC > it.end) {
      const bool past = mx_past_type<VB, F16>(x.v, x.vs);
      const auto [k4, q4] = part();
      smem[W::FLAGS_OFF + stage * 4 * BC + 4 * k4 + q4] = past;
      if (past) mx_drop_past_type<VB, F16>(x.v, x.vs);
    }
    const float s = mx_scale(x.vs);
#pragma unroll
    for (int j = 0; j < CHUNKS; ++j) {
      const bf16x8 y = VB == 4 ? mx_decode8<VB, F16>(x.v[j % VW], 0u, s) : mx_decode8<VB, F16>(x.v[(2 * j) % VW], x.v[(2 * j + 1) % VW], s);
      *(bf16x8*)(smem + V_OFF + stage * TILEB + swz_off<ROWB>(tk, quarter * CHUNKS + j)) = y;
    }
  };

  Raw next;
  request_k(it.begin, next);
  request_v(it.begin, next);
  bf16x8 Qf[KS];
  {
    const __bf16* qp = a.Q + out_row(a, it, prow).at * D + 8 * hh;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) Qf[ks] = *(const bf16x8*)(qp + 16 * ks);
  }
  put_k(next, 0);
  put_v(next, it.begin, 0);
  if (it.begin + BC < it.end) {
    request_k(it.begin + BC, next);
    put_k(next, TILEB);
    request_v(it.begin + BC, next);
    if (it.begin + 2 * BC < it.end) request_k(it.begin + 2 * BC, next);
  }
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
  auto hide = [&](f32x16 (&S)[2], int key0) {
    if (key0 + BC - 1 > lim_least || key0 + BC > it.end) {
      asm volatile("; keep this a branch" ::);
      mask_past(S, lim_end - key0 - 4 * hh);
    }
  };
  __syncthreads();
  f32x16 Sa[2], Sb[2];
  scores(Sa, 0);
  hide(Sa, it.begin);
  m = row_maximum(Sa);
  // Iteration of the tile at key0 (stage `buf`). On entry `next` holds V of the next tile and K of the one after it.
  auto iteration = [&](int key0, auto BUF, f32x16 (&S)[2], f32x16 (&Sn)[2]) {
    constexpr int buf = decltype(BUF)::value;
    const bool more = key0 + BC < it.end;
    __syncthreads();
    if (more) {
      put_v(next, key0 + BC, buf ^ 1);
      if (key0 + 2 * BC < it.end) {
        put_k(next, buf * TILEB);
        request_v(key0 + 2 * BC, next);
        if (key0 + 3 * BC < it.end) request_k(key0 + 3 * BC, next);
      }
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
    if (key0 + BC - 1 > lim_item || key0 + BC > it.end) {
      int ln = lane;  // (hidden from the compiler, as in part())
      asm volatile("" : "+v"(ln));
      const uint32_t past = *(const uint32_t*)(smem + W::FLAGS_OFF + buf * 4 * BC + 4 * ln);  // of key `ln` of the tile
      for (unsigned long long b = __builtin_amdgcn_ballot_w64(past != 0u); b; b &= b - 1) {
        const int k = __builtin_ctzll(b);
        if (key0 + k >= it.end) break;  // (the last key once more)
        const uint32_t which = (uint32_t)__builtin_amdgcn_readlane((int)past, k);
        const long row = mx_row(cv, it.s, it.g, key0 + k);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
          if (!((which >> (8 * (4 / DT) * dt)) & (DT == 4 ? 0xffu : 0xffffu))) continue;
          const uint32_t ee = a.c.Vs[row * (D / 32) + dt];
#pragma unroll
          for (int r4 = 0; r4 < 4; ++r4) {
            const f32x4 x = mx_past_type4<VB, F16>(a.c.Vc + row * (D * VB / 8) + (32 * dt + 8 * r4 + 4 * (ln >> 5)) * VB / 8, ee);
            if (key0 + k <= lim_end)
#pragma unroll
              for (int u = 0; u < 4; ++u) O[dt][4 * r4 + u] += x[u];
          }
        }
      }
    }
    if (more) hide(Sn, key0 + BC);
  };
  using B0 = std::integral_constant<int, 0>;
  using B1 = std::integral_constant<int, 1>;
  for (int key0 = it.begin;;) {
    iteration(key0, B0{}, Sa, Sb);
    if ((key0 += BC) >= it.end) break;
    iteration(key0, B1{}, Sb, Sa);
    if ((key0 += BC) >= it.end) break;
  }
  // ---- through LDS, so that whole rows are stored
  const float lsum = sum_with_partner32(l);
  const float inv = lsum == 0.f ? 0.f : 1.f / lsum;
  const float lse = lsum == 0.f ? -INFINITY : m * a.scale + fast_log2(lsum) * kLn2;
  __syncthreads();  // everyone has read the last tiles
  char* const stage = smem + w * (32 * 4 * D);
  if (it.slot < 0) {
    store_rows_via_lds<DT, F16>(stage, O, inv, [&](int r) { return a.O + out_row(a, it, r0 + r).at * D; }, it.rows - r0, D, lane);
    if (hh == 0 && mine < it.rows) a.LSE[out_row(a, it, mine).lse] = lse;
  } else {
    constexpr int CPR = D / 4;  // 16-byte chunks of a row
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
      if (r0 + r < it.rows) *(f32x4*)(part_o(a, plan, it.slot, r0 + r) + 4 * c) = o;
    }
    if (hh == 0 && mine < it.rows) a.Lpart[(long)it.slot * plan.rows + mine] = lse;
  }
  __syncthreads();
}

template <int D, bool F16, int KB, int VB>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2))) void qattend_wide_kernel(QAttendArgs a, QAttendPlan plan) {
  __shared__ __attribute__((aligned(1024))) char smem[Wide<D>::LDS];
  for_segments(a, plan, smem, [&](const QSegment& it) { wide_segment<D, F16, KB, VB>(a, plan, it, smem); });
}

template <int D, bool F16>
hipError_t launch_type(const QAttendArgs& a, const QAttendPlan& plan, hipStream_t st) {
  const dim3 grid((unsigned)plan.groups), block(256);
  if (a.c.k_bits == 4 && a.c.v_bits == 4) hipLaunchKernelGGL((qattend_wide_kernel<D, F16, 4, 4>), grid, block, 0, st, a, plan);
  else if (a.c.k_bits == 4) hipLaunchKernelGGL((qattend_wide_kernel<D, F16, 4, 8>), grid, block, 0, st, a, plan);
  else if (a.c.v_bits == 4) hipLaunchKernelGGL((qattend_wide_kernel<D, F16, 8, 4>), grid, block, 0, st, a, plan);
  else hipLaunchKernelGGL((qattend_wide_kernel<D, F16, 8, 8>), grid, block, 0, st, a, plan);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_qattend_wide(const QAttendArgs& a, const QAttendPlan& plan, hipStream_t st) {
  if (a.c.c.d == 64) return a.f16 ? launch_type<64, true>(a, plan, st) : launch_type<64, false>(a, plan, st);
  return a.f16 ? launch_type<128, true>(a, plan, st) : launch_type<128, false>(a, plan, st);
}

}  // namespace fa
