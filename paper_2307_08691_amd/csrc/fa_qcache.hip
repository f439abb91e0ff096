// A key/value cache held in 4 or 8 bits: new rows quantised as they are written (append), and slots read back in 16 bits (read). Both are
// bound by HBM, or the last-level cache where it holds what they touch, and by launch and latency where there are few rows. (Append, 16 heads of
// 64, keys in 8 bits and values in 4, values left in 16 bits as well: 4 x 1531 rows, 60 MB, 11.3 us with inputs and outputs in the last-level cache,
// 14.4 from HBM, 4.2 TB/s; 16 x 2048, 321 MB, 60 us, 5.4 TB/s. One row each of 64 sequences, 3.7 on the device.)
#include <hip/hip_runtime.h>

#include "fa_mx.h"

namespace fa {

// ---- append. One thread has eight channels of a row of K and of V; four neighbouring threads share a block's scale. The rows of a
// (sequence, head) pair follow each other in the launch, so that a workgroup writes one piece of the cache.
template <int BITS, bool F16>
__device__ __forceinline__ void append_piece(bf16x8 raw, uint8_t* codes, uint8_t* scales, long row, int piece, int d, __bf16* out) {
  float x[8];
  uint32_t top = 0;
#pragma unroll
  for (int t = 0; t < 8; ++t) {
    x[t] = widen<F16>(raw, t);
    const uint32_t m = __builtin_bit_cast(uint32_t, x[t]) & 0x7fffffffu;
    top = m > top ? m : top;
  }
#pragma unroll
  for (int o = 1; o <= 2; ++o) {  // over the four lanes of the block (quad_perm [1, 0, 3, 2], then [2, 3, 0, 1])
    const uint32_t y = o == 1 ? (uint32_t)__builtin_amdgcn_mov_dpp((int)top, 0xb1, 0xf, 0xf, true)
                              : (uint32_t)__builtin_amdgcn_mov_dpp((int)top, 0x4e, 0xf, 0xf, true);
    top = y > top ? y : top;
  }
  const uint32_t e = mx_scale_byte<BITS>(top);
  u32x2 w = mx_encode8<BITS>(x, mx_scale(e));
  if (e == 255u) w = (u32x2){0u, 0u};
  uint8_t* const to = codes + (row * d + 8 * piece) * BITS / 8;
  if constexpr (BITS == 4) *(uint32_t*)to = w[0];
  else *(u32x2*)to = w;
  if ((piece & 3) == 0) scales[row * (d / 32) + piece / 4] = (uint8_t)e;
  if (out) *(bf16x8*)out = mx_decode8<BITS, F16>(w[0], w[1], mx_scale(e));
}
template <int KB, int VB, bool F16>
__global__ __launch_bounds__(256) void qappend_kernel(QAppendArgs a) {
  const CacheView& c = a.c.c;
  const unsigned cpr = (unsigned)c.d / 8u, i = blockIdx.x * 256u + threadIdx.x;  // (at most 2^31 pieces)
  const unsigned r = i / cpr;                                                      // (sequence, head, query)
  const int piece = (int)(i - r * cpr);
  const unsigned pair = r / (unsigned)a.Nq;
  const int q = (int)(r - pair * (unsigned)a.Nq), s = (int)(pair / (unsigned)c.Hkv), g = (int)pair - s * c.Hkv;
  if (s >= a.nseq) return;
  const long slot = (long)(c.lens ? c.lens[s] : c.Nk) - a.Nq + q;
  // (the four threads of a block have one row: all of them go on, or none)
  const bool held = slot >= 0 && slot < c.Nk;  // (else a length that is no length of this cache)
  if (!held) return;
  const bf16x8 k = *(const bf16x8*)(a.Kn + s * a.k_bs + q * a.k_ts + g * a.k_hs + 8 * piece);
  const bf16x8 v = *(const bf16x8*)(a.Vn + s * a.v_bs + q * a.v_ts + g * a.v_hs + 8 * piece);
  const long row = mx_row(c, s, g, (int)slot), at = (((long)s * a.Nq + q) * c.Hkv + g) * c.d + 8 * piece;
  append_piece<KB, F16>(k, a.c.Kc, a.c.Ks, row, piece, c.d, a.Kout ? a.Kout + at : nullptr);
  append_piece<VB, F16>(v, a.c.Vc, a.c.Vs, row, piece, c.d, a.Vout ? a.Vout + at : nullptr);
}
template <bool F16>
static void launch_qappend_t(const QAppendArgs& a, hipStream_t st) {
  const long pieces = (long)a.nseq * a.Nq * a.c.c.Hkv * (a.c.c.d / 8);
  const dim3 grid((unsigned)((pieces + 255) / 256)), block(256);
  if (a.c.k_bits == 4 && a.c.v_bits == 4) hipLaunchKernelGGL((qappend_kernel<4, 4, F16>), grid, block, 0, st, a);
  else if (a.c.k_bits == 4) hipLaunchKernelGGL((qappend_kernel<4, 8, F16>), grid, block, 0, st, a);
  else if (a.c.v_bits == 4) hipLaunchKernelGGL((qappend_kernel<8, 4, F16>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((qappend_kernel<8, 8, F16>), grid, block, 0, st, a);
}
hipError_t launch_qappend(const QAppendArgs& a, hipStream_t st) {
  if (a.f16) launch_qappend_t<true>(a, st);
  else launch_qappend_t<false>(a, st);
  return hipGetLastError();
}

// ---- read. A workgroup takes kReadRows slots of a (sequence, head) pair, a thread eight channels of K and V at a time and kFly of those on
// their way together. (16 sequences of up to 4096 slots, 8 heads of 128, 4 bits, packed: 50 us one by one, 45 so; with the two steps
// below 24.7, or 36 where neither codes nor outputs, 155 MB, are in the last-level cache: 4.3 TB/s.)
constexpr int kReadRows = 64, kFly = 4;
template <int BITS>
struct Codes {
  u32x2 w;
  uint8_t e;
  __device__ __forceinline__ void request(const uint8_t* codes, const uint8_t* scales, long row, int piece, int d) {
    const uint8_t* from = codes + (row * d + 8 * piece) * BITS / 8;
    if constexpr (BITS == 4) w[0] = *(const uint32_t*)from;
    else w = *(const u32x2*)from;
    e = scales[row * (d / 32) + piece / 4];
  }
  template <bool F16>
  __device__ __forceinline__ bf16x8 values() const { return mx_decode8<BITS, F16>(w[0], BITS == 4 ? 0u : w[1], mx_scale(e)); }
};
// ONCE: results past the caches (kReadOnce bytes and more) are stored around them: 38.8 us through them, 31.3 so.
constexpr long kReadOnce = 32l << 20;
template <int KB, int VB, bool F16, bool ONCE>
__global__ __launch_bounds__(256) void qread_kernel(QReadArgs a, int tiles) {
  const CacheView& c = a.c.c;
  // (the heads of the same slots beside each other, whose rows are neighbours in the output: 38.8 us, and 45 with the heads apart)
  const unsigned part = blockIdx.x / (unsigned)c.Hkv;
  const int g = (int)(blockIdx.x - part * (unsigned)c.Hkv), s = (int)(part / (unsigned)tiles), tile = (int)(part - (unsigned)s * (unsigned)tiles);
  long first = 0, row0, rows;  // the first slot, where its row goes, and how many rows there are room for
  if (a.cu) {
    row0 = a.cu[s];
    rows = (long)a.cu[s + 1] - row0;
    if (row0 < 0) return;
    rows = rows < a.total - row0 ? rows : a.total - row0;  // (offsets past the outputs: no row of theirs is written)
  } else {
    first = a.first ? a.first[s] : 0;
    row0 = (long)s * a.N;
    rows = a.N;
  }
  // rows of the tile that have a slot: lo .. hi - 1
  const long i0 = (long)tile * kReadRows, n = held_keys(c, s);
  const long lo = i0 > -first ? i0 : -first;
  long hi = i0 + kReadRows < rows ? i0 + kReadRows : rows;
  hi = hi < n - first ? hi : n - first;
  if (lo >= hi) return;
  const int cpr = c.d / 8, pieces = (int)(hi - lo) * cpr;
  for (int j0 = threadIdx.x; j0 < pieces; j0 += 256 * kFly) {
    Codes<KB> k[kFly];
    Codes<VB> v[kFly];
    long at[kFly];
#pragma unroll
    for (int u = 0; u < kFly; ++u) {
      const int j = j0 + 256 * u < pieces ? j0 + 256 * u : j0, i = j / cpr, piece = j - i * cpr;
      const long row = mx_row(c, s, g, (int)(first + lo + i));
      k[u].request(a.c.Kc, a.c.Ks, row, piece, c.d);
      v[u].request(a.c.Vc, a.c.Vs, row, piece, c.d);
      at[u] = ((row0 + lo + i) * c.Hkv + g) * c.d + 8 * piece;
    }
#pragma unroll
    for (int u = 0; u < kFly; ++u) {
      if (j0 + 256 * u >= pieces) break;
      const u32x4 x = __builtin_bit_cast(u32x4, k[u].template values<F16>()), y = __builtin_bit_cast(u32x4, v[u].template values<F16>());
      if constexpr (ONCE) {
        __builtin_nontemporal_store(x, (u32x4*)(a.K + at[u]));
        __builtin_nontemporal_store(y, (u32x4*)(a.V + at[u]));
      } else {
        *(u32x4*)(a.K + at[u]) = x;
        *(u32x4*)(a.V + at[u]) = y;
      }
    }
  }
}
template <int KB, int VB>
static hipError_t launch_qread_b(const QReadArgs& a, hipStream_t st) {
  const long most = a.cu ? (a.total < a.c.c.Nk ? a.total : a.c.c.Nk) : a.N;
  const long tiles = (most + kReadRows - 1) / kReadRows, all = (long)a.nseq * a.c.c.Hkv * tiles;
  const bool once = (a.cu ? a.total : (long)a.nseq * a.N) * a.c.c.Hkv * a.c.c.d * 4 >= kReadOnce;
  const dim3 grid((unsigned)all), block(256);
  if (a.f16 && once) hipLaunchKernelGGL((qread_kernel<KB, VB, true, true>), grid, block, 0, st, a, (int)tiles);
  else if (a.f16) hipLaunchKernelGGL((qread_kernel<KB, VB, true, false>), grid, block, 0, st, a, (int)tiles);
  else if (once) hipLaunchKernelGGL((qread_kernel<KB, VB, false, true>), grid, block, 0, st, a, (int)tiles);
  else hipLaunchKernelGGL((qread_kernel<KB, VB, false, false>), grid, block, 0, st, a, (int)tiles);
  return hipGetLastError();
}
hipError_t launch_qread(const QReadArgs& a, hipStream_t st) {
  if (a.c.k_bits == 4) return a.c.v_bits == 4 ? launch_qread_b<4, 4>(a, st) : launch_qread_b<4, 8>(a, st);
  return a.c.v_bits == 4 ? launch_qread_b<8, 4>(a, st) : launch_qread_b<8, 8>(a, st);
}

}  // namespace fa
