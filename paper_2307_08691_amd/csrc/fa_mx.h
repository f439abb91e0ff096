// Caches held in 4 or 8 bits: where a slot's codes and scales lie, and what they stand for.
//
// Blocks of 32 consecutive channels of a row share a scale byte e, which stands for 2^(e - 127) (255: every element is NaN); elements are
// E2M1 (4 bits: 0, 0.5, 1, 1.5, 2, 3, 4, 6 and a sign; the even channel in the low half of a byte) or E4M3 (8 bits). A power of two
// as the scale makes quantising exact up to the one rounding of the element, and an element times its scale exact in bfloat16 and, within
// its range, in half precision: gfx950 converts two elements with their scale in one instruction (v_cvt_scalef32_pk_*).
// Codes [pages, Hkv, page, d * bits / 8] and scales [pages, Hkv, page, d / 32] (slabs [nseq, Hkv, Nk, ..]): the slots of a head follow each
// other, so that 32 of them are one piece of memory for the attention of that head.
#pragma once
#include "fa_kernels.h"

namespace fa {

typedef __attribute__((ext_vector_type(2))) short s16x2;
typedef __attribute__((ext_vector_type(8))) unsigned short u16x8;

// Row of the codes (and of the scales) in which head g of sequence s keeps slot c
__device__ __forceinline__ long mx_row(const CacheView& v, int s, int g, int c) {
  if (!v.table) return ((long)s * v.Hkv + g) * v.Nk + c;
  const int page = v.table[(long)s * v.table_stride + (c >> v.page_log2)];
  return (((long)page * v.Hkv + g) << v.page_log2) + (c & ((1 << v.page_log2) - 1));
}

__device__ __forceinline__ float mx_scale(uint32_t e) { return __builtin_bit_cast(float, e << 23); }  // (255: read as NaN by the conversions)

// Eight elements (4 bits: one word, 8 bits: two) times their scale, as 16-bit elements
template <int BITS, bool F16>
__device__ __forceinline__ bf16x8 mx_decode8(uint32_t w0, uint32_t w1, float s) {
  u32x4 r;
  if constexpr (BITS == 4 && F16) {
    r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w0, s, 0));
    r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w0, s, 1));
    r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w0, s, 2));
    r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w0, s, 3));
  } else if constexpr (BITS == 4) {
    r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w0, s, 0));
    r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w0, s, 1));
    r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w0, s, 2));
    r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w0, s, 3));
  } else if constexpr (F16) {
    r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w0, s, false));
    r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w0, s, true));
    r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w1, s, false));
    r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w1, s, true));
  } else {
    r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, s, false));
    r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, s, true));
    r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, s, false));
    r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, s, true));
  }
  return __builtin_bit_cast(bf16x8, r);
}

// ---- Elements that are no finite 16-bit number: blocks of e = 255, E4M3's own NaN codes, and values that round past the type's range. A product
// with them is NaN also where the weight is zero, so that what hides a key from some rows has to take them out of the product and give them to the
// rows that do see it.

// Whether a piece of a block may have one
template <int BITS, bool F16, int N>
__device__ __forceinline__ bool mx_past_type(const uint32_t (&w)[N], uint32_t e) {
  // (elements up to 6 and 448; from these scales on 4 and 256 of them are 2^16 or 2^128)
  bool past = e >= (F16 ? (BITS == 4 ? 141u : 135u) : (BITS == 4 ? 253u : 247u));
  if constexpr (BITS == 8) {
#pragma unroll
    for (int j = 0; j < N; ++j) past |= (((w[j] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) != 0u;
  }
  return past;
}
template <bool F16>
__device__ __forceinline__ bool not_finite16(bf16x8 y, int t) {
  const uint32_t mask = F16 ? 0x7c00u : 0x7f80u;
  return ((uint32_t)__builtin_bit_cast(u16x8, y)[t] & mask) == mask;
}
// The piece without them: zeros in their place
template <int BITS, bool F16, int N>
__device__ __forceinline__ void mx_drop_past_type(uint32_t (&w)[N], uint32_t& e) {
#pragma unroll
  for (int j = 0; j < N * 4 / BITS; ++j) {
    uint32_t& w0 = w[BITS == 4 ? j : 2 * j];
    uint32_t& w1 = w[BITS == 4 ? j : 2 * j + 1];
    const bf16x8 y = mx_decode8<BITS, F16>(w0, BITS == 4 ? 0u : w1, mx_scale(e));
#pragma unroll
    for (int t = 0; t < 8; ++t) {
      const uint32_t code = not_finite16<F16>(y, t) ? (BITS == 4 ? 0xfu : 0xffu) << (BITS * t % 32) : 0u;
      if (BITS == 4 || t < 4) w0 &= ~code;
      else w1 &= ~code;
    }
  }
  e = e == 255u ? 127u : e;
}
// Of four elements the ones that were taken out; zero for the others
template <int BITS, bool F16>
__device__ __forceinline__ f32x4 mx_past_type4(const uint8_t* codes, uint32_t e) {
  const bf16x8 y = mx_decode8<BITS, F16>(BITS == 4 ? (uint32_t) * (const uint16_t*)codes : *(const uint32_t*)codes, 0u, mx_scale(e));
  f32x4 x;
#pragma unroll
  for (int t = 0; t < 4; ++t) x[t] = not_finite16<F16>(y, t) ? widen<F16>(y, t) : 0.f;
  return x;
}

// Eight values over their scale, rounded to the nearest element (halves to even)
template <int BITS>
__device__ __forceinline__ u32x2 mx_encode8(const float (&x)[8], float s) {
  u32x2 w = {0u, 0u};
  if constexpr (BITS == 4) {
    w[0] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w[0], x[0], x[1], s, 0);
    w[0] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w[0], x[2], x[3], s, 1);
    w[0] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w[0], x[4], x[5], s, 2);
    w[0] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w[0], x[6], x[7], s, 3);
  } else {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      s16x2 q = {0, 0};
      q = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(q, x[4 * i], x[4 * i + 1], s, false);
      q = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(q, x[4 * i + 2], x[4 * i + 3], s, true);
      w[i] = __builtin_bit_cast(uint32_t, q);
    }
  }
  return w;
}

// The scale byte of a block whose largest magnitude has the bits `top` (of a float32): the smallest power of two with no element above
// 1.75 * 2^2 (E2M1: 7, half a step from 6) or 1.75 * 2^8 (E4M3: 448, its largest), so that every element is off by half a step at most;
// 16 at least, which keeps every element a normal bfloat16; 255 where an element is not finite.
template <int BITS>
__device__ __forceinline__ uint32_t mx_scale_byte(uint32_t top) {
  if (top >= 0x7f800000u) return 255u;
  const int e = (int)((top + 0x1fffffu) >> 23) - (BITS == 4 ? 2 : 8);
  return (uint32_t)(e < 16 ? 16 : e);
}

}  // namespace fa
