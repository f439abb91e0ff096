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
