// Queries and keys rotated by their positions: pair i of a row's channels, (x1, x2), turns by the angle a = position * inv_freq[i], where the
// position is that of the token on the pair's axis (text has one; images rows and columns; video time, rows and columns):
//     y1 = x1 cos a - x2 sin a,  y2 = x1 sin a + x2 cos a
// The gradient is the rotation by -a. Channels past the pairs pass through. The angle is the exact product of the two numbers, reduced in
// float64 (a float32 angle would be off by 0.06 at position 10^6), sine and cosine are right to float32, the rotation is float32.
//
// A workgroup has one token and all heads of both tensors, so that a token's sines and cosines are computed once, into LDS; each thread then
// moves VEC channels of either half (or 2 VEC neighbouring ones) at a time. With many heads bound by HBM, a copy's traffic; few tokens by launch and
// latency. (2 x 8192 tokens, 32 + 8 heads of 128, bf16: 65 us, 5.15 TB/s; one token each of 64 sequences, 6.) With few heads most threads have
// nothing to move, and a workgroup's start, its positions and its two barriers are the time, about 0.9 ns a token over the chip: 131072 tokens, bf16,
// 1 + 1 heads of 64 124 us (0.5 TB/s), 8 + 2 of 128 237 (2.8), 16 + 4 of 128 310 (4.3), 32 + 8 of 128 474 (5.7).
#include <hip/hip_runtime.h>

#include "fa_kernels.h"

namespace fa {

constexpr int kRopeMaxPairs = 128;
constexpr long kRopeGrid = 1 << 20;  // workgroups at most (threads of a grid are counted in 32 bits)

// Sine and cosine of position * freq, to float32. Reduced to a quarter turn in float64 (n pi/2 as the sum of two float64, products by
// fused multiply-add: right to 2^-50 for all 32-bit positions and frequencies up to 1), then Taylor series (the next terms are below 2^-53).
__device__ __forceinline__ void sincos_of(int position, float freq, float& sn, float& cs) {
  const double a = (double)position * (double)freq, rest = __builtin_fma((double)position, (double)freq, -a);  // (55 bits in all)
  const double n = __builtin_rint(a * 0.63661977236758134308);  // 2 / pi
  double r = __builtin_fma(-n, 1.5707963267948966192, a);       // pi / 2, and what its float64 leaves
  r = __builtin_fma(-n, 6.123233995736766036e-17, r) + rest;
  const double z = r * r;
  double s = -1.0 / 1307674368000.0;  // r - r^3 / 3! + .. - r^15 / 15!
  s = __builtin_fma(s, z, 1.0 / 6227020800.0);
  s = __builtin_fma(s, z, -1.0 / 39916800.0);
  s = __builtin_fma(s, z, 1.0 / 362880.0);
  s = __builtin_fma(s, z, -1.0 / 5040.0);
  s = __builtin_fma(s, z, 1.0 / 120.0);
  s = __builtin_fma(s, z, -1.0 / 6.0);
  s = __builtin_fma(s * z, r, r);
  double c = 1.0 / 20922789888000.0;  // 1 - r^2 / 2! + .. + r^16 / 16!
  c = __builtin_fma(c, z, -1.0 / 87178291200.0);
  c = __builtin_fma(c, z, 1.0 / 479001600.0);
  c = __builtin_fma(c, z, -1.0 / 3628800.0);
  c = __builtin_fma(c, z, 1.0 / 40320.0);
  c = __builtin_fma(c, z, -1.0 / 720.0);
  c = __builtin_fma(c, z, 1.0 / 24.0);
  c = __builtin_fma(c, z, -0.5);
  c = __builtin_fma(c, z, 1.0);
  const int quarter = (int)(n - 4.0 * __builtin_floor(n * 0.25));  // n mod 4
  const float fs = (float)(quarter & 1 ? c : s), fc = (float)(quarter & 1 ? s : c);
  sn = quarter & 2 ? -fs : fs;
  cs = (quarter + 1) & 2 ? -fc : fc;
}

// VEC elements as they lie in memory
template <int BYTES>
struct Piece;
template <> struct Piece<2> { typedef uint16_t type; };
template <> struct Piece<4> { typedef uint32_t type; };
template <> struct Piece<8> { typedef u32x2 type; };
template <> struct Piece<16> { typedef u32x4 type; };
template <class T, int VEC>
struct Elements {
  T x[VEC];
};
template <class T, int VEC>
__device__ __forceinline__ Elements<T, VEC> load_piece(const T* p) {
  return __builtin_bit_cast(Elements<T, VEC>, *(const typename Piece<sizeof(T) * VEC>::type*)p);
}
template <class T, int VEC>
__device__ __forceinline__ void store_piece(T* p, const Elements<T, VEC>& e) {
  *(typename Piece<sizeof(T) * VEC>::type*)p = __builtin_bit_cast(typename Piece<sizeof(T) * VEC>::type, e);
}

template <class T, int VEC, bool NEIGHBOURS>
__global__ __launch_bounds__(256) void rope_kernel(RopeArgs a) {
  __shared__ float cosine[kRopeMaxPairs], sine[kRopeMaxPairs];
  const unsigned tokens = (unsigned)a.nseq * (unsigned)a.N;
  for (unsigned token = blockIdx.x; token < tokens; token += gridDim.x) {
    const int s = (int)(token / (unsigned)a.N), i = (int)(token - (unsigned)s * (unsigned)a.N);
    if (token != blockIdx.x) __syncthreads();  // (everyone is done with the last token's angles)
    for (int p = threadIdx.x; p < a.pairs; p += 256) {
      int ax = a.axis ? a.axis[p] : 0;
      ax = ax < 0 ? 0 : (ax < a.axes ? ax : a.axes - 1);  // (an axis that is none reads no other memory)
      float sn, cs;
      sincos_of(a.positions[ax * a.p_as + s * a.p_bs + i], a.inv_freq[p], sn, cs);
      cosine[p] = cs;
      sine[p] = a.inverse ? -sn : sn;
    }
    __syncthreads();
    const int turns = a.pairs / VEC, rest = (a.d - 2 * a.pairs) / VEC, per = turns + rest, all = (a.t[0].heads + a.t[1].heads) * per;
    for (int j = threadIdx.x; j < all; j += 256) {
      int h = j / per;
      const int c = j - h * per;
      const bool second = h >= a.t[0].heads;
      const RopeTensor& t = a.t[second ? 1 : 0];
      if (second) h -= a.t[0].heads;
      const T* x = (const T*)t.x + s * t.x_bs + i * t.x_ts + h * t.x_hs;
      T* y = (T*)t.y + s * t.y_bs + i * t.y_ts + h * t.y_hs;
      if (c >= turns) {
        const int at = 2 * a.pairs + (c - turns) * VEC;
        store_piece<T, VEC>(y + at, load_piece<T, VEC>(x + at));
        continue;
      }
      const int at = NEIGHBOURS ? 2 * VEC * c : VEC * c, to = NEIGHBOURS ? at + VEC : at + a.pairs;
      Elements<T, VEC> u = load_piece<T, VEC>(x + at), v = load_piece<T, VEC>(x + to);
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const float cs = cosine[VEC * c + e], sn = sine[VEC * c + e];
        T& p = NEIGHBOURS ? (2 * e < VEC ? u.x[(2 * e) % VEC] : v.x[(2 * e) % VEC]) : u.x[e];
        T& q = NEIGHBOURS ? (2 * e + 1 < VEC ? u.x[(2 * e + 1) % VEC] : v.x[(2 * e + 1) % VEC]) : v.x[e];
        const float x1 = (float)p, x2 = (float)q;
        p = (T)(x1 * cs - x2 * sn);
        q = (T)(x1 * sn + x2 * cs);
      }
      store_piece<T, VEC>(y + at, u);
      store_piece<T, VEC>(y + to, v);
    }
  }
}

template <class T, int VEC>
static void launch_rope_v(const RopeArgs& a, hipStream_t st) {
  const long tokens = (long)a.nseq * a.N;
  const dim3 grid((unsigned)(tokens < kRopeGrid ? tokens : kRopeGrid)), block(256);
  if (a.neighbours) hipLaunchKernelGGL((rope_kernel<T, VEC, true>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((rope_kernel<T, VEC, false>), grid, block, 0, st, a);
}
template <class T>
static void launch_rope_t(const RopeArgs& a, hipStream_t st) {
  if constexpr (sizeof(T) == 2)
    if (a.vec == 8) return launch_rope_v<T, 8>(a, st);
  if (a.vec >= 4) launch_rope_v<T, 4>(a, st);
  else if (a.vec == 2) launch_rope_v<T, 2>(a, st);
  else launch_rope_v<T, 1>(a, st);
}
hipError_t launch_rope(const RopeArgs& a, hipStream_t st) {
  if (a.type == 0) launch_rope_t<float>(a, st);
  else if (a.type == 1) launch_rope_t<__bf16>(a, st);
  else launch_rope_t<_Float16>(a, st);
  return hipGetLastError();
}

}  // namespace fa
