// Microscaled 4-bit rows: what the kernels on them share.
//
// A row of dim features is B = ceil(dim / 32) blocks of 32 consecutive ones.  A block has a power of two, held as its
// exponent (byte s: 2^(s - 127); 255: the whole block is NaN), and 32 elements of four bits, sign and magnitude
// (0, 0.5, 1, 1.5, 2, 3, 4, 6), element 2 i in the low half of byte i: 16 bytes, one 16-byte load, and exactly what a lane
// holds of an operand of v_mfma_scale_f32_16x16x128_f8f6f4.  That instruction multiplies 16 rows with 16 rows over four blocks:
// lane l has block l / 16 of row l % 16 of either operand and that block's exponent in a byte of a register of its own;
// of D = A B^T + C it has column l % 16, rows 4 (l / 16) .. + 3.
//
// Its rounding: the 32 products of a block are multiples of 1/4 and their sum is below 2^11, so it is exact; the four block sums are added to
// C one after the other, each time rounded to nearest (1 + 4 terms of 2^-24 gives 1, of 1.5 x 2^-24 1 + 8 x 2^-24; 1 - 4 terms of 0.75 x 2^-24 1 - 4 x
// 2^-24).  Four roundings lose at most 4 x 2^-24 of the sum of the magnitudes (2^-22.2 was seen over 1e6 results with exponents 0 to 30 apart).
#pragma once

#include "som_internal.hpp"

namespace som {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float mx_f32x4 __attribute__((ext_vector_type(4)));
typedef float mx_f32x2 __attribute__((ext_vector_type(2)));
typedef _Float16 mx_f16x2 __attribute__((ext_vector_type(2)));

constexpr double kMx4Delta = 2.384185791015625e-07;       // 2^-22

// D = A B^T + C of 16 x 16 x 128; kA, kB: which byte of scale_a, scale_b holds the lane's exponent.
template <int kA, int kB>
__device__ __forceinline__ mx_f32x4 mx4_mfma(i32x4 a, i32x4 b, mx_f32x4 c, int scale_a, int scale_b) {
  const i32x8 a8 = __builtin_shufflevector(a, a, 0, 1, 2, 3, -1, -1, -1, -1);
  const i32x8 b8 = __builtin_shufflevector(b, b, 0, 1, 2, 3, -1, -1, -1, -1);
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a8, b8, c, 4, 4, kA, scale_a, kB, scale_b);
}

// 2^(s - 127) as the conversions take it: the exponent field of a float (0 means 2^-127, 255 NaN).
__device__ __forceinline__ float mx4_scale(unsigned s) { return __uint_as_float(s << 23); }

// Elements 2 kByte, 2 kByte + 1 of a word of eight, times the scale.
template <int kByte>
__device__ __forceinline__ mx_f32x2 mx4_pair(unsigned word, float scale) {
  return __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, scale, kByte);
}
template <int kByte>
__device__ __forceinline__ mx_f16x2 mx4_pair_f16(unsigned word) {
  return __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(word, 1.0f, kByte);
}

// Dot product of two blocks without their scales, and the second one with itself: exact (multiples of 1/4 below 2^11,
// every partial sum is a float).
__device__ __forceinline__ void mx4_block_dots(i32x4 x, i32x4 w, float &xw, float &ww) {
  float p = 0.f, q = 0.f;
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const mx_f16x2 x0 = mx4_pair_f16<0>(x[u]), x1 = mx4_pair_f16<1>(x[u]), x2 = mx4_pair_f16<2>(x[u]), x3 = mx4_pair_f16<3>(x[u]);
    const mx_f16x2 w0 = mx4_pair_f16<0>(w[u]), w1 = mx4_pair_f16<1>(w[u]), w2 = mx4_pair_f16<2>(w[u]), w3 = mx4_pair_f16<3>(w[u]);
    p = __builtin_amdgcn_fdot2(x0, w0, p, false); p = __builtin_amdgcn_fdot2(x1, w1, p, false);
    p = __builtin_amdgcn_fdot2(x2, w2, p, false); p = __builtin_amdgcn_fdot2(x3, w3, p, false);
    q = __builtin_amdgcn_fdot2(w0, w0, q, false); q = __builtin_amdgcn_fdot2(w1, w1, q, false);
    q = __builtin_amdgcn_fdot2(w2, w2, q, false); q = __builtin_amdgcn_fdot2(w3, w3, q, false);
  }
  xw = p;
  ww = q;
}

// 2^e for |e| <= 1000.
__device__ __forceinline__ double mx4_pow2(int e) { return __hiloint2double((e + 1023) << 20, 0); }

}  // namespace som
