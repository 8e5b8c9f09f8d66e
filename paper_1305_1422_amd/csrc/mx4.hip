// Rows into microscaled 4-bit form and back (mx4.hpp; som_mx4_quantize, som_mx4_dequantize).
//
// Four lanes take a block of 32 features, eight each: 32 bytes of fp32 or 16 of a 16-bit type in, one word of codes out.
// The block's power of two comes from the largest magnitude's exponent field e (an integer maximum, which also
// finds infinities and NaN): byte max(e - 2, 0), so that the largest element lies in [4, 8) and what is above 6 is cut
// to 6.  v_cvt_scalef32_pk_fp4_f32 divides by the power of two, rounds to nearest with ties to even and saturates (checked
// against those rules over the whole range of scales, subnormal values included).
//
// Bound by HBM: 4.53 bytes per feature from fp32, 2.53 from 16-bit types, either way.
#include "mx4.hpp"

namespace som {

template <typename T> struct Mx4Type;
template <> struct Mx4Type<float> {
  static __device__ __forceinline__ float up(float v) { return v; }
  static __device__ __forceinline__ float down(float v) { return v; }
};
template <> struct Mx4Type<_Float16> {
  static __device__ __forceinline__ float up(_Float16 v) { return (float)v; }
  static __device__ __forceinline__ _Float16 down(float v) { return (_Float16)v; }
};
template <> struct Mx4Type<__bf16> {
  static __device__ __forceinline__ float up(__bf16 v) { return (float)v; }
  static __device__ __forceinline__ __bf16 down(float v) { return (__bf16)v; }
};

// Row of block `block` (blocks of all rows counted through): block / blocks by one multiplication, exact for block < 2^31
// with m = ceil(2^(31 + sh) / blocks), sh = ceil(log2 blocks).
struct Mx4Div {
  unsigned m, sh;
};
static Mx4Div mx4_div(unsigned blocks) {
  Mx4Div d;
  d.sh = 0;
  while ((1ull << d.sh) < blocks) ++d.sh;
  d.m = (unsigned)(((1ull << (31 + d.sh)) + blocks - 1) / blocks);
  return d;
}
__device__ __forceinline__ unsigned mx4_row(unsigned block, Mx4Div d) {
  return (unsigned)(((unsigned long long)block * d.m) >> (31 + d.sh));
}

// Eight consecutive elements at p; kVec: 16-byte loads, all of them inside the row.  Otherwise `left` of them are.
template <typename T, bool kVec>
__device__ __forceinline__ void mx4_load8(const T *p, int left, float v[8]) {
  if (kVec) {
    T t[8];
    const i32x4 *q = reinterpret_cast<const i32x4 *>(p);
    *reinterpret_cast<i32x4 *>(t) = q[0];
    if (sizeof(T) == 4) *reinterpret_cast<i32x4 *>(t + 4) = q[1];
#pragma unroll
    for (int u = 0; u < 8; ++u) v[u] = Mx4Type<T>::up(t[u]);
  } else {
#pragma unroll
    for (int u = 0; u < 8; ++u) v[u] = u < left ? Mx4Type<T>::up(p[u]) : 0.f;
  }
}

// kVec: the groups of eight are whole (dim % 8 == 0) and aligned, or entirely past the end of the row.
template <typename T, bool kVec>
__global__ __launch_bounds__(256) void k_mx4_quantize(const T *__restrict__ rows, int64_t stride, int dim, int blocks, Mx4Div div,
                                                      unsigned items, unsigned *__restrict__ codes,
                                                      uint8_t *__restrict__ scales) {
  const unsigned item = blockIdx.x * 256u + threadIdx.x;
  if (item >= items) return;                  // (items is a multiple of four: a block's lanes stay together)
  const unsigned block = item >> 2, row = mx4_row(block, div);
  const int at = (int)(block - row * (unsigned)blocks) * 32 + (int)(item & 3u) * 8;
  float v[8];
  if (!kVec || at < dim) mx4_load8<T, kVec>(rows + (int64_t)row * stride + at, dim - at, v);
  else
#pragma unroll
    for (int u = 0; u < 8; ++u) v[u] = 0.f;
  int top = 0;
#pragma unroll
  for (int u = 0; u < 8; ++u) top = max(top, __float_as_int(v[u]) & 0x7fffffff);
  top = max(top, __builtin_amdgcn_mov_dpp(top, 0xB1, 0xF, 0xF, true));      // lane ^ 1
  top = max(top, __builtin_amdgcn_mov_dpp(top, 0x4E, 0xF, 0xF, true));      // lane ^ 2
  const int e = top >> 23;
  const unsigned s = e == 255 ? 255u : (unsigned)max(e - 2, 0);
  const float scale = mx4_scale(s);
  unsigned word = 0;
  if (e != 255) {
    word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, v[0], v[1], scale, 0);
    word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, v[2], v[3], scale, 1);
    word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, v[4], v[5], scale, 2);
    word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, v[6], v[7], scale, 3);
  }
  codes[item] = word;
  if ((item & 3u) == 0) scales[block] = (uint8_t)s;
}

template <typename T, bool kVec>
__global__ __launch_bounds__(256) void k_mx4_dequantize(const unsigned *__restrict__ codes, const uint8_t *__restrict__ scales,
                                                        int dim, int blocks, Mx4Div div, unsigned items, T *__restrict__ rows,
                                                        int64_t stride) {
  const unsigned item = blockIdx.x * 256u + threadIdx.x;
  if (item >= items) return;
  const unsigned block = item >> 2, row = mx4_row(block, div);
  const int at = (int)(block - row * (unsigned)blocks) * 32 + (int)(item & 3u) * 8;
  if (at >= dim) return;
  const unsigned word = codes[item];
  const float scale = mx4_scale(scales[block]);
  const mx_f32x2 p0 = mx4_pair<0>(word, scale), p1 = mx4_pair<1>(word, scale), p2 = mx4_pair<2>(word, scale), p3 = mx4_pair<3>(word, scale);
  T t[8] = {Mx4Type<T>::down(p0[0]), Mx4Type<T>::down(p0[1]), Mx4Type<T>::down(p1[0]), Mx4Type<T>::down(p1[1]),
            Mx4Type<T>::down(p2[0]), Mx4Type<T>::down(p2[1]), Mx4Type<T>::down(p3[0]), Mx4Type<T>::down(p3[1])};
  T *dst = rows + (int64_t)row * stride + at;
  if (kVec) {
    i32x4 *q = reinterpret_cast<i32x4 *>(dst);
    q[0] = *reinterpret_cast<const i32x4 *>(t);
    if (sizeof(T) == 4) q[1] = *reinterpret_cast<const i32x4 *>(t + 4);
  } else {
#pragma unroll
    for (int u = 0; u < 8; ++u)
      if (at + u < dim) dst[u] = t[u];
  }
}

// Rows of a launch: their groups of eight are counted in 32 bits, blocks in 31.
static int64_t mx4_rows_at_once(int blocks) { return (1ll << 28) / blocks > 0 ? (1ll << 28) / blocks : 1; }

template <typename T>
static hipError_t quantize_rows(hipStream_t stream, const T *rows, int64_t n, int64_t stride, int dim, uint8_t *codes, uint8_t *scales) {
  const int blocks = mx4_blocks(dim);
  const int64_t step = mx4_rows_at_once(blocks);
  const bool vec = dim % 8 == 0 && (uintptr_t)rows % 16 == 0 && (stride * (int64_t)sizeof(T)) % 16 == 0;
  for (int64_t r0 = 0; r0 < n; r0 += step) {
    const int64_t m = n - r0 < step ? n - r0 : step;
    const unsigned items = (unsigned)(4 * m * blocks), grid = (items + 255) / 256;
    const T *src = rows + r0 * stride;
    unsigned *dst = reinterpret_cast<unsigned *>(codes + r0 * blocks * 16);
    if (vec) hipLaunchKernelGGL((k_mx4_quantize<T, true>), dim3(grid), dim3(256), 0, stream, src, stride, dim, blocks, mx4_div(blocks), items, dst, scales + r0 * blocks);
    else hipLaunchKernelGGL((k_mx4_quantize<T, false>), dim3(grid), dim3(256), 0, stream, src, stride, dim, blocks, mx4_div(blocks), items, dst, scales + r0 * blocks);
  }
  return hipGetLastError();
}

template <typename T>
static hipError_t dequantize_rows(hipStream_t stream, Mx4Rows x, int dim, T *rows, int64_t stride) {
  const int blocks = mx4_blocks(dim);
  const int64_t step = mx4_rows_at_once(blocks);
  const bool vec = dim % 8 == 0 && (uintptr_t)rows % 16 == 0 && (stride * (int64_t)sizeof(T)) % 16 == 0;
  for (int64_t r0 = 0; r0 < x.n; r0 += step) {
    const int64_t m = x.n - r0 < step ? x.n - r0 : step;
    const unsigned items = (unsigned)(4 * m * blocks), grid = (items + 255) / 256;
    const unsigned *src = reinterpret_cast<const unsigned *>(x.codes + r0 * blocks * 16);
    T *dst = rows + r0 * stride;
    if (vec) hipLaunchKernelGGL((k_mx4_dequantize<T, true>), dim3(grid), dim3(256), 0, stream, src, x.scales + r0 * blocks, dim, blocks, mx4_div(blocks), items, dst, stride);
    else hipLaunchKernelGGL((k_mx4_dequantize<T, false>), dim3(grid), dim3(256), 0, stream, src, x.scales + r0 * blocks, dim, blocks, mx4_div(blocks), items, dst, stride);
  }
  return hipGetLastError();
}

hipError_t launch_mx4_quantize(hipStream_t stream, const void *rows, int type, int64_t n, int64_t stride, int dim, uint8_t *codes,
                               uint8_t *scales) {
  if (type == SOM_FP32) return quantize_rows(stream, static_cast<const float *>(rows), n, stride, dim, codes, scales);
  if (type == SOM_FP16) return quantize_rows(stream, static_cast<const _Float16 *>(rows), n, stride, dim, codes, scales);
  return quantize_rows(stream, static_cast<const __bf16 *>(rows), n, stride, dim, codes, scales);
}

hipError_t launch_mx4_dequantize(hipStream_t stream, Mx4Rows x, int dim, void *rows, int type, int64_t stride) {
  if (type == SOM_FP32) return dequantize_rows(stream, x, dim, static_cast<float *>(rows), stride);
  if (type == SOM_FP16) return dequantize_rows(stream, x, dim, static_cast<_Float16 *>(rows), stride);
  return dequantize_rows(stream, x, dim, static_cast<__bf16 *>(rows), stride);
}

}  // namespace som
