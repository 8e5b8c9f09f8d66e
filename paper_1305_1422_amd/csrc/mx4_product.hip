// Dot products of all pairs of two sets of microscaled 4-bit rows (mx4.hpp; som_mx4_product):
// out[i][j] = sum_c a_ic b_jc, fp32 accumulation on the scaled matrix cores, rounded once to the type of the output.
//
// A wavefront takes 16 rows of a and 64 of b straight from global memory.  The rows of b are the instruction's first operand, so that a lane
// ends up with four consecutive products of one row of the output.
#include "mx4.hpp"

namespace som {

template <typename T> __device__ __forceinline__ T mx4_out(float v) { return (T)v; }

template <typename T>
__global__ __launch_bounds__(256) void k_mx4_product(Mx4Rows a, Mx4Rows b, int blocks, T *__restrict__ out, int64_t stride) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l16 = lane & 15, q = lane >> 4;
  const int64_t i = ((int64_t)blockIdx.y * 4 + wave) * 16 + l16, j0 = (int64_t)blockIdx.x * 64;
  if (i - l16 >= a.n) return;
  const int64_t ia = i < a.n ? i : a.n - 1;
  int64_t jb[4];
#pragma unroll
  for (int t = 0; t < 4; ++t) jb[t] = j0 + 16 * t + l16 < b.n ? j0 + 16 * t + l16 : b.n - 1;
  mx_f32x4 acc[4] = {};
  for (int k0 = 0; k0 < blocks; k0 += 4) {
    const int k = k0 + q;
    const bool in = k < blocks;
    const i32x4 none = {0, 0, 0, 0};
    const i32x4 x = in ? *reinterpret_cast<const i32x4 *>(a.codes + (ia * blocks + k) * 16) : none;
    const int sx = in ? a.scales[ia * blocks + k] : 0;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const i32x4 y = in ? *reinterpret_cast<const i32x4 *>(b.codes + (jb[t] * blocks + k) * 16) : none;
      const int sy = in ? b.scales[jb[t] * blocks + k] : 0;
      acc[t] = mx4_mfma<0, 0>(y, x, acc[t], sy, sx);
    }
  }
  if (i >= a.n) return;
#pragma unroll
  for (int t = 0; t < 4; ++t)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int64_t j = j0 + 16 * t + 4 * q + r;
      if (j < b.n) out[i * stride + j] = mx4_out<T>(acc[t][r]);
    }
}

template <typename T>
static hipError_t product(som_ctx *c, Mx4Rows a, Mx4Rows b, T *out, int64_t stride) {
  const int blocks = mx4_blocks(c->dim);
  const int64_t step = 65535ll * 64;             // rows of a a launch can take in its second grid direction
  for (int64_t i0 = 0; i0 < a.n; i0 += step) {
    const Mx4Rows part = {a.codes + i0 * blocks * 16, a.scales + i0 * blocks, a.n - i0 < step ? a.n - i0 : step};
    const dim3 grid((unsigned)((b.n + 63) / 64), (unsigned)((part.n + 63) / 64));
    hipLaunchKernelGGL(k_mx4_product<T>, grid, dim3(256), 0, c->stream, part, b, blocks, out + i0 * stride, stride);
  }
  return hipGetLastError();
}

hipError_t launch_mx4_product(som_ctx *c, Mx4Rows a, Mx4Rows b, void *out, int type, int64_t stride) {
  if (type == SOM_FP32) return product(c, a, b, static_cast<float *>(out), stride);
  if (type == SOM_FP16) return product(c, a, b, static_cast<_Float16 *>(out), stride);
  return product(c, a, b, static_cast<__bf16 *>(out), stride);
}

}  // namespace som
