// Best-matching units of microscaled 4-bit rows among microscaled 4-bit nodes (mx4.hpp; som_bmus_mx4): the node of the
// smallest |x - w|^2 = |x|^2 - 2 (x.w - |w|^2 / 2), the lowest of equally near ones.
//
// Direct search: every score x.w - |w|^2 / 2 in fp64.  The dot product of two blocks is exact in fp32 (mx4.hpp), the sum over the
// blocks is taken in fp64, exact while the exponents of a row's products lie within 2^40 of each other.  Groups of lanes share a node's blocks.
#include "mx4.hpp"

namespace som {

// Is (s, i) to replace (best, arg)?  A larger score, or an equal one at a lower index; never a NaN.
__device__ __forceinline__ bool mx4_better(double s, int i, double best, int arg) {
  return s > best || (s == best && i < arg);
}

struct Mx4Best {
  double score;
  int node, pad;
};

__device__ __forceinline__ Mx4Best mx4_best_of_block(double best, int arg) {
  __shared__ double s_best[4];
  __shared__ int s_arg[4];
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    const double s = __shfl_xor(best, o);
    const int i = __shfl_xor(arg, o);
    if (mx4_better(s, i, best, arg)) { best = s; arg = i; }
  }
  const int wave = threadIdx.x >> 6;
  if ((threadIdx.x & 63) == 0) { s_best[wave] = best; s_arg[wave] = arg; }
  __syncthreads();
  Mx4Best r = {s_best[0], s_arg[0], 0};
#pragma unroll
  for (int w = 1; w < 4; ++w)
    if (mx4_better(s_best[w], s_arg[w], r.score, r.node)) { r.score = s_best[w]; r.node = s_arg[w]; }
  return r;
}

// blockIdx.y: the instance; blockIdx.x: a share of the nodes.  2^log_lanes lanes take a node.
__global__ __launch_bounds__(256) void k_mx4_direct(Mx4Rows x, Mx4Rows w, int blocks, int log_lanes, Mx4Best *__restrict__ rec,
                                                    int32_t *__restrict__ bmus) {
  const int lanes = 1 << log_lanes, sub = threadIdx.x & (lanes - 1), per = 256 >> log_lanes;
  const int64_t row = blockIdx.y;
  const uint8_t *xs = x.scales + row * blocks;
  const i32x4 *xc = reinterpret_cast<const i32x4 *>(x.codes + row * blocks * 16);
  double best = -INFINITY;
  int arg = 0x7fffffff;
  for (int64_t n0 = (int64_t)blockIdx.x * per; n0 < w.n; n0 += (int64_t)gridDim.x * per) {
    const int64_t node = n0 + (threadIdx.x >> log_lanes);
    double s = 0.0;
    if (node < w.n) {
      const uint8_t *ws = w.scales + node * blocks;
      const i32x4 *wc = reinterpret_cast<const i32x4 *>(w.codes + node * blocks * 16);
      for (int b = sub; b < blocks; b += lanes) {
        const int ex = xs[b], ew = ws[b];
        float xw, ww;
        mx4_block_dots(xc[b], wc[b], xw, ww);
        s += (double)xw * mx4_pow2(ex + ew - 254) - (double)ww * mx4_pow2(2 * ew - 255);
        if (ex == 255 || ew == 255) s = NAN;
      }
    }
    for (int o = 1; o < lanes; o <<= 1) s += __shfl_xor(s, o);
    if (sub == 0 && node < w.n && mx4_better(s, (int)node, best, arg)) { best = s; arg = (int)node; }
  }
  const Mx4Best r = mx4_best_of_block(best, arg);
  if (threadIdx.x == 0) {
    if (gridDim.x == 1) bmus[row] = r.node == 0x7fffffff ? 0 : r.node;
    else rec[row * gridDim.x + blockIdx.x] = r;
  }
}

__global__ __launch_bounds__(256) void k_mx4_direct_join(const Mx4Best *__restrict__ rec, int shares, int32_t *__restrict__ bmus) {
  const Mx4Best *mine = rec + (int64_t)blockIdx.x * shares;
  double best = -INFINITY;
  int arg = 0x7fffffff;
  for (int t = threadIdx.x; t < shares; t += 256)
    if (mx4_better(mine[t].score, mine[t].node, best, arg)) { best = mine[t].score; arg = mine[t].node; }
  const Mx4Best r = mx4_best_of_block(best, arg);
  if (threadIdx.x == 0) bmus[blockIdx.x] = r.node == 0x7fffffff ? 0 : r.node;
}

// Shares of the nodes per instance: enough workgroups to fill the chip, a pass over their lanes at least.
static int direct_shares(const som_ctx *c, int64_t n, int lanes) {
  const int64_t all = ((int64_t)c->k * lanes + 255) / 256, want = (8 * (int64_t)c->n_cu + n - 1) / n;
  return (int)(want < all ? want : all);
}

static int direct_lanes_log(int blocks) {
  int l = 0;
  while (l < 3 && (2 << l) <= blocks) ++l;
  return l;
}

size_t mx4_search_bytes(const som_ctx *c, int64_t n) {
  const int shares = direct_shares(c, n, 1 << direct_lanes_log(mx4_blocks(c->dim)));
  return shares > 1 ? (size_t)n * shares * sizeof(Mx4Best) : 0;
}

hipError_t launch_bmu_mx4(som_ctx *c, Mx4Rows x, Mx4Rows w, void *scratch, int32_t *bmus) {
  const int blocks = mx4_blocks(c->dim), log_lanes = direct_lanes_log(blocks), shares = direct_shares(c, x.n, 1 << log_lanes);
  Mx4Best *rec = static_cast<Mx4Best *>(scratch);
  for (int64_t r0 = 0; r0 < x.n; r0 += 65535) {
    const Mx4Rows part = {x.codes + r0 * blocks * 16, x.scales + r0 * blocks, x.n - r0 < 65535 ? x.n - r0 : 65535};
    hipLaunchKernelGGL(k_mx4_direct, dim3(shares, (unsigned)part.n), dim3(256), 0, c->stream, part, w, blocks, log_lanes, rec, bmus + r0);
  }
  if (shares > 1) hipLaunchKernelGGL(k_mx4_direct_join, dim3((unsigned)x.n), dim3(256), 0, c->stream, rec, shares, bmus);
  return hipGetLastError();
}

}  // namespace som
