// Best-matching units of microscaled 4-bit rows among microscaled 4-bit nodes (mx4.hpp; som_bmus_mx4): the node of the
// smallest |x - w|^2 = |x|^2 - 2 (x.w - |w|^2 / 2), the lowest of equally near ones.
//
// Small searches are direct: every score x.w - |w|^2 / 2 in fp64.  The dot product of two blocks is exact in fp32 (mx4.hpp), the sum over the
// blocks is taken in fp64.  With M and m the largest and smallest product of scales among x.w and |w|^2, all terms are multiples of m / 8 and their
// magnitudes add up to B (1152 + 576) M at most: every sum is exact while B 13824 M <= 2^53 m, so for M / m up to 2^39 / B.  Groups of lanes
// share a node's blocks.
//
// Larger ones go through the matrix cores, whose fp32 sums are off by a bound that is known (margin below):
//   k_mx4_nodes    -|w|^2 / 2 of every node (what the accumulators start from) and the nodes' scales, packed;
//   k_mx4_search   tiles of scores (mx4_tiles.hpp), never stored: per instance and group of 16 consecutive nodes - what a lane holds of a
//                  tile - their maximum, of those the largest with its group and the largest of the other groups;
//   k_mx4_resolve  where no other group comes within the margin: the 16 scores of the group again, and if one of them alone is within the
//                  margin of the largest, that is the node.  A wavefront has 16 instances, and an instruction multiplies the 16 nodes of a
//                  group with all of them; columns of instances whose group it is not are of no use;
//   k_mx4_search   again for the instances of which another group did: it lists the groups within the margin;
//   k_mx4_exact    what is left, in fp64: the listed groups of these, the one group of the others; all nodes, shared out as in a direct
//                  search, where there are more than kMx4List groups, or where fp32 could overflow.
#include "mx4_tiles.hpp"

namespace som {

// Is (s, i) to replace (best, arg)?  A larger score, or an equal one at a lower index; never a NaN.
__device__ __forceinline__ bool mx4_better(double s, int i, double best, int arg) {
  return s > best || (s == best && i < arg);
}

struct Mx4Best {
  double score;
  int node;
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
  __syncthreads();                             // (it may have been called before)
  if ((threadIdx.x & 63) == 0) { s_best[wave] = best; s_arg[wave] = arg; }
  __syncthreads();
  Mx4Best r = {s_best[0], s_arg[0]};
#pragma unroll
  for (int w = 1; w < 4; ++w)
    if (mx4_better(s_best[w], s_arg[w], r.score, r.node)) { r.score = s_best[w]; r.node = s_arg[w]; }
  return r;
}

// What a workgroup does with one of `shares` shares of the nodes for an instance; 2^log_lanes lanes take a node.  The share that finishes last
// joins them: ticket `at` (zero between calls) counts them, records at * shares .. and tickets are read and written past the XCDs' own caches.
struct Mx4Joined {
  double *score;
  int *node, *tickets;
};
__device__ __forceinline__ void mx4_scan(const Mx4Rows &x, const Mx4Rows &w, int blocks, int log_lanes, int64_t row, int share, int shares, int at,
                                         const Mx4Joined &join, int32_t *__restrict__ bmus) {
  __shared__ int s_last;
  const int lanes = 1 << log_lanes, sub = threadIdx.x & (lanes - 1), per = 256 >> log_lanes;
  const uint8_t *xs = x.scales + row * blocks;
  const i32x4 *xc = reinterpret_cast<const i32x4 *>(x.codes + row * blocks * 16);
  double best = -INFINITY;
  int arg = 0x7fffffff;
  for (int64_t n0 = (int64_t)share * per; n0 < w.n; n0 += (int64_t)shares * per) {
    const int64_t node = n0 + (threadIdx.x >> log_lanes);
    double s = 0.0;
    if (node < w.n) {
      const uint8_t *ws = w.scales + node * blocks;
      const i32x4 *wc = reinterpret_cast<const i32x4 *>(w.codes + node * blocks * 16);
#pragma unroll 4
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
  Mx4Best r = mx4_best_of_block(best, arg);
  if (shares > 1) {
    if (threadIdx.x == 0) {
      __hip_atomic_store(&join.score[at * shares + share], r.score, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      __hip_atomic_store(&join.node[at * shares + share], r.node, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      // (the stores have reached memory before the ticket does; a release at this scope would write back the whole L2, 34 us for 2,000 workgroups
      // instead of 6)
      asm volatile("s_waitcnt vmcnt(0)" : : : "memory");
      s_last = __hip_atomic_fetch_add(&join.tickets[at], 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == shares - 1;
    }
    __syncthreads();
    if (!s_last) return;
    best = -INFINITY;
    arg = 0x7fffffff;
    for (int t = threadIdx.x; t < shares; t += 256) {
      const double score = __hip_atomic_load(&join.score[at * shares + t], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      const int node = __hip_atomic_load(&join.node[at * shares + t], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      if (mx4_better(score, node, best, arg)) { best = score; arg = node; }
    }
    r = mx4_best_of_block(best, arg);
    if (threadIdx.x == 0) __hip_atomic_store(&join.tickets[at], 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  if (threadIdx.x == 0) bmus[row] = r.node == 0x7fffffff ? 0 : r.node;
}

// blockIdx.y: the instance; blockIdx.x: a share of the nodes.
__global__ __launch_bounds__(256) void k_mx4_direct(Mx4Rows x, Mx4Rows w, int blocks, int log_lanes, Mx4Joined join, int32_t *__restrict__ bmus) {
  mx4_scan(x, w, blocks, log_lanes, blockIdx.y, blockIdx.x, gridDim.x, blockIdx.y, join, bmus);
}

// ---------------------------------------------------------------- direct search
// Shares of the nodes per instance: enough workgroups to fill the chip, a pass over their lanes at least; with more than one there are at most
// kMx4Tickets instances.
static int direct_shares(const som_ctx *c, int64_t n, int lanes) {
  if (n > kMx4Tickets) return 1;
  if (n >= 2 * c->n_cu) return 1;
  const int64_t all = ((int64_t)c->k * lanes + 255) / 256, want = (8 * (int64_t)c->n_cu + n - 1) / n;
  return (int)(want < all ? want : all);
}

static int direct_lanes_log(int blocks) {
  int l = 0;
  while (l < 3 && (2 << l) <= blocks) ++l;
  return l;
}

static hipError_t search_direct(som_ctx *c, Mx4Rows x, Mx4Rows w, void *scratch, int *tickets, int32_t *bmus) {
  const int blocks = mx4_blocks(c->dim), log_lanes = direct_lanes_log(blocks), shares = direct_shares(c, x.n, 1 << log_lanes);
  double *score = static_cast<double *>(scratch);
  int *node = reinterpret_cast<int *>(score + x.n * shares);
  for (int64_t r0 = 0; r0 < x.n; r0 += 65535) {          // (one launch where there are several shares)
    const Mx4Rows part = {x.codes + r0 * blocks * 16, x.scales + r0 * blocks, x.n - r0 < 65535 ? x.n - r0 : 65535};
    hipLaunchKernelGGL(k_mx4_direct, dim3(shares, (unsigned)part.n), dim3(256), 0, c->stream, part, w, blocks, log_lanes,
                       Mx4Joined{score, node, tickets}, bmus + r0);
  }
  return hipGetLastError();
}

// ---------------------------------------------------------------- search on the matrix cores
typedef Mx4Tile<8, 4, 2, 4, true> Mx4Sweep;      // 256 nodes x 256 instances

constexpr int kMx4List = 32;            // groups an instance's list holds (maps of a wide radius came to 23)
constexpr int kMx4ScanBlocks = 2048;    // workgroups of the exact pass at most
constexpr int kMx4NodeBlocks = 1024;     // workgroups of the node pass at most
constexpr float kMx4Lowest = -3.0e38f;  // below every score that counts

struct Mx4Counts {
  int listed, single;      // instances to list groups of (slots from the front), with one group (slots from the back)
  int whole;               // instances to be compared with all nodes (whole_list)
};

// Largest and second largest of the groups' maxima.
struct Mx4Record {
  float best, second;
  int group;
};

// The stream of nodes, 64 at a time (a unit): per step and group of 16 nodes their fragment (lane l: block l / 16 of node l % 16; 1 KB), then
// per step the packed scales (mx4_tiles.hpp), then what the accumulators start from in the order of the nodes, rounded up to whole KB.
__host__ __device__ constexpr int64_t mx4_stream_bytes(int64_t steps) { return steps * 4096 + ((steps + 1) * 256 + 1023) / 1024 * 1024; }
// By group of 16 nodes besides, for k_mx4_resolve: per step the scales of its fragment, then its 16 starting values (in the stream they share
// their lines with those of other groups).
__host__ __device__ constexpr int64_t mx4_group_bytes(int64_t steps) { return (steps + 1) * 64; }

// A workgroup takes 64 nodes at a time.  parts[blockIdx.x]: the largest |w|^2 it saw (fp64, rounded up to fp32; infinity if it overflows).
// packed, init: the scales and starting values by themselves for k_mx4_search, or null.
__global__ __launch_bounds__(256) void k_mx4_nodes(Mx4Rows w, int blocks, int cols, int64_t padded, float *__restrict__ init, char *__restrict__ stream,
                                                   char *__restrict__ by_group, int *__restrict__ packed, float *__restrict__ parts, Mx4Counts *__restrict__ counts) {
  __shared__ double s_norm[4][64];
  __shared__ unsigned s_same[4][16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = lane & 15, q = lane >> 4;
  const int64_t steps = (blocks - 1) / 4 + 1;
  if (blockIdx.x == 0 && threadIdx.x == 0) *counts = Mx4Counts{0, 0, 0};
  float most = 0.f;
  for (int64_t g = blockIdx.x; g < padded / 64; g += gridDim.x) {
    char *mine = stream + g * mx4_stream_bytes(steps);
    double norm[4] = {0, 0, 0, 0};
    unsigned same = 255;                       // bit t: like the node before it, so far; bit 4 + t: like the one a map row before it
    for (int64_t s = wave; s < steps; s += 4) {
      const int64_t block = 4 * s + q;
      unsigned v = 0;
      i32x4 x[4], left[4], up[4];
      int ex[4], eleft[4], eup[4];
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const int64_t node = 64 * g + mx4_dealt(t, i);
        const int64_t b = (node < w.n ? node : w.n - 1) * blocks + (block < blocks ? block : blocks - 1);
        // (a node without the other one is compared with itself, and told apart below)
        const int64_t bl = node >= 1 && node < w.n ? b - blocks : b, bu = node >= cols && node < w.n ? b - (int64_t)cols * blocks : b;
        x[t] = *reinterpret_cast<const i32x4 *>(w.codes + b * 16);
        left[t] = *reinterpret_cast<const i32x4 *>(w.codes + bl * 16);
        up[t] = *reinterpret_cast<const i32x4 *>(w.codes + bu * 16);
        ex[t] = w.scales[b];
        eleft[t] = w.scales[bl];
        eup[t] = w.scales[bu];
      }
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const i32x4 dl = x[t] ^ left[t], du = x[t] ^ up[t];
        v |= (unsigned)ex[t] << (8 * t);
        if ((dl[0] | dl[1] | dl[2] | dl[3] | (ex[t] ^ eleft[t])) != 0) same &= ~(1u << t);
        if ((du[0] | du[1] | du[2] | du[3] | (ex[t] ^ eup[t])) != 0) same &= ~(16u << t);
      }
#pragma unroll
      for (int t = 0; t < 4; ++t)
        if (block >= blocks || 64 * g + mx4_dealt(t, i) >= w.n) {
          x[t] = i32x4{0, 0, 0, 0};
          v &= ~(255u << (8 * t));
        }
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const int e = (v >> (8 * t)) & 255;
        float xx, ww;
        mx4_block_dots(x[t], x[t], xx, ww);
        norm[t] += e == 255 ? (double)NAN : (double)ww * mx4_pow2(2 * e - 254);
        *reinterpret_cast<i32x4 *>(mine + s * 4096 + (i >> 2) * 1024 + (16 * q + 4 * t + (i & 3)) * 16) = x[t];
        by_group[(4 * g + (i >> 2)) * mx4_group_bytes(steps) + s * 64 + 16 * q + 4 * t + (i & 3)] = (char)e;
      }
      *reinterpret_cast<unsigned *>(mine + steps * 4096 + s * 256 + lane * 4) = v;
      if (packed && 64 * g < w.n) packed[(g * steps + s) * 64 + lane] = (int)v;
    }
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      norm[t] += __shfl_xor(norm[t], 16);
      norm[t] += __shfl_xor(norm[t], 32);
      if (q == t) s_norm[wave][mx4_dealt(t, i)] = norm[t];
    }
    same &= __shfl_xor(same, 16);
    same &= __shfl_xor(same, 32);
    if (q == 0) s_same[wave][i] = same;
    __syncthreads();
    if (threadIdx.x < 64) {
      const double n2 = ((s_norm[0][threadIdx.x] + s_norm[1][threadIdx.x]) + s_norm[2][threadIdx.x]) + s_norm[3][threadIdx.x];
      const int64_t node = 64 * g + threadIdx.x;
      // A node with a NaN, and what is past the last one, can never win; nor can one that is like a node before it, which takes the ties: while the
      // radius is wide, whole regions of the map have the same 4-bit rows, and the lists of equally near groups would overflow.
      const int at = threadIdx.x / 16 * 4 + threadIdx.x % 4, t = threadIdx.x % 16 / 4;
      const unsigned like = (s_same[0][at] & s_same[1][at] & s_same[2][at] & s_same[3][at]) >> t;
      const bool usable = node < w.n && n2 == n2 && !((like & 1) && node >= 1) && !((like & 16) && node >= cols);
      const float from = usable ? (float)(-0.5 * n2) : -INFINITY;
      if (init) init[node] = from;
      *reinterpret_cast<float *>(by_group + node / 16 * mx4_group_bytes(steps) + steps * 64 + node % 16 * 4) = from;
      *reinterpret_cast<float *>(mine + steps * 4096 + steps * 256 + threadIdx.x * 4) = from;
      if (usable) most = fmaxf(most, __double2float_ru(n2));
    }
    __syncthreads();
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor(most, o));
  if (threadIdx.x == 0) parts[blockIdx.x] = most;
}

// ---------------------------------------------------------------- rows of up to 8 steps (1,024 features)
// The instances stay in registers, the nodes stream through LDS.  A wavefront has 16 kF instances; for a step of 64 nodes (a piece) it
// reads four fragments for 4 kF instructions of 16 cycles.  The results of four instructions are a lane's 16 scores of one
// instance: eight v_max3, and four operations for the running maximum, its place and the runner-up - in the issue slots between the
// products of the next 64 nodes (kT = 1: of the next instances; there the 12 operations to four instructions take as many slots as there are).
// The compiler keeps reads, products and maxima apart unless the order is fixed, as it is here.  Two stages in LDS of kUnits times 64 nodes: a
// piece is read into registers while the one before it is multiplied, so when the last of a stage begins the stage is free and gets the
// loads of the one after the next.
template <int kT, int kF, int kUnits, int kWavesPerSimd>
struct Mx4SweepShape {
  static constexpr int F = kF, units = kUnits, rows = 64 * kF, waves = kWavesPerSimd;
  static constexpr int unit = (int)mx4_stream_bytes(kT), stage = kUnits * unit, rest = unit / 1024 - 4 * kT, lds = 2 * stage;
};
// F: as many as two wavefronts a SIMD leave registers for (one fewer with the lists to write); from 7 steps on a single wavefront with twice
// as many (100,000 x 10,000, whole search, us, two wavefronts / one: 384 features 201 / 232, 512 251 / 267, 640 302 / 315, 768 360 / 384,
// 900 485 / 473, 1,000 504 / 498).
template <int kT, bool kCollect> struct Mx4ShapeOf { typedef Mx4SweepShape<kT, kCollect ? 3 : 4, 1, 2> type; };
template <bool kCollect> struct Mx4ShapeOf<1, kCollect> { typedef Mx4SweepShape<1, 8, 4, 2> type; };
template <bool kCollect> struct Mx4ShapeOf<2, kCollect> { typedef Mx4SweepShape<2, kCollect ? 5 : 6, 2, 2> type; };
template <bool kCollect> struct Mx4ShapeOf<3, kCollect> { typedef Mx4SweepShape<3, kCollect ? 4 : 5, 2, 2> type; };
template <bool kCollect> struct Mx4ShapeOf<6, kCollect> { typedef Mx4SweepShape<6, kCollect ? 2 : 4, 1, 2> type; };
template <bool kCollect> struct Mx4ShapeOf<7, kCollect> { typedef Mx4SweepShape<7, kCollect ? 4 : 6, 1, 1> type; };
template <bool kCollect> struct Mx4ShapeOf<8, kCollect> { typedef Mx4SweepShape<8, kCollect ? 4 : 6, 1, 1> type; };
constexpr int kMx4SweepSteps = 8;

// The work of a pass, (block of instances, stage of nodes) pairs in that order, is cut into one piece of `per` stages for every workgroup, so
// that all of them have the same to do whatever the sizes; a piece may end one block of instances and begin another.
struct Mx4Cut {
  int64_t stages, per;     // of a block of instances, of a workgroup
  int rows;                // instances of a block
};
// Records of an instance: those of the workgroups first .. last that have stages of its block.
__host__ __device__ inline int64_t mx4_first_piece(const Mx4Cut &c, int64_t block) { return block * c.stages / c.per; }
__host__ __device__ inline int64_t mx4_last_piece(const Mx4Cut &c, int64_t block) { return ((block + 1) * c.stages - 1) / c.per; }

// Nothing moves across: neither the loads (the assembly) nor anything else (the barrier of the scheduler).
__device__ __forceinline__ void mx4_in_order() {
  asm volatile("" : : : "memory");
  __builtin_amdgcn_sched_barrier(0);
}

// kCollect as in k_mx4_search.
template <int kT, bool kCollect>
__global__ __launch_bounds__(256, (Mx4ShapeOf<kT, kCollect>::type::waves)) void k_mx4_sweep(Mx4Rows x, int blocks, const char *__restrict__ stream, Mx4Cut cut,
                                                      Mx4Record *__restrict__ records, Mx4Counts *__restrict__ counts,
                                                      const int *__restrict__ list, const float *__restrict__ threshold,
                                                      int *__restrict__ found, int *__restrict__ groups, int *__restrict__ whole) {
  typedef typename Mx4ShapeOf<kT, kCollect>::type Shape;
  constexpr int kF = Shape::F, kUnits = Shape::units;
  constexpr bool kByF = kT == 1;
  __shared__ __attribute__((aligned(16))) char smem[Shape::lds];
  const unsigned lds = (unsigned)(size_t)(mx4_lds_t)smem;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l16 = lane & 15, q = lane >> 4;
  const int64_t n = kCollect ? counts->listed : x.n, nb = (n + Shape::rows - 1) / Shape::rows;
  if (kCollect) {                              // how many there are is known here only
    if (n == 0) return;
    cut.per = (nb * cut.stages + gridDim.x - 1) / gridDim.x;
  }
  int64_t pos = blockIdx.x * cut.per;
  const int64_t end = pos + cut.per < nb * cut.stages ? pos + cut.per : nb * cut.stages;
  // Wavefront t fetches the fragments t that the products take (mx4_dealt: a quarter of the rows from each group of 16), so that LDS has
  // them as the reads below want them.
  const int deal = (l16 >> 2) * 1024 + q * 256 + (l16 & 3) * 16 + wave * 64;
  int64_t first = 0, last = 0;
  auto load = [&](int64_t at, int half) {      // (past the share: its last stage again, which nobody reads)
    const char *src = stream + (at < last ? at : last - 1) * Shape::stage;
    const unsigned dst = lds + half * Shape::stage;
#pragma unroll
    for (int u = 0; u < kUnits; ++u)
#pragma unroll
      for (int s = 0; s < kT; ++s)
        load16_to_lds_at(src + u * Shape::unit + s * 4096, deal, dst + u * Shape::unit + (4 * s + wave) * 1024);
#pragma unroll
    for (int u = 0; u < (kUnits * Shape::rest + 3) / 4; ++u) {
      int c = 4 * u + wave;                    // (no branch, which would tear the order below apart: the last one more than once)
      if ((kUnits * Shape::rest) % 4 != 0 && c >= kUnits * Shape::rest) c = kUnits * Shape::rest - 1;
      const int off = c / Shape::rest * Shape::unit + kT * 4096 + c % Shape::rest * 1024;
      load16_to_lds_at(src + off, lane * 16, dst + off);
    }
  };
  struct Piece {
    i32x4 w[4];
    int sw;
    mx_f32x4 from[4];
  };
  // one of the reads of a piece: the step's fragments and scales, what the accumulators start from
  auto read = [&](Piece &p, const char *unit, int s, int i) {
    if (i < 4) p.w[i] = *reinterpret_cast<const i32x4 *>(unit + (s * 4 + i) * 1024 + lane * 16);
    else if (i == 4) p.sw = *reinterpret_cast<const int *>(unit + kT * 4096 + s * 256 + lane * 4);
    else if (i < 9 && s == 0) p.from[i - 5] = *reinterpret_cast<const mx_f32x4 *>(unit + kT * 4352 + (16 * q + 4 * (i - 5)) * 4);
  };
  while (pos < end) {
    const int64_t block = pos / cut.stages, row0 = block * Shape::rows;
    first = pos - block * cut.stages;
    last = first + (end - pos) < cut.stages ? first + (end - pos) : cut.stages;
    pos += last - first;
    load(first, 0);
    load(first + 1, 1);
    i32x4 y[kF][kT];
    int sy[(kF + 3) / 4][kT];
    float best[kF], second[kF];
    int at[kF];
#pragma unroll
    for (int f = 0; f < kF; ++f) {
      const int64_t slot = row0 + 16 * (wave * kF + f) + l16;
      int64_t row = slot < n ? slot : n - 1;
      if (kCollect) row = list[row];
#pragma unroll
      for (int s = 0; s < kT; ++s) {
        // (what is past the end meets zeros of the stream)
        const int64_t b = row * blocks + (4 * s + q < blocks ? 4 * s + q : blocks - 1);
        y[f][s] = *reinterpret_cast<const i32x4 *>(x.codes + b * 16);
        const int e = x.scales[b];
        sy[f / 4][s] = f % 4 == 0 ? e : sy[f / 4][s] | e << (8 * (f % 4));
      }
      best[f] = kCollect ? (slot < n ? threshold[slot] : INFINITY) : kMx4Lowest;
      second[f] = kMx4Lowest;
      at[f] = 0;
    }
    // Scores a of instance fragment f and nodes 64 unit + 16 q .. + 15, a quarter of the work at a time.
    float m = kMx4Lowest;
    bool larger = false;
    auto maxima = [&](const mx_f32x4 (&a)[4], int f, int unit, int part) {
      if (part == 0) {
        m = fmaxf(fmaxf(kMx4Lowest, a[0][0]), a[0][1]);
        m = fmaxf(fmaxf(m, a[0][2]), a[0][3]);
        m = fmaxf(fmaxf(m, a[1][0]), a[1][1]);
      } else if (part == 1) {
        m = fmaxf(fmaxf(m, a[1][2]), a[1][3]);
        m = fmaxf(fmaxf(m, a[2][0]), a[2][1]);
        m = fmaxf(fmaxf(m, a[2][2]), a[2][3]);
      } else if (part == 2) {
        m = fmaxf(fmaxf(m, a[3][0]), a[3][1]);
        m = fmaxf(fmaxf(m, a[3][2]), a[3][3]);
        if (!kCollect) second[f] = __builtin_amdgcn_fmed3f(second[f], best[f], m);
      } else if (!kCollect) {
        larger = m > best[f];
        at[f] = larger ? unit : at[f];
        best[f] = larger ? m : best[f];
      } else if (m >= best[f]) {
        const int64_t slot = row0 + 16 * (wave * kF + f) + l16;
        const int place = atomicAdd(&found[slot], 1);
        if (place < kMx4List) groups[slot * kMx4List + place] = 4 * unit + q;
        else if (place == kMx4List) whole[atomicAdd(&counts->whole, 1)] = list[slot];
      }
    };
    // kByF: the scores of two fragments of instances, the last ones' to begin with [1]; else those of all
    constexpr int kAcc = kByF ? 2 : kF;
    static_assert(!kByF || kF % 2 == 0, "the last fragment's scores are acc[1]");
    mx_f32x4 acc[kAcc][4];
#pragma unroll
    for (int f = 0; f < kAcc; ++f)
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) acc[f][t][r] = kMx4Lowest;
    mx4_wait<0>();
    mx4_barrier();
    Piece now, next;
#pragma unroll
    for (int i = 0; i < 9; ++i) read(now, smem, 0, i);
#pragma unroll 1
    for (int64_t it = first; it < last; ++it) {
      const int half = (int)(it - first) & 1;
      const char *stage = smem + half * Shape::stage, *other = smem + (half ^ 1) * Shape::stage;
#pragma unroll
      for (int u = 0; u < kUnits; ++u) {
        const int unit = (int)it * kUnits + u;
#pragma unroll
        for (int s = 0; s < kT; ++s) {
          if (u == kUnits - 1 && s == kT - 1) {
            mx4_wait<0>();                     // everybody has read this stage, and the other one is there
            mx4_barrier();
            load(it + 2, half);
          }
          const char *from = s + 1 < kT ? stage + u * Shape::unit : u + 1 < kUnits ? stage + (u + 1) * Shape::unit : other;
#pragma unroll
          for (int f = 0; f < kF; ++f)
#pragma unroll
            for (int t = 0; t < 4; ++t) {
              mx_f32x4 &to = acc[kByF ? f & 1 : f][t];
              to = mx4_mfma_at(t, f & 3, now.w[t], y[f][s], s == 0 ? now.from[t] : to, now.sw, sy[f / 4][s]);
              read(next, from, s + 1 < kT ? s + 1 : 0, 4 * f + t);
              if (f == kF - 1 && t == 3)       // (fewer products than reads)
                for (int i = 4 * kF; i < 9; ++i) read(next, from, s + 1 < kT ? s + 1 : 0, i);
              if (s == 0 && f == 0) maxima(acc[kAcc - 1], kF - 1, unit - 1, t);
              else if (s == kT - 1 && f > 0) maxima(acc[kByF ? (f & 1) ^ 1 : f - 1], f - 1, unit, t);
              mx4_in_order();
            }
          now = next;
        }
      }
    }
#pragma unroll
    for (int t = 0; t < 4; ++t) maxima(acc[kAcc - 1], kF - 1, (int)last * kUnits - 1, t);
    mx4_wait<0>();
    mx4_barrier();                             // the stages may be filled again
    if (!kCollect) {
#pragma unroll
      for (int f = 0; f < kF; ++f) {
        int id = 4 * at[f] + q;
        float b = best[f], s = second[f];
#pragma unroll
        for (int o = 16; o < 64; o <<= 1) {
          const float ob = __shfl_xor(b, o), os = __shfl_xor(s, o);
          const int oid = __shfl_xor(id, o);
          s = fmaxf(fmaxf(s, os), fminf(b, ob));
          id = ob > b ? oid : id;
          b = fmaxf(b, ob);
        }
        const int64_t row = row0 + 16 * (wave * kF + f) + l16;
        if (q == 0 && row < n) records[(blockIdx.x - mx4_first_piece(cut, block)) * n + row] = Mx4Record{b, s, id};
      }
    }
  }
}

// ---------------------------------------------------------------- rows of any length
// kCollect: the instances are those of list (counts->listed of them); the groups whose maximum reaches an instance's threshold are appended to its
// list.  Otherwise one record per instance, piece of its block (Mx4Cut; a stage is a tile) and half of the wavefronts.
template <bool kCollect>
__global__ __launch_bounds__(512) void k_mx4_search(Mx4Operand x, Mx4Operand w, const float *__restrict__ init, int blocks,
                                                    const void *__restrict__ zero16, Mx4Cut cut, Mx4Record *__restrict__ records,
                                                    Mx4Counts *__restrict__ counts, const int *__restrict__ list,
                                                    const float *__restrict__ threshold, int *__restrict__ found,
                                                    int *__restrict__ groups, int *__restrict__ whole) {
  typedef Mx4Sweep Tile;
  __shared__ __attribute__((aligned(16))) char smem[Tile::kLds];
  const int64_t n = kCollect ? counts->listed : x.rows.n, nb = (n + Tile::kRowsB - 1) / Tile::kRowsB;
  if (kCollect) {
    if (n == 0) return;
    cut.per = (nb * cut.stages + gridDim.x - 1) / gridDim.x;
  }
  const int64_t total = x.rows.n;
  x.rows.n = n;
  int64_t pos = blockIdx.x * cut.per;
  const int64_t end = pos + cut.per < nb * cut.stages ? pos + cut.per : nb * cut.stages;
  while (pos < end) {
    const int64_t block = pos / cut.stages, row0 = block * Tile::kRowsB, first = pos - block * cut.stages;
    const int64_t last = first + (end - pos) < cut.stages ? first + (end - pos) : cut.stages;
    pos += last - first;
    Tile t;
    t.setup(smem, w, x, init, blocks, zero16);
    t.tile_b(row0, n, kCollect ? list : nullptr);
    float best[Tile::kFragB], second[Tile::kFragB];
    int at[Tile::kFragB];
#pragma unroll
    for (int v = 0; v < Tile::kFragB; ++v) {
      best[v] = second[v] = kMx4Lowest;
      at[v] = 0;
      if (kCollect) {
        const int64_t slot = row0 + 16 * (t.wb * Tile::kFragB + v) + t.l16;
        best[v] = slot < n ? threshold[slot] : INFINITY;
      }
    }
    t.run(first, last, [&](int64_t tile) {
#pragma unroll
      for (int g = 0; g < Tile::kFragA / 4; ++g)
#pragma unroll
        for (int v = 0; v < Tile::kFragB; ++v) {
          float m = kMx4Lowest;
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            const mx_f32x4 a = t.acc[4 * g + u][v];
            m = fmaxf(fmaxf(m, a[0]), a[1]);
            m = fmaxf(fmaxf(m, a[2]), a[3]);
          }
          const int id = (int)tile * (Tile::kFragA / 4) + g;
          if (kCollect) {
            if (m >= best[v]) {
              const int64_t slot = row0 + 16 * (t.wb * Tile::kFragB + v) + t.l16;
              const int place = atomicAdd(&found[slot], 1);
              if (place < kMx4List)
                groups[slot * kMx4List + place] = ((int)tile * (Tile::kRowsA / 64) + t.wa * (Tile::kFragA / 4) + g) * 4 + t.q;
              else if (place == kMx4List) whole[atomicAdd(&counts->whole, 1)] = list[slot];
            }
          } else {
            second[v] = fmaxf(second[v], fminf(best[v], m));
            at[v] = m > best[v] ? id : at[v];
            best[v] = fmaxf(best[v], m);
          }
        }
    });
    if (!kCollect) {
#pragma unroll
      for (int v = 0; v < Tile::kFragB; ++v) {
        // group of 16 nodes: tile, this wavefront's 64-node part, the lane's quarter of it
        int id = ((at[v] / (Tile::kFragA / 4)) * (Tile::kRowsA / 64) + t.wa * (Tile::kFragA / 4) + at[v] % (Tile::kFragA / 4)) * 4 + t.q;
        float b = best[v], s = second[v];
#pragma unroll
        for (int o = 16; o < 64; o <<= 1) {
          const float ob = __shfl_xor(b, o), os = __shfl_xor(s, o);
          const int oid = __shfl_xor(id, o);
          s = fmaxf(fmaxf(s, os), fminf(b, ob));
          id = ob > b ? oid : id;
          b = fmaxf(b, ob);
        }
        const int64_t row = row0 + 16 * (t.wb * Tile::kFragB + v) + t.l16;
        if (t.q == 0 && row < n) records[((blockIdx.x - mx4_first_piece(cut, block)) * Tile::kWavesA + t.wa) * total + row] = Mx4Record{b, s, id};
      }
    }
  }
}

// What two scores of an instance may differ by in fp32 without being in order: twice the error of one.  steps + 1 roundings of sums of terms whose
// magnitudes add up to |x| |w| + |w|^2 / 2 at most, |x|^2 taken as what its scales allow (x2: the sum of their squares); a term below the
// smallest normal fp32 number may be lost.  Infinite where the scores could overflow.
__device__ __forceinline__ double mx4_margin(double x2, float wmax2, int blocks) {
  const double size = sqrt(36.0 * 32.0 * x2) * sqrt((double)wmax2) + 0.5 * (double)wmax2;
  if (!(size < 1e37)) return INFINITY;
  return 2.0 * (((blocks - 1) / 4 + 2) * kMx4Delta * size + 1e-34 * blocks);
}

// A workgroup takes kEach instances, puts them in the order of their groups (more than 64 of them), and a wavefront multiplies 16 of them at a
// time with each of the groups among them, kBatch in flight (1 KB a step in one piece of the stream).  What bounds it is the groups' way from
// L2: 16 KB a step for 16 instances of as many groups.  See launch_resolve for the sizes.
template <int kThreads, int kEach, int kBatch>
__global__ __launch_bounds__(kThreads, 4) void k_mx4_resolve(Mx4Rows x, const char *__restrict__ stream, const char *__restrict__ by_group, int blocks,
                                                      int ngroups, const Mx4Record *__restrict__ records, Mx4Cut cut, int halves,
                                                      const float *__restrict__ parts, int nparts, Mx4Counts *__restrict__ counts,
                                                      int *__restrict__ list, float *__restrict__ threshold, int *__restrict__ found,
                                                      int *__restrict__ groups, int *__restrict__ whole, int32_t *__restrict__ bmus) {
  constexpr bool kSort = kEach > 64;             // (of fewer there is nothing to gain)
  __shared__ float s_best[kEach], s_second[kEach], s_inner[kEach];     // largest score, of the other groups, second one of the group
  __shared__ int s_group[kEach], s_first[kEach];                       // the group, the largest score's place in it
  __shared__ double s_x2[kEach];
  __shared__ int s_order[kSort ? kEach : 1], s_from[kSort ? kThreads : 1], s_wave[kThreads / 64];
  __shared__ float s_max[kThreads / 64];
  __shared__ int s_count[3], s_base[3];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l16 = lane & 15, q = lane >> 4, steps = (blocks - 1) / 4 + 1;
  const int64_t unit = mx4_stream_bytes(steps), row0 = (int64_t)blockIdx.x * kEach;
  const int mine = x.n - row0 < kEach ? (int)(x.n - row0) : kEach;
  float wmax2 = 0.f;
  for (int t = threadIdx.x; t < nparts; t += kThreads) wmax2 = fmaxf(wmax2, parts[t]);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) wmax2 = fmaxf(wmax2, __shfl_xor(wmax2, o));
  if (lane == 0) s_max[wave] = wmax2;
  if (threadIdx.x < 3) s_count[threadIdx.x] = 0;
  if (kSort) s_from[threadIdx.x] = 0;
  __syncthreads();
  wmax2 = s_max[0];
#pragma unroll
  for (int w = 1; w < kThreads / 64; ++w) wmax2 = fmaxf(wmax2, s_max[w]);
  constexpr int kTurns = (kEach + kThreads - 1) / kThreads;
  const int bits = 32 - __clz(ngroups - 1), most = 31 - __clz(kThreads), shift = bits > most ? bits - most : 0;
  int bucket[kTurns], place[kTurns];
#pragma unroll
  for (int u = 0; u < kTurns; ++u) {
    const int i = u * kThreads + threadIdx.x;
    bucket[u] = place[u] = 0;
    if (i < mine) {
      const int64_t row = row0 + i, block = row / cut.rows, pieces = mx4_last_piece(cut, block) - mx4_first_piece(cut, block) + 1;
      float best = kMx4Lowest, second = kMx4Lowest;
      int group = 0;
      for (int64_t p = 0; p < pieces * halves; ++p) {
        const Mx4Record r = records[p * x.n + row];
        second = fmaxf(fmaxf(second, r.second), fminf(best, r.best));
        group = r.best > best ? r.group : group;
        best = fmaxf(best, r.best);
      }
      s_best[i] = best;
      s_second[i] = second;
      s_group[i] = group;
      bucket[u] = group >> shift;
      if (kSort) place[u] = atomicAdd(&s_from[bucket[u]], 1);
    }
  }
  __syncthreads();
  if (kSort) {
    const int here = s_from[threadIdx.x];        // of a bucket; where it begins:
    int sum = here;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int t = __shfl_up(sum, o);
      if (lane >= o) sum += t;
    }
    if (lane == 63) s_wave[wave] = sum;
    __syncthreads();
    int before = 0;
    for (int w = 0; w < wave; ++w) before += s_wave[w];
    s_from[threadIdx.x] = before + sum - here;
    __syncthreads();
#pragma unroll
    for (int u = 0; u < kTurns; ++u)
      if (u * kThreads + (int)threadIdx.x < mine) s_order[s_from[bucket[u]] + place[u]] = u * kThreads + threadIdx.x;
    __syncthreads();
  }
#pragma unroll 1
  for (int i0 = wave * 16; i0 < mine; i0 += kThreads / 4) {
    const int nth = i0 + l16 < mine ? i0 + l16 : mine - 1, i = kSort ? s_order[nth] : nth;
    const int64_t row = row0 + i;
    const int group = s_group[i];
    double x2 = 0.0;                             // sum of the squares of the scales, NaN if one is
    mx_f32x4 mine4 = {0.f, 0.f, 0.f, 0.f};       // scores of nodes 4 q .. of instance l16's group
    unsigned left = 0xffff;
#pragma unroll 1
    for (bool begin = true; left != 0; begin = false) {
      int g[kBatch];
      mx_f32x4 acc[kBatch];
      const char *codes[kBatch], *scales[kBatch];
#pragma unroll
      for (int r = 0; r < kBatch; ++r) {         // (the last group again where there are fewer)
        g[r] = left != 0 || r == 0 ? __builtin_amdgcn_readlane(group, __builtin_ctz(left | 0x10000)) : g[r > 0 ? r - 1 : 0];
        left &= ~(unsigned)__ballot(group == g[r]);
        codes[r] = stream + (g[r] >> 2) * unit + (g[r] & 3) * 1024;
        scales[r] = by_group + (int64_t)g[r] * mx4_group_bytes(steps);
        acc[r] = *reinterpret_cast<const mx_f32x4 *>(scales[r] + steps * 64 + q * 16);
      }
      for (int s = 0; s < steps; ++s) {
        i32x4 c[kBatch];
        int e[kBatch];
#pragma unroll
        for (int r = 0; r < kBatch; ++r) {
          c[r] = *reinterpret_cast<const i32x4 *>(codes[r] + (int64_t)s * 4096 + lane * 16);
          e[r] = reinterpret_cast<const uint8_t *>(scales[r])[s * 64 + lane];
        }
        const int64_t b = row * blocks + (4 * s + q < blocks ? 4 * s + q : blocks - 1);
        const i32x4 xc = *reinterpret_cast<const i32x4 *>(x.codes + b * 16);
        const int xs = x.scales[b];
#pragma unroll
        for (int r = 0; r < kBatch; ++r) acc[r] = mx4_mfma<0, 0>(c[r], xc, acc[r], e[r], xs);
        if (begin && 4 * s + q < blocks) x2 += xs == 255 ? (double)NAN : mx4_pow2(2 * xs - 254);
      }
#pragma unroll
      for (int r = 0; r < kBatch; ++r)
        if (group == g[r]) mine4 = acc[r];
    }
    float b = kMx4Lowest, second = kMx4Lowest;
    int at = 4 * q;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const float m = fmaxf(mine4[u], kMx4Lowest);       // (not of a node with a NaN)
      second = fmaxf(second, fminf(b, m));
      at = m > b ? 4 * q + u : at;
      b = fmaxf(b, m);
    }
#pragma unroll
    for (int o = 16; o < 64; o <<= 1) {
      const float ob = __shfl_xor(b, o), os = __shfl_xor(second, o);
      const int oat = __shfl_xor(at, o);
      second = fmaxf(fmaxf(second, os), fminf(b, ob));
      at = ob > b ? oat : at;
      b = fmaxf(b, ob);
      x2 += __shfl_xor(x2, o);
    }
    if (q == 0 && i0 + l16 < mine) {
      s_inner[i] = second;
      s_first[i] = at;
      s_x2[i] = x2;
    }
  }
  __syncthreads();
  int where[kTurns];
  float reach[kTurns];
#pragma unroll
  for (int u = 0; u < kTurns; ++u) {
    const int i = u * kThreads + threadIdx.x;
    where[u] = -1;                               // which list it goes to; its place among this workgroup's
    if (i < mine) {
      const double x2 = s_x2[i], margin = mx4_margin(x2, wmax2, blocks);
      const float best = s_best[i];
      reach[u] = __double2float_rd((double)best - margin);
      if (x2 != x2) {                            // no finite distance to any node
        bmus[row0 + i] = 0;
      } else if (!(margin < INFINITY) || !(best > kMx4Lowest)) {
        where[u] = 2;
      } else if (s_second[i] >= reach[u]) {
        where[u] = 0;
      } else if (s_inner[i] < reach[u]) {
        bmus[row0 + i] = 16 * s_group[i] + s_first[i];
      } else {
        where[u] = 1;
      }
      if (where[u] >= 0) place[u] = atomicAdd(&s_count[where[u]], 1);
    }
  }
  __syncthreads();
  // (one addition a workgroup and list: with one for every instance the additions, all to one word, would take as long as the rest)
  if (threadIdx.x < 3 && s_count[threadIdx.x] > 0)
    s_base[threadIdx.x] = atomicAdd(threadIdx.x == 0 ? &counts->listed : threadIdx.x == 1 ? &counts->single : &counts->whole, s_count[threadIdx.x]);
  __syncthreads();
#pragma unroll
  for (int u = 0; u < kTurns; ++u) {
    const int i = u * kThreads + threadIdx.x;
    if (where[u] == 2) {
      whole[s_base[2] + place[u]] = (int)(row0 + i);
    } else if (where[u] >= 0) {
      const int64_t slot = where[u] == 0 ? s_base[0] + place[u] : x.n - 1 - (s_base[1] + place[u]);
      list[slot] = (int)(row0 + i);
      threshold[slot] = reach[u];
      found[slot] = where[u];
      if (where[u] == 1) groups[slot * kMx4List] = s_group[i];
    }
  }
}

// A wavefront an instance: lane l has node l % 16 of a group and every fourth block, kEach of those at a time.
template <int kEach>
__global__ __launch_bounds__(256) void k_mx4_exact(Mx4Rows x, Mx4Rows w, int blocks, const Mx4Counts *__restrict__ counts,
                                                   const int *__restrict__ list, const int *__restrict__ found,
                                                   const int *__restrict__ groups, const int *__restrict__ whole, int log_lanes,
                                                   Mx4Joined join, int32_t *__restrict__ bmus) {
  // those for all nodes first: they take longest
  const int all = counts->whole, most = (int)gridDim.x / (all > 0 ? all : 1);
  const int shares = all >= kMx4Tickets || most < 1 ? 1 : most < 64 ? most : 64;
  for (int64_t job = blockIdx.x; job < (int64_t)all * shares; job += gridDim.x) {
    mx4_scan(x, w, blocks, log_lanes, whole[job / shares], (int)(job % shares), shares, (int)(job / shares), join, bmus);
    __syncthreads();
  }
  const int lane = threadIdx.x & 63, l16 = lane & 15, q = lane >> 4;
  const int64_t listed = counts->listed, total = listed + counts->single;
  for (int64_t u = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); u < total; u += (int64_t)gridDim.x * 4) {
    const int64_t slot = u < listed ? u : x.n - 1 - (u - listed);
    const int64_t row = list[slot];
    const int ng = found[slot];
    if (ng > kMx4List) continue;               // (among those above)
    double best = -INFINITY;
    int arg = 0x7fffffff;
    for (int g = 0; g < ng; ++g) {
      const int64_t node = 16 * (int64_t)groups[slot * kMx4List + g] + l16, wr = node < w.n ? node : w.n - 1;
      double s = 0.0;
      for (int b0 = q; b0 < blocks; b0 += 4 * kEach) {
        i32x4 xc[kEach], wc[kEach];
        int ex[kEach], ew[kEach];
#pragma unroll
        for (int u = 0; u < kEach; ++u) {
          const int b = b0 + 4 * u < blocks ? b0 + 4 * u : blocks - 1;      // (a load under a condition would be waited for by itself)
          xc[u] = *reinterpret_cast<const i32x4 *>(x.codes + (row * blocks + b) * 16);
          wc[u] = *reinterpret_cast<const i32x4 *>(w.codes + (wr * blocks + b) * 16);
          ex[u] = x.scales[row * blocks + b];
          ew[u] = w.scales[wr * blocks + b];
        }
#pragma unroll
        for (int u = 0; u < kEach; ++u) {
          float xw, ww;
          mx4_block_dots(xc[u], wc[u], xw, ww);
          double part = (double)xw * mx4_pow2(ex[u] + ew[u] - 254) - (double)ww * mx4_pow2(2 * ew[u] - 255);
          if (ex[u] == 255 || ew[u] == 255) part = NAN;
          s += b0 + 4 * u < blocks ? part : 0.0;
        }
      }
      s += __shfl_xor(s, 16);
      s += __shfl_xor(s, 32);
      if (node < w.n && mx4_better(s, (int)node, best, arg)) { best = s; arg = (int)node; }
    }
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) {
      const double s = __shfl_xor(best, o);
      const int i = __shfl_xor(arg, o);
      if (mx4_better(s, i, best, arg)) { best = s; arg = i; }
    }
    if (lane == 0) bmus[row] = arg == 0x7fffffff ? 0 : arg;
  }
}

// How the pass over all instances is laid out.
struct Mx4Layout {
  bool sweep;              // k_mx4_sweep, else k_mx4_search
  Mx4Cut cut;
  int at_once;             // workgroups a CU holds
  int grid, records;       // workgroups; records of an instance
  int64_t padded;          // nodes rounded up to whole stages
};

template <int kT>
static void sweep_shape(int steps, int *rows, int *nodes, int *at_once) {
  if (steps == kT) {
    typedef typename Mx4ShapeOf<kT, false>::type Shape;
    *rows = Shape::rows;
    *at_once = Shape::waves;
    *nodes = 64 * Shape::units;
  }
}

static Mx4Layout search_layout(const som_ctx *c, int64_t n) {
  Mx4Layout l;
  const int steps = (mx4_blocks(c->dim) - 1) / 4 + 1;
  int nodes = Mx4Sweep::kRowsA, at_once = 1;      // nodes of a stage, workgroups a CU holds
  l.sweep = steps <= kMx4SweepSteps;
  l.cut.rows = Mx4Sweep::kRowsB;
  if (l.sweep) {
    sweep_shape<1>(steps, &l.cut.rows, &nodes, &at_once); sweep_shape<2>(steps, &l.cut.rows, &nodes, &at_once);
    sweep_shape<3>(steps, &l.cut.rows, &nodes, &at_once); sweep_shape<4>(steps, &l.cut.rows, &nodes, &at_once);
    sweep_shape<5>(steps, &l.cut.rows, &nodes, &at_once); sweep_shape<6>(steps, &l.cut.rows, &nodes, &at_once);
    sweep_shape<7>(steps, &l.cut.rows, &nodes, &at_once); sweep_shape<8>(steps, &l.cut.rows, &nodes, &at_once);
  }
  l.cut.stages = ((int64_t)c->k + nodes - 1) / nodes;
  l.padded = l.cut.stages * nodes;
  const int64_t all = (n + l.cut.rows - 1) / l.cut.rows * l.cut.stages, most = at_once * (int64_t)c->n_cu;
  l.cut.per = (all + most - 1) / most;
  l.at_once = at_once;
  l.grid = (int)((all + l.cut.per - 1) / l.cut.per);
  // pieces that a block's stages can be spread over
  const int64_t pieces = (l.cut.stages + l.cut.per - 2) / l.cut.per + 1;
  l.records = (int)(pieces < l.grid ? pieces : l.grid) * (l.sweep ? 1 : Mx4Sweep::kWavesA);
  return l;
}

// Direct, or on the matrix cores?  What either takes, in us, fitted to measurements (instances, nodes, features, us matrix cores / direct: 1, 2,500,
// 1,000 32 / 7; 100, 2,500, 1,000 49 / 34; 200 62 / 56; 400 68 / 101; 10,000, 400, 32 42 / 23; 20,000 43 / 42; 30, 40,000, 256 111 / 48; 100 114 / 135;
// 3,000, 1,000, 128 34 / 46; 300, 300, 4,000 152 / 49; 100,000, 9, 100 27 / 115).
static bool direct_pays(const som_ctx *c, int64_t n) {
  const double blocks = mx4_blocks(c->dim), steps = (mx4_blocks(c->dim) - 1) / 4 + 1;
  const double direct = 8.0 + 2.6e-6 * n * c->k * (blocks + 0.6) + 8e-4 * n;
  const double matrix = 30.0 + 2.5 * steps + 6e-4 * c->k * steps + 2e-4 * n;
  return direct <= matrix;
}

struct Mx4SearchScratch {
  float *init, *parts, *threshold;
  char *stream, *by_group;
  int *packed_w, *packed_x, *list, *found, *groups, *whole, *joined_node;
  double *joined_score;
  Mx4Counts *counts;
  Mx4Record *records;
  size_t bytes;
};

static Mx4SearchScratch search_scratch(const som_ctx *c, int64_t n, const Mx4Layout &l, void *base) {
  const int blocks = mx4_blocks(c->dim), steps = (blocks - 1) / 4 + 1;
  const size_t N = (size_t)n;
  Mx4SearchScratch m;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    void *p = static_cast<char *>(base) + at;
    at += (bytes + 255) / 256 * 256;
    return p;
  };
  m.init = static_cast<float *>(take(l.sweep ? 0 : (size_t)l.padded * 4));
  m.parts = static_cast<float *>(take(kMx4NodeBlocks * 4));
  m.counts = static_cast<Mx4Counts *>(take(sizeof(Mx4Counts)));
  m.stream = static_cast<char *>(take((size_t)(l.padded / 64) * mx4_stream_bytes(steps)));
  m.by_group = static_cast<char *>(take((size_t)(l.padded / 16) * mx4_group_bytes(steps)));
  m.packed_w = static_cast<int *>(take(l.sweep ? 0 : mx4_packed_bytes(c->k, blocks)));
  m.packed_x = static_cast<int *>(take(l.sweep ? 0 : mx4_packed_bytes(n, blocks)));
  m.records = static_cast<Mx4Record *>(take((size_t)l.records * N * sizeof(Mx4Record)));
  m.list = static_cast<int *>(take(N * 4));
  m.threshold = static_cast<float *>(take(N * 4));
  m.found = static_cast<int *>(take(N * 4));
  m.groups = static_cast<int *>(take(N * kMx4List * 4));
  m.whole = static_cast<int *>(take(N * 4));
  m.joined_score = static_cast<double *>(take(kMx4ScanBlocks * sizeof(double)));
  m.joined_node = static_cast<int *>(take(kMx4ScanBlocks * sizeof(int)));
  m.bytes = at;
  return m;
}

// A search takes its instances in equal parts, of at most kMx4AtOnce instances and so many that what grows with them (168 bytes each, of rows of
// more than 1,024 features 192 and four for every 128) is at most kMx4PartBytes: its scratch stays bounded, besides the nodes', however large
// the set and long the rows.  The first instance too many costs 6 % on rows as short as this matters for (4,194,304 x 32 on 900 nodes 494 us, one more
// 521).
constexpr int64_t kMx4AtOnce = 1 << 22, kMx4PartBytes = 1 << 30;
static int64_t part_of(const som_ctx *c, int64_t n) {
  int64_t parts = (n + kMx4AtOnce - 1) / kMx4AtOnce;
  for (;;) {
    const int64_t part = (n + parts - 1) / parts;
    if (part <= 4096 || direct_pays(c, part)) return part;
    const Mx4Layout l = search_layout(c, part);
    const int64_t each = (int64_t)l.records * sizeof(Mx4Record) + (4 + kMx4List) * 4 + (l.sweep ? 0 : mx4_packed_bytes(64, mx4_blocks(c->dim)) / 64);
    if (part * each <= kMx4PartBytes) return part;
    const int64_t wanted = (n * each + kMx4PartBytes - 1) / kMx4PartBytes;
    parts = wanted > parts ? wanted : parts + 1;
  }
}

static size_t part_bytes(const som_ctx *c, int64_t n) {
  if (!direct_pays(c, n)) return search_scratch(c, n, search_layout(c, n), nullptr).bytes;
  const int shares = direct_shares(c, n, 1 << direct_lanes_log(mx4_blocks(c->dim)));
  return shares > 1 ? (size_t)n * shares * (sizeof(double) + sizeof(int)) : 0;
}

size_t mx4_search_bytes(const som_ctx *c, int64_t n) {
  const int64_t part = part_of(c, n), last = (n - 1) % part + 1;
  const size_t a = part_bytes(c, part), b = part_bytes(c, last);
  return a > b ? a : b;
}

template <int kT, bool kCollect>
static void launch_sweep(som_ctx *c, Mx4Rows x, const Mx4Layout &l, const Mx4SearchScratch &m, dim3 grid) {
  hipLaunchKernelGGL((k_mx4_sweep<kT, kCollect>), grid, dim3(256), 0, c->stream, x, mx4_blocks(c->dim), m.stream, l.cut, m.records,
                     m.counts, m.list, m.threshold, m.found, m.groups, m.whole);
}

// The pass over all instances (kCollect: over those that are listed, as many workgroups as fill the chip at most).
template <bool kCollect>
static hipError_t launch_pass(som_ctx *c, Mx4Rows x, Mx4Rows w, const Mx4Layout &l, const Mx4SearchScratch &m) {
  const int blocks = mx4_blocks(c->dim);
  const dim3 grid(kCollect ? l.at_once * c->n_cu : l.grid);
  if (l.sweep) {
    switch ((blocks - 1) / 4 + 1) {
      case 1: launch_sweep<1, kCollect>(c, x, l, m, grid); break;
      case 2: launch_sweep<2, kCollect>(c, x, l, m, grid); break;
      case 3: launch_sweep<3, kCollect>(c, x, l, m, grid); break;
      case 4: launch_sweep<4, kCollect>(c, x, l, m, grid); break;
      case 5: launch_sweep<5, kCollect>(c, x, l, m, grid); break;
      case 6: launch_sweep<6, kCollect>(c, x, l, m, grid); break;
      case 7: launch_sweep<7, kCollect>(c, x, l, m, grid); break;
      default: launch_sweep<8, kCollect>(c, x, l, m, grid);
    }
    return hipGetLastError();
  }
  const hipError_t e = launch_mx4_pack_scales(c->stream, blocks, Mx4Unpacked{x.scales, x.n, false, m.packed_x, kCollect ? m.list : nullptr,
                                                                             kCollect ? &m.counts->listed : nullptr});
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(k_mx4_search<kCollect>, grid, dim3(Mx4Sweep::kThreads), 0, c->stream, Mx4Operand{x, m.packed_x}, Mx4Operand{w, m.packed_w},
                     m.init, blocks, c->zero16, l.cut, m.records, m.counts, m.list, m.threshold, m.found, m.groups, m.whole);
  return hipGetLastError();
}

template <int kThreads, int kEach, int kBatch>
static void launch_resolve_of(som_ctx *c, Mx4Rows x, const Mx4Layout &l, const Mx4SearchScratch &m, int parts, int32_t *bmus) {
  hipLaunchKernelGGL((k_mx4_resolve<kThreads, kEach, kBatch>), dim3((unsigned)((x.n + kEach - 1) / kEach)), dim3(kThreads), 0, c->stream, x, m.stream,
                     m.by_group, mx4_blocks(c->dim), (int)(l.padded / 16), m.records, l.cut, l.sweep ? 1 : Mx4Sweep::kWavesA, m.parts, parts, m.counts,
                     m.list, m.threshold, m.found, m.groups, m.whole, bmus);
}

// The more instances are put in order the more of 16 have the same group, but fewer workgroups share the work: half as many as
// CUs are enough (whole search, us, 64 / 512 / 2,048 instances a workgroup: 1e6 x 10,000 x 128 721 / 714 / 653, 200,000 x 2,500 x 1,000 361 / 327 / 340, 100,000
// x 2,500 x 1,000 214 / 191 / 240, 50,000 x 2,500 x 128 56 / 56 / 64, 16,000 x 2,500 x 1,000 96 / 120 / 171).
static void launch_resolve(som_ctx *c, Mx4Rows x, const Mx4Layout &l, const Mx4SearchScratch &m, int parts, int32_t *bmus) {
  if (x.n >= 1024 * (int64_t)c->n_cu) launch_resolve_of<1024, 2048, 4>(c, x, l, m, parts, bmus);
  else if (x.n >= 256 * (int64_t)c->n_cu) launch_resolve_of<1024, 512, 6>(c, x, l, m, parts, bmus);
  else launch_resolve_of<256, 64, 8>(c, x, l, m, parts, bmus);
}

static hipError_t search_part(som_ctx *c, Mx4Rows x, Mx4Rows w, void *scratch, int *tickets, int32_t *bmus) {
  if (direct_pays(c, x.n)) return search_direct(c, x, w, scratch, tickets, bmus);
  const Mx4Layout l = search_layout(c, x.n);
  const Mx4SearchScratch m = search_scratch(c, x.n, l, scratch);
  const int blocks = mx4_blocks(c->dim);
  const int parts = l.padded / 64 < kMx4NodeBlocks ? (int)(l.padded / 64) : kMx4NodeBlocks;
  hipLaunchKernelGGL(k_mx4_nodes, dim3(parts), dim3(256), 0, c->stream, w, blocks, c->cols, l.padded, l.sweep ? nullptr : m.init, m.stream, m.by_group,
                     l.sweep ? nullptr : m.packed_w, m.parts, m.counts);
  hipError_t e = launch_pass<false>(c, x, w, l, m);
  if (e != hipSuccess) return e;
  launch_resolve(c, x, l, m, parts, bmus);
  e = launch_pass<true>(c, x, w, l, m);
  if (e != hipSuccess) return e;
  const int64_t wanted = (x.n + 3) / 4;
  const dim3 grid((unsigned)(wanted < kMx4ScanBlocks ? wanted : kMx4ScanBlocks));
  const Mx4Joined join = {m.joined_score, m.joined_node, tickets};
  if (blocks > 8)
    hipLaunchKernelGGL(k_mx4_exact<4>, grid, dim3(256), 0, c->stream, x, w, blocks, m.counts, m.list, m.found, m.groups, m.whole,
                       direct_lanes_log(blocks), join, bmus);
  else
    hipLaunchKernelGGL(k_mx4_exact<1>, grid, dim3(256), 0, c->stream, x, w, blocks, m.counts, m.list, m.found, m.groups, m.whole,
                       direct_lanes_log(blocks), join, bmus);
  return hipGetLastError();
}

hipError_t launch_bmu_mx4(som_ctx *c, Mx4Rows x, Mx4Rows w, void *scratch, int *tickets, int32_t *bmus) {
  const int64_t part = part_of(c, x.n), blocks = mx4_blocks(c->dim);
  for (int64_t r0 = 0; r0 < x.n; r0 += part) {
    const Mx4Rows rows = {x.codes + r0 * blocks * 16, x.scales + r0 * blocks, x.n - r0 < part ? x.n - r0 : part};
    const hipError_t e = search_part(c, rows, w, scratch, tickets, bmus + r0);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace som
