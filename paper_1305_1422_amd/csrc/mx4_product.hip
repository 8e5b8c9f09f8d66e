// Dot products of all pairs of two sets of microscaled 4-bit rows (som_mx4_product): out[i][j] = sum_c a_ic b_jc, fp32
// accumulation on the scaled matrix cores, rounded once to the type of the output.  The rows of b are operand A of the
// instruction (mx4_tiles.hpp), so that a lane ends up with 16 consecutive products of a row of the output.
#include "mx4_tiles.hpp"

namespace som {

// ---------------------------------------------------------------- scales
// One set of rows or two (b.packed null: one).
__global__ __launch_bounds__(256) void k_mx4_pack_scales(Mx4Unpacked a, Mx4Unpacked b, int blocks, int steps) {
  const int64_t na = a.count ? *a.count : a.n;
  const int64_t words_a = (na + 63) / 64 * steps * 64, words = words_a + (b.n + 63) / 64 * steps * 64;
  for (int64_t w0 = (int64_t)blockIdx.x * 256 + threadIdx.x; w0 < words; w0 += (int64_t)gridDim.x * 256) {
    const bool second = w0 >= words_a;
    const int64_t w = second ? w0 - words_a : w0, n = second ? b.n : na;
    const uint8_t *scales = second ? b.scales : a.scales;
    const int *list = second ? b.list : a.list;
    const bool dealt = second ? b.dealt : a.dealt;
    const int lane = (int)(w & 63), i = lane & 15;
    const int64_t gs = w >> 6, g = gs / steps;
    const int block = 4 * (int)(gs - g * steps) + (lane >> 4);
    unsigned v = 0;
    if (block < blocks)
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const int64_t r = 64 * g + (dealt ? mx4_dealt(t, i) : 16 * t + i);
        if (r < n) v |= (unsigned)scales[(list ? list[r] : r) * blocks + block] << (8 * t);
      }
    (second ? b.packed : a.packed)[w] = (int)v;
  }
}

hipError_t launch_mx4_pack_scales(hipStream_t stream, int blocks, Mx4Unpacked a, Mx4Unpacked b) {
  const int steps = (blocks - 1) / 4 + 1;
  int64_t grid = ((a.n + 63) / 64 + (b.n + 63) / 64) * steps / 4 + 1;
  if (grid > 4096) grid = 4096;
  hipLaunchKernelGGL(k_mx4_pack_scales, dim3((unsigned)grid), dim3(256), 0, stream, a, b, blocks, steps);
  return hipGetLastError();
}

// ---------------------------------------------------------------- few rows: a wavefront's 16 rows of a and 64 of b straight from memory
template <typename T>
__global__ __launch_bounds__(256) void k_mx4_product_few(Mx4Rows a, Mx4Rows b, int blocks, T *__restrict__ out, int64_t stride) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l16 = lane & 15, q = lane >> 4;
  const int64_t j0 = ((int64_t)blockIdx.x * 4 + wave) * 64, i = (int64_t)blockIdx.y * 16 + l16;
  if (j0 >= b.n) return;
  const int64_t ia = i < a.n ? i : a.n - 1;
  int64_t jb[4];
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    jb[t] = j0 + mx4_dealt(t, l16);
    if (jb[t] >= b.n) jb[t] = b.n - 1;
  }
  mx_f32x4 acc[4] = {};
  for (int k0 = 0; k0 < blocks; k0 += 4) {
    const bool in = k0 + q < blocks;
    const int k = in ? k0 + q : blocks - 1;      // (a load under a condition would be waited for by itself)
    i32x4 x = *reinterpret_cast<const i32x4 *>(a.codes + (ia * blocks + k) * 16);
    const int sx = a.scales[ia * blocks + k];
    i32x4 y[4];
    int sy[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      y[t] = *reinterpret_cast<const i32x4 *>(b.codes + (jb[t] * blocks + k) * 16);
      sy[t] = b.scales[jb[t] * blocks + k];
    }
    if (!in) x = i32x4{0, 0, 0, 0};
#pragma unroll
    for (int t = 0; t < 4; ++t) acc[t] = mx4_mfma<0, 0>(y[t], x, acc[t], sy[t], sx);
  }
  if (i >= a.n) return;
#pragma unroll
  for (int t = 0; t < 4; ++t)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int64_t j = j0 + 16 * q + 4 * t + r;
      if (j < b.n) out[i * stride + j] = (T)acc[t][r];
    }
}

// ---------------------------------------------------------------- tiles
// A wavefront's results leave through LDS, 16 rows at a time, so that its stores are whole stretches of a row (written as the lanes hold them, 16
// bytes in each of 16 rows an instruction, 50,000 x 10,000 products of 256 features to bf16 take 281 us instead of 256).  kWidth bytes a lane.
template <typename T, int kCols, int kWidth>
__device__ __forceinline__ void mx4_store_rows(const T *block, int pitch, T *__restrict__ out, int64_t stride, int64_t rows, int64_t cols, int lane) {
  constexpr int kEach = kWidth / (int)sizeof(T), kLanes = kCols / kEach, kAtOnce = kLanes < 64 ? 64 / kLanes : 1;
  typedef T Vec __attribute__((ext_vector_type(kEach)));
#pragma unroll
  for (int r0 = 0; r0 < 16; r0 += kAtOnce)
#pragma unroll
    for (int c0 = 0; c0 < kLanes; c0 += 64) {
      const int r = r0 + (kLanes < 64 ? lane / kLanes : 0), c = (c0 + (kLanes < 64 ? lane % kLanes : lane)) * kEach;
      if (r >= rows || c >= cols) continue;
      const T *src = block + r * pitch + c;
      T *dst = out + r * stride + c;
      if (c + kEach <= cols) {
        *reinterpret_cast<Vec *>(dst) = *reinterpret_cast<const Vec *>(src);
      } else {
#pragma unroll
        for (int u = 0; u < kEach; ++u)
          if (c + u < cols) dst[u] = src[u];
      }
    }
}

constexpr int kMx4Band = 8;

// width: bytes that the rows of the output are aligned to, 16, 4 or 2.
template <typename T, typename Tile>
__global__ __launch_bounds__(512, (Tile::kFragB == 2 ? 4 : 2)) void k_mx4_product(Mx4Operand a, Mx4Operand b, int blocks, const void *__restrict__ zero16,
                                                     T *__restrict__ out, int64_t stride, unsigned tiles_j, int width) {
  constexpr int kCols = 16 * Tile::kFragA, kPitch = kCols + 16 / (int)sizeof(T);
  __shared__ __attribute__((aligned(16))) char smem[Tile::kLds];
  static_assert(Tile::kWaves * 16 * kPitch * (int)sizeof(T) <= Tile::kLds, "the results of 16 rows of every wavefront");
  Tile t;
  // Workgroups are dealt to the eight XCDs in turn.  Each XCD gets a stretch of consecutive tiles, kMx4Band rows of tiles column by column, so that the
  // lines of the output that two tiles share meet in one L2 and so do the operands (us, as dealt / row by row of tiles / in bands: to bf16, 50,000 x 10,000
  // x 256 326 / 323 / 247, 20,000 x 10,000 x 1,000 212 / 198 / 187, 8,192 x 8,192 x 4,096 160 / 172 / 160; to fp32, 100,000 x 2,500 x 1,000 456 / - / 377).
  const unsigned share = gridDim.x / 8, spare = gridDim.x % 8, xcd = blockIdx.x % 8;
  const unsigned tile = xcd * share + (xcd < spare ? xcd : spare) + blockIdx.x / 8;
  const unsigned band = tile / (kMx4Band * tiles_j), in_band = tile - band * kMx4Band * tiles_j;
  const unsigned high = min((unsigned)kMx4Band, gridDim.x / tiles_j - band * kMx4Band);
  const unsigned tj = in_band / high, ti = band * kMx4Band + in_band - tj * high;
  t.setup(smem, b, a, nullptr, blocks, zero16);
  const int64_t i0 = (int64_t)ti * Tile::kRowsB, j0 = (int64_t)tj * Tile::kRowsA + t.wa * kCols;
  t.tile_b(i0, a.rows.n, nullptr);
  t.run(tj, tj + 1, [](int64_t) {});
  T *block = reinterpret_cast<T *>(smem) + t.wave * 16 * kPitch;
#pragma unroll
  for (int v = 0; v < Tile::kFragB; ++v) {
#pragma unroll
    for (int g = 0; g < Tile::kFragA / 4; ++g) {
      T row[16];
#pragma unroll
      for (int u = 0; u < 16; ++u) row[u] = (T)t.acc[4 * g + u / 4][v][u & 3];
#pragma unroll
      for (int u = 0; u < (int)sizeof(T); ++u)
        reinterpret_cast<i32x4 *>(block + t.l16 * kPitch + 64 * g + 16 * t.q)[u] = reinterpret_cast<const i32x4 *>(row)[u];
    }
    const int64_t i = i0 + 16 * (t.wb * Tile::kFragB + v);
    T *dst = out + i * stride + j0;
    if (width == 16) mx4_store_rows<T, kCols, 16>(block, kPitch, dst, stride, a.rows.n - i, b.rows.n - j0, t.lane);
    else if (width == 4) mx4_store_rows<T, kCols, 4>(block, kPitch, dst, stride, a.rows.n - i, b.rows.n - j0, t.lane);
    else mx4_store_rows<T, kCols, (int)sizeof(T)>(block, kPitch, dst, stride, a.rows.n - i, b.rows.n - j0, t.lane);
    __builtin_amdgcn_wave_barrier();           // (a wavefront's LDS accesses are in order: the next rows may follow)
  }
}

typedef Mx4Tile<8, 4, 2, 4, false> Mx4Wide;       // 256 x 256
typedef Mx4Tile<8, 2, 2, 4, false> Mx4Low;        // 256 columns x 128 rows: two workgroups a CU
typedef Mx4Tile<4, 2, 2, 4, false> Mx4Narrow;     // 128 x 128

// Up to this many rows of a the operands come straight from memory.
constexpr int64_t kFewRows = 64;

static int64_t tiles(int64_t rows, int per) { return (rows + per - 1) / per; }

size_t mx4_product_bytes(const som_ctx *c, int64_t n, int64_t m) {
  const int blocks = mx4_blocks(c->dim);
  return n <= kFewRows ? 0 : mx4_packed_bytes(n, blocks) + mx4_packed_bytes(m, blocks);
}

template <typename T, typename Tile>
static hipError_t product_tiles(som_ctx *c, Mx4Operand a, Mx4Operand b, T *out, int64_t stride) {
  const int blocks = mx4_blocks(c->dim);
  const int64_t tj = tiles(b.rows.n, Tile::kRowsA), ti = tiles(a.rows.n, Tile::kRowsB);
  const uintptr_t both = (uintptr_t)out | (uintptr_t)(a.rows.n > 1 ? stride * (int64_t)sizeof(T) : 0);
  const int width = both % 16 == 0 ? 16 : both % 4 == 0 ? 4 : 2;
  // tile rows of a launch: HIP takes fewer than 2^32 threads in one (one row of tiles always fits: 65 rows of 2^31 products do not fit the card)
  const int64_t fit = ((1ll << 32) - 1) / Tile::kThreads / tj, most = fit > 0 ? fit : 1;
  for (int64_t t0 = 0; t0 < ti; t0 += most) {
    const int64_t now = ti - t0 < most ? ti - t0 : most, i0 = t0 * Tile::kRowsB;
    Mx4Operand part = a;
    part.rows.codes += i0 * blocks * 16;
    part.rows.scales += i0 * blocks;
    part.rows.n = a.rows.n - i0;
    part.packed += (size_t)(i0 / 64) * ((blocks - 1) / 4 + 1) * 64;
    const dim3 grid((unsigned)(now * tj));
    hipLaunchKernelGGL((k_mx4_product<T, Tile>), grid, dim3(Tile::kThreads), 0, c->stream, part, b, blocks, c->zero16, out + i0 * stride, stride,
                       (unsigned)tj, width);
  }
  return hipGetLastError();
}

template <typename T>
static hipError_t product(som_ctx *c, Mx4Rows a, Mx4Rows b, T *out, int64_t stride, void *scratch) {
  const int blocks = mx4_blocks(c->dim);
  if (a.n <= kFewRows) {
    const dim3 grid((unsigned)((b.n + 255) / 256), (unsigned)((a.n + 15) / 16));
    hipLaunchKernelGGL(k_mx4_product_few<T>, grid, dim3(256), 0, c->stream, a, b, blocks, out, stride);
    return hipGetLastError();
  }
  int *pa = static_cast<int *>(scratch), *pb = pa + mx4_packed_bytes(a.n, blocks) / 4;
  const hipError_t e = launch_mx4_pack_scales(c->stream, blocks, Mx4Unpacked{a.scales, a.n, false, pa}, Mx4Unpacked{b.scales, b.n, true, pb});
  if (e != hipSuccess) return e;
  const Mx4Operand oa = {a, pa}, ob = {b, pb};
  // Rows of up to 512 features are bound by the output: two workgroups a CU, one's stores beside the other's products (to bf16, us, wide / low
  // tiles: 50,000 x 10,000 x 128 255 / 216, 256 290 / 247, 384 338 / 282, 20,000 x 10,000 x 500 145 / 141, 1,000 187 / 208; to fp32, 100,000 x 2,500 x
  // 128 292 / 260, 384 309 / 264, 512 320 / 287, 768 351 / 363, 1,000 378 / 412, 20,000 x 10,000 x 500 204 / 191, 1,000 241 / 261).
  if (tiles(a.n, Mx4Wide::kRowsB) * tiles(b.n, Mx4Wide::kRowsA) >= c->n_cu)
    return blocks <= 16 ? product_tiles<T, Mx4Low>(c, oa, ob, out, stride) : product_tiles<T, Mx4Wide>(c, oa, ob, out, stride);
  return product_tiles<T, Mx4Narrow>(c, oa, ob, out, stride);
}

hipError_t launch_mx4_product(som_ctx *c, Mx4Rows a, Mx4Rows b, void *out, int type, int64_t stride, void *scratch) {
  if (type == SOM_FP32) return product(c, a, b, static_cast<float *>(out), stride, scratch);
  if (type == SOM_FP16) return product(c, a, b, static_cast<_Float16 *>(out), stride, scratch);
  return product(c, a, b, static_cast<__bf16 *>(out), stride, scratch);
}

}  // namespace som
