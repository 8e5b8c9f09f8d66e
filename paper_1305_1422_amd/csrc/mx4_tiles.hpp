// Products of two sets of microscaled 4-bit rows in tiles: the loop that som_mx4_product and the searches share (mx4.hpp has the format and the instruction).
//
// Eight wavefronts take a tile of kRowsA rows of operand A and kRowsB of operand B, a step of 128 features at a time.
// Operand layout in LDS is the instruction's own: a fragment (16 rows x 128 features) is 64 lanes x 16 bytes, filled by one
// direct-to-LDS load in which lane l fetches block l / 16 of row l % 16 (four consecutive blocks of a row are 64 bytes), and read back by one
// ds_read_b128 without bank conflicts.  The scales come packed: for 64 rows and a step one word per lane, byte t for fragment t
// (k_mx4_pack_scales), so that the instruction's byte selectors take them apart.  A's rows are dealt to the fragments so that a lane's
// results of four fragments are 16 consecutive rows of A: fragment t, row i of 64 rows is row 16 (i / 4) + 4 t + i % 4.
//
// A wavefront multiplies kFragA x kFragB fragments: with 8 x 4 a step is 32 instructions of 16 cycles for 12 KB of LDS reads, 94 bytes a cycle
// and CU of 128; two wavefronts a SIMD, so that one's reads and epilogue run under the other's products.  Three stages in LDS: the loads of
// step j + 2 are issued before the products of step j, one barrier a step.
#pragma once

#include "lds_load.hpp"
#include "mx4.hpp"

namespace som {

typedef __attribute__((address_space(3))) void *mx4_lds_t;

// All but the wavefront's kLeft most recent vector memory operations are done, and its LDS reads.
template <int kLeft>
__device__ __forceinline__ void mx4_wait() {
  asm volatile("" : : : "memory");
  __builtin_amdgcn_s_waitcnt(0x0070 | (kLeft & 15) | ((kLeft >> 4) << 14));
  asm volatile("" : : : "memory");
}
__device__ __forceinline__ void mx4_barrier() {
  asm volatile("" : : : "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" : : : "memory");
}

// The instruction with the scale bytes a and b, which are constants once the loops around it are unrolled.
__device__ __forceinline__ mx_f32x4 mx4_mfma_at(int a, int b, i32x4 x, i32x4 y, mx_f32x4 c, int sx, int sy) {
#define MX4_CASE(A, B) if (a == A && b == B) return mx4_mfma<A, B>(x, y, c, sx, sy);
  MX4_CASE(0, 0) MX4_CASE(0, 1) MX4_CASE(0, 2) MX4_CASE(0, 3) MX4_CASE(1, 0) MX4_CASE(1, 1) MX4_CASE(1, 2) MX4_CASE(1, 3)
  MX4_CASE(2, 0) MX4_CASE(2, 1) MX4_CASE(2, 2) MX4_CASE(2, 3) MX4_CASE(3, 0) MX4_CASE(3, 1) MX4_CASE(3, 2)
#undef MX4_CASE
  return mx4_mfma<3, 3>(x, y, c, sx, sy);
}

// Row of the 64 that fragment t holds as its row i (operand A).
__device__ __forceinline__ int mx4_dealt(int t, int i) { return 16 * (i >> 2) + 4 * t + (i & 3); }

// An operand: its rows, and their scales packed for the tiles ([ceil(n / 64)][steps][64] words).
struct Mx4Operand {
  Mx4Rows rows;
  const int *packed;
};

// kInit: the accumulators start from numbers of A's rows instead of zero.
template <int kFragA_, int kFragB_, int kWavesA_, int kWavesB_, bool kInit>
struct Mx4Tile {
  static constexpr int kFragA = kFragA_, kFragB = kFragB_, kWavesA = kWavesA_, kWavesB = kWavesB_;
  static constexpr int kWaves = kWavesA * kWavesB, kThreads = 64 * kWaves;
  static constexpr int kAllA = kFragA * kWavesA, kAllB = kFragB * kWavesB;      // fragments of the tile
  static constexpr int kRowsA = 16 * kAllA, kRowsB = 16 * kAllB;
  static constexpr int kLoadA = kAllA / kWaves, kLoadB = kAllB / kWaves;        // fragments a wavefront loads
  static_assert(kWaves == 8 && kAllA % kWaves == 0 && kAllB % kWaves == 0 && kFragA % 4 == 0, "");
  static_assert(kRowsA % 64 == 0 && kRowsB % 64 == 0 && kRowsA <= 256 && kRowsB <= 256, "one load for a stage's scales of an operand");
  static constexpr int kOffB = kAllA * 1024, kOffScaleA = kOffB + kAllB * 1024, kOffScaleB = kOffScaleA + 4 * kRowsA;
  static constexpr int kOffInit = kOffScaleB + 4 * kRowsB, kStage = kOffInit + (kInit ? 4 * kRowsA : 0);
  static constexpr int kStages = 3, kLds = kStages * kStage;

  mx_f32x4 acc[kFragA][kFragB];
  const char *smem;
  unsigned lds;                    // its LDS address
  int lane, wave, wa, wb, l16, q, blocks, steps;
  const uint8_t *src_a[kLoadA], *src_b[kLoadB];   // lane's block of step 0 of the fragments it loads
  const uint8_t *zero;

  // what the accumulators of A's rows start from, [ceil(rows / kRowsA) kRowsA] floats
  const float *init;
  Mx4Operand a, b;
  int64_t group_b;                 // first packed group of 64 of B's tile

  __device__ __forceinline__ void setup(const char *shared, const Mx4Operand &opa, const Mx4Operand &opb, const float *from, int nblocks,
                                        const void *zero16) {
    smem = shared;
    lds = (unsigned)(size_t)(mx4_lds_t)shared;
    lane = threadIdx.x & 63;
    wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    wa = wave / kWavesB;
    wb = wave % kWavesB;
    l16 = lane & 15;
    q = lane >> 4;
    a = opa; b = opb; init = from;
    blocks = nblocks;
    steps = (nblocks - 1) / 4 + 1;
    zero = static_cast<const uint8_t *>(zero16);
  }

  // B's tile from row row0 on; list: the rows' places in b.rows (its scales are packed in the order of the list), or null
  __device__ __forceinline__ void tile_b(int64_t row0, int64_t n, const int *list) {
#pragma unroll
    for (int u = 0; u < kLoadB; ++u) {
      int64_t r = row0 + 16 * (wave * kLoadB + u) + l16;
      if (r >= n) r = n - 1;
      if (list) r = list[r];
      src_b[u] = b.rows.codes + (r * blocks + q) * 16;
    }
    group_b = row0 / 64;
  }

  __device__ __forceinline__ void tile_a(int64_t tile) {
#pragma unroll
    for (int u = 0; u < kLoadA; ++u) {
      const int f = wave * kLoadA + u;
      int64_t r = tile * kRowsA + 64 * (f / 4) + mx4_dealt(f & 3, l16);
      if (r >= a.rows.n) r = a.rows.n - 1;
      src_a[u] = a.rows.codes + (r * blocks + q) * 16;
    }
  }

  // Loads of one step of A's tile `tile` (tile_a was called for it) into a stage.  Scales: wavefront 0 A's, 1 B's, 2 the starting values.
  // Groups of 64 rows past the operand's end are read from its last one.
  __device__ __forceinline__ void load(int stage, int64_t tile, int step) {
    const unsigned base = lds + stage * kStage;
    const bool in = 4 * step + q < blocks;
#pragma unroll
    for (int u = 0; u < kLoadA; ++u)
      load16_to_lds(in ? src_a[u] + 64 * step : zero, base + (wave * kLoadA + u) * 1024);
#pragma unroll
    for (int u = 0; u < kLoadB; ++u)
      load16_to_lds(in ? src_b[u] + 64 * step : zero, base + kOffB + (wave * kLoadB + u) * 1024);
    if (wave == 0) {
      if (lane < kRowsA / 4) {
        int64_t g = tile * (kRowsA / 64) + lane / 16;
        const int64_t last = (a.rows.n - 1) / 64;
        if (g > last) g = last;
        load16_to_lds(reinterpret_cast<const char *>(a.packed) + (g * steps + step) * 256 + (lane & 15) * 16, base + kOffScaleA);
      }
    } else if (wave == 1) {
      if (lane < kRowsB / 4) {
        int64_t g = group_b + lane / 16;
        const int64_t last = (b.rows.n - 1) / 64;
        if (g > last) g = last;
        load16_to_lds(reinterpret_cast<const char *>(b.packed) + (g * steps + step) * 256 + (lane & 15) * 16, base + kOffScaleB);
      }
    } else if (kInit && wave == 2) {
      if (lane < kRowsA / 4) load16_to_lds(init + tile * kRowsA + 4 * lane, base + kOffInit);
    }
  }
  // The loads of all steps but the last one issued are in LDS, for this wavefront's part.
  __device__ __forceinline__ void wait_one_left() {
    if (wave < 2 || (kInit && wave == 2)) mx4_wait<kLoadA + kLoadB + 1>();
    else mx4_wait<kLoadA + kLoadB>();
  }

  template <bool kFirst>
  __device__ __forceinline__ void multiply(int stage) {
    const char *base = smem + stage * kStage;
    i32x4 y[kFragB];
    int sy = *reinterpret_cast<const int *>(base + kOffScaleB + ((wb * kFragB) / 4) * 256 + lane * 4);
    if (kFragB < 4) sy >>= 8 * ((wb * kFragB) & 3);
#pragma unroll
    for (int v = 0; v < kFragB; ++v) y[v] = *reinterpret_cast<const i32x4 *>(base + kOffB + (wb * kFragB + v) * 1024 + lane * 16);
#pragma unroll
    for (int u = 0; u < kFragA; ++u) {
      const i32x4 x = *reinterpret_cast<const i32x4 *>(base + (wa * kFragA + u) * 1024 + lane * 16);
      const int sx = *reinterpret_cast<const int *>(base + kOffScaleA + (wa * (kFragA / 4) + u / 4) * 256 + lane * 4);
      mx_f32x4 from = {0.f, 0.f, 0.f, 0.f};
      if (kFirst && kInit) from = *reinterpret_cast<const mx_f32x4 *>(base + kOffInit + (64 * (wa * (kFragA / 4) + u / 4) + 16 * q + 4 * (u & 3)) * 4);
#pragma unroll
      for (int v = 0; v < kFragB; ++v) acc[u][v] = mx4_mfma_at(u & 3, v & 3, x, y[v], kFirst ? from : acc[u][v], sx, sy);
    }
  }

  // Tiles first .. last - 1 of A against B's tile; done(tile) after each.
  template <typename Done>
  __device__ __forceinline__ void run(int64_t first, int64_t last, Done done) {
    const int64_t total = (last - first) * steps;
    int64_t at = first;                    // tile and step of the next loads
    int step = 0;
    tile_a(at);
    auto next = [&](int stage) {
      load(stage, at, step);
      if (++step == steps) {
        step = 0;
        if (++at < last) tile_a(at);
      }
    };
    next(0);
    if (total > 1) next(1);
    int stage = 0;
    int64_t tile = first;
    int s = 0;
    for (int64_t it = 0; it < total; ++it) {
      if (it + 1 < total) wait_one_left(); else mx4_wait<0>();
      mx4_barrier();
      const int behind = stage == 0 ? 2 : stage - 1;      // (stage + 2) mod 3
      if (it + 2 < total) next(behind);
      if (s == 0) multiply<true>(stage); else multiply<false>(stage);
      if (++s == steps) {
        done(tile);
        ++tile;
        s = 0;
      }
      stage = stage == 2 ? 0 : stage + 1;
    }
    mx4_wait<0>();
    mx4_barrier();                         // the stages may be filled again
  }
};

// Words of packed scales: [ceil(n / 64)][steps][64]; lane l's byte t is that of block 4 step + l / 16 of row 64 g + 16 t + l % 16
// (kDealt: + mx4_dealt(t, l % 16)).
inline size_t mx4_packed_bytes(int64_t n, int blocks) { return (size_t)((n + 63) / 64) * ((blocks - 1) / 4 + 1) * 256; }
struct Mx4Unpacked {
  const uint8_t *scales;
  int64_t n;
  bool dealt;
  int *packed;
  const int *list, *count;         // or null: the rows that are meant, on the device how many (n of them at most)
};
hipError_t launch_mx4_pack_scales(hipStream_t stream, int blocks, Mx4Unpacked a, Mx4Unpacked b = {});

}  // namespace som
