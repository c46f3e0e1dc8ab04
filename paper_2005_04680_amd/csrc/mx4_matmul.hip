// Scores of all rows of a 4-bit microscaled table: out = q(x) W^T.
//
// Both sides are blocks of 32 codes with a power of two, which the scaled matrix instructions
// take as they are: the products are exact and the sums FP32.  Three ways, by the rows of x: up to 16
// stream W straight into the products (bound by W's bytes), more go through LDS in
// tiles.  4096 x 65536 x 4096, BF16 in and out: 611 us, 3.6 PFLOP/s, of which 18 us round x and
// copy W's scales; the same instructions from registers reach 5.7 PFLOP/s on such data (8.7 on
// zeros: the clock falls with the bits that toggle, to 1.9 GHz on average here), a BF16 library
// product of these sizes takes 1548 us.  With k = 256 the output's bytes bound it (145 us for 537 MB).
// Outputs whose rows do not begin at 128-byte lines are slower there: 2889 x 89088 x 64 into BF16 110
// us, 2889 x 89061 178; the L2s' write requests grow by half.
//
// x may come as 8-bit rows instead (E4M3 codes, twice the bytes): the same kernels with X8.  Products
// of an 8-bit and a 4-bit side run at the 8-bit rate, half the 4-bit one, but the scaled instructions
// add eight products at a time, aligned to the largest of them, and drop what lies more than 13 bits below
// it (measured).  4-bit sides have no such bits; an 8-bit side does: sums over a norm's rows are off by 3e-6 of
// themselves, far below a BF16 output's rounding.  Into FP32 the values of both sides, which BF16 holds
// exactly, go through the BF16 instructions.  4096 x 65536 x 4096 into BF16: 836 us, 2.6 PFLOP/s (4-bit rows
// 611), as those bound by the products with their LDS reads, now of twice the bytes, and the stores.
#include <type_traits>

#include "head.hpp"

namespace embbag {
namespace {

typedef int i8v __attribute__((ext_vector_type(8)));
typedef float f16v __attribute__((ext_vector_type(16)));
typedef u4 u4_word __attribute__((aligned(4)));

// A fragment of 32 codes as the products take it.
__device__ __forceinline__ i8v frag8(const u4& v) {
  return i8v{int(v.x), int(v.y), int(v.z), int(v.w), 0, 0, 0, 0};
}
// One of 32 8-bit codes: of a product's elements in order, 16 bytes per lane group of its first half,
// then of its second.
struct Bytes32 {
  u4 lo, hi;
};
__device__ __forceinline__ i8v frag8(const Bytes32& v) {
  return i8v{int(v.lo.x), int(v.lo.y), int(v.lo.z), int(v.lo.w),
             int(v.hi.x), int(v.hi.y), int(v.hi.z), int(v.hi.w)};
}
// The side of x: 8-bit rows (X8) or codes of 4 bits.
template <bool X8>
using XFrag = std::conditional_t<X8, Bytes32, u4>;
template <bool X8>
constexpr int kXFormat = X8 ? 0 : 4;  // E4M3, E2M1
template <bool X8>
constexpr int kXRow = X8 ? 128 : 64;  // bytes of a row per step

constexpr int kGroup = 128;      // elements of a step: 4 blocks, whose scales are one word
constexpr int kGroupBytes = 64;  // their codes
constexpr int kPad = 256;        // rows of scales are padded to the largest tile
constexpr size_t kLdsPerCu = 160 * 1024;

// The codes of 8 elements of a row from e0 on (zeros past k) and their block's scale byte; four
// neighbouring lanes hold a block, as in mx4_quantize.
template <class T>
__device__ __forceinline__ uint32_t quantize8(const T* row, int e0, int k, uint32_t* byte) {
  const f4 zero = {0.f, 0.f, 0.f, 0.f};
  const f4 x0 = e0 < k ? load4(row + e0) : zero;
  const f4 x1 = e0 + 4 < k ? load4(row + e0 + 4) : zero;
  float y[8] = {x0.x, x0.y, x0.z, x0.w, x1.x, x1.y, x1.z, x1.w};
  uint32_t amax = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) amax = max(amax, __float_as_uint(y[i]) & 0x7FFFFFFFu);
  amax = max(amax, uint32_t(__shfl_xor(int(amax), 1, 4)));
  amax = max(amax, uint32_t(__shfl_xor(int(amax), 2, 4)));
  float factor;
  *byte = mx4_scale_of(amax, &factor);
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] *= factor;
  return *byte == 255u ? 0u : mx4_codes8(y);
}

// Whether the products run on BF16 values of both sides.
template <bool X8, class T>
constexpr bool kExact = X8 && sizeof(T) == 4;

// Values of 32 codes, in order, as the operands of four BF16 products.
__device__ __forceinline__ void bf16_values(const u4& c, uint32_t scale, u4 (&v)[4]) {
  const float s = mx4_scale(scale);
#pragma unroll
  for (int t = 0; t < 4; ++t)
    v[t] = u4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c[t], s, 0)),
              __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c[t], s, 1)),
              __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c[t], s, 2)),
              __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c[t], s, 3))};
}
__device__ __forceinline__ void bf16_values(const Bytes32& c, uint32_t scale, u4 (&v)[4]) {
  const float s = mx4_scale(scale);
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    const u4& q = t < 2 ? c.lo : c.hi;
    const uint32_t a = q[t % 2 * 2], b = q[t % 2 * 2 + 1];
    v[t] = u4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, s, false)),
              __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, s, true)),
              __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, s, false)),
              __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, s, true))};
  }
}

// Block number `block` of a copy of scales [rows][G] to words [G][pitch]: 64 rows, a quarter of the
// groups for each wavefront, 4 groups at a time.
__device__ __forceinline__ void copy_scales(uint32_t block, const uint32_t* __restrict__ scales,
                                            int64_t rows, int G, uint32_t* __restrict__ out,
                                            int64_t pitch) {
  const int64_t row = int64_t(block) * kWave + lane_id();
  if (row >= rows) return;
  const uint32_t* src = scales + row * G;
  for (int g = wave_id() * 4; g < G; g += kWavesPerBlock * 4) {
    uint32_t v[4];
    if (G % 4 == 0) {
      const u4 q = *reinterpret_cast<const u4_word*>(src + g);
      v[0] = q.x, v[1] = q.y, v[2] = q.z, v[3] = q.w;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = g + i < G ? src[g + i] : 0u;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (g + i < G) out[(g + i) * pitch + row] = v[i];
  }
}

// x rounded to the storage of the table: codes [m][groups * 64] (zeros past k), scales as words of
// 4 blocks [groups][xpitch].  Four lanes per block, as mx4_quantize.  Blocks from `xblocks` on
// copy W's scales to words [groups][wpitch].  The launch begins with block `first`.
template <class T>
__global__ __launch_bounds__(kBlock) void pack_x(const T* __restrict__ x, int64_t stride, int32_t m,
                                                 int32_t k, FastDiv groups,
                                                 uint8_t* __restrict__ codes,
                                                 uint8_t* __restrict__ scales, int64_t xpitch,
                                                 uint32_t xblocks, const uint32_t* __restrict__ ws,
                                                 int64_t n, uint32_t* __restrict__ ws_out,
                                                 int64_t wpitch, uint32_t first) {
  const int G = int(groups.div);
  const uint32_t block = first + blockIdx.x;
  if (block >= xblocks) {
    copy_scales(block - xblocks, ws, n, G, ws_out, wpitch);
    return;
  }
  const int64_t u = int64_t(block) * (kBlock / 4) + threadIdx.x / 4;
  const int part = threadIdx.x % 4;
  const int64_t g4 = u / 4;
  if (g4 >= int64_t(m) * G) return;
  const uint32_t row = quotient(uint32_t(g4), groups);
  const int g = int(uint32_t(g4) - row * groups.div), j = int(u % 4);
  uint32_t byte;
  const uint32_t c = quantize8(x + int64_t(row) * stride, g * kGroup + j * kMxBlock + part * 8, k, &byte);
  *reinterpret_cast<uint32_t*>(codes + (int64_t(row) * G + g) * kGroupBytes + j * 16 + part * 4) = c;
  if (part == 0) scales[(int64_t(g) * xpitch + row) * 4 + j] = uint8_t(byte);
}

// The scales of 8-bit rows, and from block `xblocks` on W's, to words of 4 blocks [groups][pitch].
__global__ __launch_bounds__(kBlock) void pack_scales(const uint32_t* __restrict__ xs, int64_t m,
                                                      uint32_t* __restrict__ xs_out, int64_t xpitch,
                                                      uint32_t xblocks, const uint32_t* __restrict__ ws,
                                                      int64_t n, uint32_t* __restrict__ ws_out,
                                                      int64_t wpitch, int G, uint32_t first) {
  const uint32_t block = first + blockIdx.x;
  if (block < xblocks)
    copy_scales(block, xs, m, G, xs_out, xpitch);
  else
    copy_scales(block - xblocks, ws, n, G, ws_out, wpitch);
}

// 16 or 4 bytes per lane from memory to LDS, lane l's at `dst` + 16 l (4 l).
typedef const __attribute__((address_space(1))) void* GlobalPtr;
typedef __attribute__((address_space(3))) void* LdsPtr;
__device__ __forceinline__ void to_lds16(const void* src, void* dst) {
  __builtin_amdgcn_global_load_lds((GlobalPtr)src, (LdsPtr)dst, 16, 0, 0);
}
__device__ __forceinline__ void to_lds4(const void* src, void* dst) {
  __builtin_amdgcn_global_load_lds((GlobalPtr)src, (LdsPtr)dst, 4, 0, 0);
}

// Until at most N of this wavefront's loads are on their way, its LDS reads complete.
template <int N>
__device__ __forceinline__ void wait_loads() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N) : "memory");
}

// The block's barrier alone: unlike __syncthreads it leaves loads to LDS on their way.  No memory
// access moves across it.
__device__ __forceinline__ void block_barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// Tiles of 32 rows of W that a wavefront turns around at once: 256 bytes of a row of the output where
// it has four of them, 128 else.
template <class T>
constexpr int turn_tiles(int tn) {
  const int most = (tn < 4 ? 4 : 8) / int(sizeof(T));
  return tn < most ? tn : most;
}

// Tile number id: strips of `width` m tiles, in a strip n tile after n tile.  An XCD's blocks then
// hold `width` tiles of x at a time and neighbouring rows of W, whose stores meet in whole lines of
// the output.  Measured, us, width 1 / 2 / 8 / 32: 4096 x 65536 x 4096 628 / 611 / 630 / 671, x 512
// 176 / 202 / 191 / 212, 4096 x 65537 x 1024 269 / 290 / 286 / 305; smaller tiles, 500 x 50001 x 1024
// 40 / - / 34, 2000 x 20000 x 1024 53 / - / 49.
__device__ __forceinline__ void tile_of(uint32_t id, uint32_t mtiles, uint32_t ntiles,
                                        uint32_t strip_width, uint32_t* mt, uint32_t* nt) {
  const uint32_t strip = id / (strip_width * ntiles);
  const uint32_t m0 = strip * strip_width, width = min(strip_width, mtiles - m0);
  const uint32_t in = id - m0 * ntiles;
  *nt = in / width;
  *mt = m0 + in - *nt * width;
}

// A BN x BM tile of out^T (BN rows of W, BM of x); WN x WM wavefronts, each TN x TM
// products of 32 x 32.
//
// Per step of 128 elements the tile's codes and scales go from memory to LDS, STAGES of them in
// turn: the loads of a step are issued STAGES - 1 steps ahead.  A wavefront's load brings 16 rows of
// 64 bytes; the lane of row r and place j fetches block j ^ (r / 4 % 4), so that the fragments'
// reads (16 rows, one block) cover all banks.  Lane l's row is l % 32; product j of a step
// takes block 2 (l / 32) + j, whose scale is byte j of the row's word, shifted by l / 32
// halves.
//
// A block takes tile after tile (every XCD its own range of them), and the loads run through the
// steps of all of them: those of the next tile are on their way while a tile is stored.
//
// 256 x 256 tiles keep the accumulators of a wavefront in 256 registers and read each fragment
// from LDS for four products.  Left out one at a time at 4096 x 65536 x 4096 with both sides in 4 bits (633 us with
// strips of 8): loads to LDS 457, stores of the output 533, LDS reads and loads and stores 315.
//
// 8-bit rows (X8): a load brings 8 rows of 128 bytes, place j of row r holds chunk j ^ (r % 8); a
// fragment is two chunks, 16 elements of the product's first block and 16 of its second.
template <bool X8, int TN, int TM, int WN, int WM, int STAGES, class T>
__global__ __launch_bounds__(WN* WM* kWave, 1) void scores_tile(
    const uint8_t* __restrict__ xc, const uint32_t* __restrict__ xs, int64_t xpitch, int32_t m,
    int32_t steps, Mx4View w, const uint32_t* __restrict__ ws, int64_t wpitch, uint32_t mtiles,
    uint32_t ntiles, T* __restrict__ out, int64_t ldo) {
  constexpr int BN = 32 * TN * WN, BM = 32 * TM * WM, W = WN * WM;
  constexpr int XROW = kXRow<X8>, XROWS = 1024 / XROW;  // bytes per row, rows per load of x
  constexpr int LOADS = (BN / 16 + BM / XROWS) / W;     // codes, per wavefront and step
  constexpr int SALL = (BN + BM) / 64;        // of scales, in the block
  constexpr int SLOADS = (SALL + W - 1) / W;  // per wavefront (the last ones may come twice)
  static_assert(BN % (16 * W) == 0 && BM % (XROWS * W) == 0 && BN % 64 == 0, "whole loads");
  constexpr int WLOADS = BN / 16 / W;         // codes of W's rows, which come first
  constexpr int CODES = BN * kGroupBytes + BM * XROW;
  constexpr int STAGE = CODES + (BN + BM) * 4;
  constexpr int V = kVec<T>;
  constexpr int TILES = turn_tiles<T>(TN), PITCH = 32 * TILES + V;
  constexpr int PER_ROW = 32 * TILES / V, ROWS = kWave / PER_ROW, STORES = 32 / ROWS;
  extern __shared__ __align__(16) uint8_t lds[];

  const int lane = lane_id(), wave = wave_id();
  T* turn = reinterpret_cast<T*>(lds + STAGES * STAGE) + wave * 32 * PITCH;
  const int nb = mx4_blocks(w.dim);
  const int64_t xrow = int64_t(steps) * XROW, wrow = int64_t(nb) * 16;
  // This block's tiles: from `tile` on every `stride`-th below `end`.
  const uint32_t tiles = mtiles * ntiles, range = (tiles + kNumXcd - 1) / kNumXcd;
  const uint32_t stride = gridDim.x / kNumXcd;
  const uint32_t end = min((blockIdx.x % kNumXcd + 1) * range, tiles);
  uint32_t tile = blockIdx.x % kNumXcd * range + blockIdx.x / kNumXcd;
  if (tile >= end) return;
  const uint32_t strip_width = BM < 256 ? 8 : (steps > 16 ? 2 : 1);

  // The loads' own place in the stream of steps: number i of this wavefront brings rows
  // 16 * (i * W + wave) .. + 15 of the stage (W's rows, then x's); rows past the end repeat
  // the last one.
  const int c = (lane % 4) ^ (lane / 16);
  const int cx8 = (lane % 8) ^ (lane / 8);
  uint32_t ltile = tile;
  int lstep = 0;
  const uint8_t *wbase, *xbase;
  const uint32_t* sbase[SLOADS];  // scales' loads, each at its place in the tile's rows
  uint32_t off[LOADS];
  // Whether a load of scales is of W's rows: known from its number where sides are whole rounds of the
  // wavefronts.
  auto of_w = [&](int i) {
    if constexpr (BN % (64 * W) == 0 && BM % (64 * W) == 0) return i < BN / 64 / W;
    return (i * W + wave) % SALL < BN / 64;
  };
  auto load_tile = [&]() {
    uint32_t mt, nt;
    tile_of(ltile, mtiles, ntiles, strip_width, &mt, &nt);
    const int64_t n0 = int64_t(nt) * BN;
    const int m0 = int(mt) * BM;
    wbase = w.codes + n0 * wrow;
    xbase = xc + int64_t(m0) * xrow;
#pragma unroll
    for (int i = 0; i < SLOADS; ++i) {
      const int r0 = 64 * ((i * W + wave) % SALL);
      sbase[i] = of_w(i) ? ws + n0 + r0 + lane : xs + m0 + (r0 - BN) + lane;
    }
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      if (i < WLOADS) {
        const int r = 16 * (i * W + wave) + lane / 4;
        off[i] = uint32_t(min(int64_t(r), w.rows - 1 - n0) * wrow);
      } else {
        const int r = XROWS * ((i - WLOADS) * W + wave) + lane / (64 / XROWS);
        off[i] = uint32_t(min(r, m - 1 - m0) * xrow + (X8 ? cx8 : c) * 16);
      }
    }
  };
  // Before a step's loads.  After the last tile its steps are loaded again, so that the number
  // of loads on their way is always the same.
  auto next_load = [&]() {
    if (lstep == steps) {
      lstep = 0;
      if (ltile + stride < end) {
        ltile += stride;
        load_tile();
      }
    }
  };
  load_tile();
  // Load number i of a step (the codes', then the scales').
  constexpr int PER = LOADS + SLOADS;
  auto load = [&](uint8_t* dst, int i) {
    if (i < LOADS) {
      // (A block past W's row is its last one: x's codes are 0 there, and W's scale.)
      const uint32_t wk = uint32_t(min(lstep * 4 + c, nb - 1)) * 16;
      const uint32_t xk = uint32_t(lstep) * XROW;
      to_lds16(i < WLOADS ? wbase + (off[i] + wk) : xbase + (off[i] + xk),
               dst + (i < WLOADS ? (i * W + wave) * 1024
                                 : BN * kGroupBytes + ((i - WLOADS) * W + wave) * 1024));
    } else {
      const int r0 = 64 * (((i - LOADS) * W + wave) % SALL);
      to_lds4(sbase[i - LOADS] + lstep * (of_w(i - LOADS) ? wpitch : xpitch), dst + CODES + r0 * 4);
    }
  };

  const int wn = wave % WN, wm = wave / WN;
  const int half = lane / 32, row = lane % 32;
  f16v acc[TN][TM];
  const int frag_w = (wn * TN * 32 + row) * kGroupBytes;
  const int frag_x = BN * kGroupBytes + (wm * TM * 32 + row) * XROW;
  const int scale_w = CODES + (wn * TN * 32 + row) * 4;
  const int scale_x = CODES + (BN + wm * TM * 32 + row) * 4;
  const int at0 = ((2 * half) ^ (row / 4 % 4)) * 16;  // place of part j's block: at0 ^ (16 j)
  // Of 8-bit rows: part j's two chunks.  The scaled products take half `half` of blocks j and 2 + j,
  // the BF16 ones both halves of W's block 2 * half + j.
  constexpr bool EXACT = kExact<X8, T>;
  constexpr int HI8 = EXACT ? 16 : 64;
  const int at8 = ((EXACT ? 4 * half : half) ^ (row & 7)) * 16;
  u4 xv[EXACT ? TM : 1][4];
  u4 a[2][TN] = {};
  XFrag<X8> b[2][TM] = {};
  uint32_t cw[TN] = {}, cx[TM] = {}, nw[TN], nx[TM];  // scales of this step and the next
  // Everything is issued between the products, a few instructions after every row of TM of them,
  // which a wavefront's in-order issue would otherwise put in front of them: the reads of the
  // next part's fragments (a step's first part is read during the last part of the step
  // before) and the loads of a later step.  Those go to `nxt`, not the memory of `cur`: the
  // reads need not wait for them.
  auto fetch = [&](const uint8_t* __restrict__ cur, int j, int i) {
    if (i < TM) {
      const uint8_t* p = cur + frag_x + i * 32 * XROW;
      if constexpr (X8) {
        b[j][i].lo = *reinterpret_cast<const u4*>(p + (at8 ^ (32 * j)));
        b[j][i].hi = *reinterpret_cast<const u4*>(p + (at8 ^ (32 * j) ^ HI8));
      } else {
        b[j][i] = *reinterpret_cast<const u4*>(p + (at0 ^ (16 * j)));
      }
    } else {
      a[j][i - TM] =
          *reinterpret_cast<const u4*>(cur + frag_w + (i - TM) * 32 * kGroupBytes + (at0 ^ (16 * j)));
    }
  };
  auto fetch_scale = [&](const uint8_t* __restrict__ cur, int i) {
    if (i < TM)
      nx[i] = *reinterpret_cast<const uint32_t*>(cur + scale_x + i * 128);
    else
      nw[i - TM] = *reinterpret_cast<const uint32_t*>(cur + scale_w + (i - TM) * 128);
  };
  // (The scales' bytes are chosen in the instruction: a constant each.)
#define EMB_ROW(J, I)                                                                          \
  if constexpr (EXACT) {                                                                       \
    u4 wv[4];                                                                                  \
    if (I == 0) {                                                                              \
      _Pragma("unroll") for (int j = 0; j < TM; ++j)                                           \
          bf16_values(b[J][j], cx[j] >> (8 * J) & 255u, xv[j]);                                \
    }                                                                                          \
    bf16_values(a[J][I], cw[I] >> (8 * J) & 255u, wv);                                         \
    _Pragma("unroll") for (int t = 0; t < 4; ++t) {                                            \
      _Pragma("unroll") for (int j = 0; j < TM; ++j) acc[I][j] =                               \
          __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf8, wv[t]),              \
                                                  __builtin_bit_cast(bf8, xv[j][t]), acc[I][j], \
                                                  0, 0, 0);                                    \
    }                                                                                          \
  } else {                                                                                     \
    _Pragma("unroll") for (int j = 0; j < TM; ++j) acc[I][j] =                                 \
        __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(frag8(a[J][I]), frag8(b[J][j]),        \
                                                        acc[I][j], 4, kXFormat<X8>, J,         \
                                                        int(cw[I]), J, int(cx[j]));            \
  }                                                                                            \
  __builtin_amdgcn_sched_barrier(0);
  auto step_of = [&](const uint8_t* __restrict__ cur, uint8_t* __restrict__ nxt) {
    constexpr int N = TN + TM;  // fragments of a part, read before its last row's products
    constexpr int READS = TN > 1 ? TN - 1 : 1;
#pragma unroll
    for (int i = 0; i < TN; ++i) {
      EMB_ROW(1, i)
#pragma unroll
      for (int r = 0; r < N; ++r)
        if (r * READS / N == i) fetch(cur, 0, r), fetch_scale(cur, r);
#pragma unroll
      for (int l = 0; l < PER; ++l)
        if (l * 2 * TN / PER == i) load(nxt, l);
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int i = 0; i < TN; ++i) cw[i] = nw[i] >> (16 * half);
#pragma unroll
    for (int i = 0; i < TM; ++i) cx[i] = nx[i] >> (16 * half);
#pragma unroll
    for (int i = 0; i < TN; ++i) {
      EMB_ROW(0, i)
#pragma unroll
      for (int r = 0; r < N; ++r)
        if (r * READS / N == i) fetch(cur, 1, r);
#pragma unroll
      for (int l = 0; l < PER; ++l)
        if (l * 2 * TN / PER == TN + i) load(nxt, l);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
#pragma unroll
  for (int i = 0; i < STAGES - 1; ++i) {
    next_load();
#pragma unroll
    for (int l = 0; l < PER; ++l) load(lds + i * STAGE, l);
    ++lstep;
  }
  int cur = 0;
  for (;; tile += stride) {
#pragma unroll
  for (int i = 0; i < TN; ++i)
#pragma unroll
    for (int j = 0; j < TM; ++j) acc[i][j] = f16v{};
  for (int step = 0; step < steps; ++step) {
    next_load();
    // This step's codes are in LDS (those of the next STAGES - 2 may be on their way), and every
    // wavefront holds the last fragments of the stage before, which the next load overwrites.
    wait_loads<(STAGES - 2) * PER>();
    block_barrier();
    const int free = cur == 0 ? STAGES - 1 : cur - 1;
    step_of(lds + cur * STAGE, lds + free * STAGE);
    ++lstep;
    cur = cur == STAGES - 1 ? 0 : cur + 1;
  }
#pragma unroll
  for (int i = 0; i < TN; ++i) {
    EMB_ROW(1, i)
  }
#undef EMB_ROW

  // The next tile's first products take no fragments, and no scale: the byte 255 makes NaN of zeros
  // too, and that of a bad block, or of a row past the end, would stay in the new tile's sums.
#pragma unroll
  for (int i = 0; i < TN; ++i) a[1][i] = u4{0u, 0u, 0u, 0u}, cw[i] = 0u;
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    cx[i] = 0u;
    if constexpr (X8) b[1][i] = {};  // (8-bit codes have a NaN of their own)
  }

  // Each wavefront turns 32 rows of x and 32 * TILES of W at a time around in its own part of LDS
  // (lane: row of x lane % 32, four consecutive rows of W per quarter of its registers), then
  // stores rows of 128 or 256 bytes.
  uint32_t mt, nt;
  tile_of(tile, mtiles, ntiles, strip_width, &mt, &nt);
  const int64_t n1 = int64_t(nt) * BN + wn * TN * 32;
  const int m1 = int(mt) * BM + wm * TM * 32;
  const int col = lane % PER_ROW * V;
  const bool whole = int64_t(nt) * BN + BN <= w.rows;  // whole rows of the tile
#pragma unroll
  for (int j = 0; j < TM; ++j) {
#pragma unroll
    for (int h = 0; h < TN; h += TILES) {
#pragma unroll
      for (int i = 0; i < TILES; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          store4(turn + row * PITCH + i * 32 + q * 8 + half * 4,
                 f4{acc[h + i][j][q * 4], acc[h + i][j][q * 4 + 1], acc[h + i][j][q * 4 + 2],
                    acc[h + i][j][q * 4 + 3]});
      const int64_t n2 = n1 + h * 32 + col;
      const int m2 = m1 + j * 32 + lane / PER_ROW;
      T* p = out + int64_t(m2) * ldo + n2;
      const T* q = turn + lane / PER_ROW * PITCH + col;
      if (whole) {
        u4 v[STORES];
#pragma unroll
        for (int r = 0; r < STORES; ++r) v[r] = *reinterpret_cast<const u4*>(q + r * ROWS * PITCH);
#pragma unroll
        for (int r = 0; r < STORES; ++r)
          if (m2 + r * ROWS < m) store16(p + int64_t(r * ROWS) * ldo, v[r]);
      } else {
#pragma unroll 1
        for (int r = 0; r < STORES && m2 + r * ROWS < m; ++r) {
#pragma unroll 1
          for (int e = 0; e < V && n2 + e < w.rows; ++e)
            p[int64_t(r * ROWS) * ldo + e] = q[r * ROWS * PITCH + e];
        }
      }
    }
  }
  if (tile + stride >= end) break;
  }
  // No load to LDS outlives the block.
  wait_loads<0>();
}

// One wavefront per 16 rows of W and up to 16 of x, W straight from memory: lane l holds
// row l % 16, and of every 4 groups of 128 elements the group l / 16; the four blocks
// of its group go through four products whose scales are the bytes of one word.  Few elements of x
// (kFused) are rounded by every block for itself, others by pack_x before.  One row of x, 200003 x
// 1024: 21 us, 5.2 TB/s; bound by W.  The launch begins with block `first`.
constexpr int kFused = 8192;  // elements of x, rows padded to groups

template <class TX, class T, bool FUSED>
__global__ __launch_bounds__(kBlock) void scores_direct(const TX* __restrict__ x, int64_t stride,
                                                        const uint8_t* __restrict__ xc,
                                                        const uint32_t* __restrict__ xs,
                                                        int64_t xpitch, Mx4View w, int32_t m,
                                                        int32_t groups, T* __restrict__ out,
                                                        int64_t ldo, uint32_t first) {
  __shared__ __align__(16) uint8_t codes[FUSED ? kFused / 2 : 16];
  __shared__ __align__(16) uint8_t scales[FUSED ? kFused / kMxBlock : 16];
  const int lane = lane_id(), r = lane % 16, q = lane / 16;
  const int64_t n0 = ((int64_t(first) + blockIdx.x) * kWavesPerBlock + wave_id()) * 16;
  const int nb = mx4_blocks(w.dim);
  const int64_t wn = min(n0 + r, w.rows - 1);
  const int xm = min(r, m - 1);
  const uint8_t* wc = w.codes + wn * nb * 16;
  const uint32_t* wsc = reinterpret_cast<const uint32_t*>(w.scales) + wn * groups;

  u4 b[4];
  uint32_t sw;
  auto load_w = [&](int g) {
    sw = g < groups ? wsc[g] : 0u;
#pragma unroll
    for (int j = 0; j < 4; ++j)
      b[j] = g * 4 + j < nb ? *reinterpret_cast<const u4*>(wc + (g * 4 + j) * 16)
                            : u4{0u, 0u, 0u, 0u};
  };
  load_w(q);
  if constexpr (FUSED) {
    const int units = m * groups * 4;
    for (int u = threadIdx.x / 4; u < units; u += kBlock / 4) {
      const int row = u / (groups * 4), block = u - row * groups * 4;
      uint32_t byte;
      const uint32_t c = quantize8(x + row * stride, block * kMxBlock + int(threadIdx.x % 4) * 8, w.dim, &byte);
      *reinterpret_cast<uint32_t*>(codes + u * 16 + threadIdx.x % 4 * 4) = c;
      if (threadIdx.x % 4 == 0) scales[u] = uint8_t(byte);
    }
    __syncthreads();
  }
  f4 c = {0.f, 0.f, 0.f, 0.f};
  for (int g0 = 0; g0 < groups; g0 += 4) {
    const int g = g0 + q;
    const bool in = g < groups;
    uint32_t sx = 0u;
    u4 a[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) a[j] = u4{0u, 0u, 0u, 0u};
    if (in) {
      const int64_t at = int64_t(xm) * groups + g;
      sx = FUSED ? *reinterpret_cast<const uint32_t*>(scales + at * 4) : xs[g * xpitch + xm];
#pragma unroll
      for (int j = 0; j < 4; ++j)
        a[j] = FUSED ? *reinterpret_cast<const u4*>(codes + at * kGroupBytes + j * 16)
                     : *reinterpret_cast<const u4*>(xc + at * kGroupBytes + j * 16);
    }
    const u4 v[4] = {b[0], b[1], b[2], b[3]};
    const uint32_t sv = sw;
    if (g0 + 4 < groups) load_w(g + 4);
#define EMB_MFMA(J)                                                                          \
  c = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(frag8(a[J]), frag8(v[J]), c, 4, 4, J, \
                                                       int(sx), J, int(sv));
    EMB_MFMA(0)
    EMB_MFMA(1)
    EMB_MFMA(2)
    EMB_MFMA(3)
#undef EMB_MFMA
  }
  const int64_t n = n0 + r;
  if (n >= w.rows) return;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int mm = q * 4 + i;
    if (mm < m) out[int64_t(mm) * ldo + n] = T(c[i]);
  }
}

// The same from 8-bit rows, which every block copies to LDS first where they are few (kStaged bytes; rows
// 16 bytes further apart, so that 16 of them do not share banks), else read in place.  Into BF16, of product
// j's four blocks (one of each group) lane group q takes half q % 2 of the first or second (q / 2) and of
// the third or fourth, and gives the scale of block q; into FP32 it takes block q of x as of W.  1 x 200003 x
// 1024 into FP32: 20 us, 5.4 TB/s of W's 109 MB; 24 with x from memory.
constexpr int kStaged = 16384;

template <class T, bool STAGED>
__global__ __launch_bounds__(kBlock) void scores8_direct(const uint8_t* __restrict__ xc,
                                                         const uint32_t* __restrict__ xs, Mx4View w,
                                                         int32_t m, int32_t groups,
                                                         T* __restrict__ out, int64_t ldo,
                                                         uint32_t first) {
  const int lane = lane_id(), r = lane % 16, q = lane / 16;
  const int64_t n0 = ((int64_t(first) + blockIdx.x) * kWavesPerBlock + wave_id()) * 16;
  const int nb = mx4_blocks(w.dim);
  const int64_t wn = min(n0 + r, w.rows - 1);
  const int xm = min(r, m - 1);
  const uint8_t* wc = w.codes + wn * nb * 16;
  const uint32_t* wsc = reinterpret_cast<const uint32_t*>(w.scales) + wn * groups;
  constexpr bool EXACT = kExact<true, T>;
  __shared__ __align__(16) uint8_t rows[STAGED ? kStaged + 16 * 16 : 16];
  const int pitch = STAGED ? groups * 128 + 16 : groups * 128;
  const uint8_t* xr = (STAGED ? rows : xc) + int64_t(xm) * pitch + (EXACT ? 0 : q % 2 * 16);
  const uint32_t* xsc = xs + int64_t(xm) * groups;

  const u4 none = {0u, 0u, 0u, 0u};
  u4 b[4];
  Bytes32 a[4];
  uint32_t sw, sx;
  auto load_w = [&](int g0) {
    const int g = g0 + q;
    sw = g < groups ? wsc[g] : 0u;
    sx = g < groups ? xsc[g] : 0u;
#pragma unroll
    for (int j = 0; j < 4; ++j)
      b[j] = g * 4 + j < nb ? *reinterpret_cast<const u4*>(wc + (g * 4 + j) * 16) : none;
  };
  auto load_x = [&](int g0) {
    const int g = g0 + q, ga = EXACT ? g : g0 + q / 2, gb = EXACT ? g : ga + 2;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      a[j].lo = ga < groups ? *reinterpret_cast<const u4*>(xr + ga * 128 + j * 32) : none;
      a[j].hi = gb < groups ? *reinterpret_cast<const u4*>(xr + gb * 128 + j * 32 + (EXACT ? 16 : 0)) : none;
    }
  };
  load_w(0);
  if constexpr (STAGED) {
    const int per = groups * 8;  // of 16 bytes, of a row
    for (int i = threadIdx.x; i < m * per; i += kBlock)
      *reinterpret_cast<u4*>(rows + i / per * pitch + i % per * 16) = reinterpret_cast<const u4*>(xc)[i];
    __syncthreads();
  } else {
    load_x(0);
  }
  f4 c = {0.f, 0.f, 0.f, 0.f};
  for (int g0 = 0; g0 < groups; g0 += 4) {
    if (STAGED) load_x(g0);
    const u4 v[4] = {b[0], b[1], b[2], b[3]};
    const Bytes32 u[4] = {a[0], a[1], a[2], a[3]};
    const uint32_t tw = sw, tx = sx;
    if (g0 + 4 < groups) {
      load_w(g0 + 4);
      if (!STAGED) load_x(g0 + 4);
    }
    if constexpr (EXACT) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        u4 xv[4], wv[4];
        bf16_values(u[j], tx >> (8 * j) & 255u, xv);
        bf16_values(v[j], tw >> (8 * j) & 255u, wv);
#pragma unroll
        for (int t = 0; t < 4; ++t)
          c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf8, xv[t]),
                                                      __builtin_bit_cast(bf8, wv[t]), c, 0, 0, 0);
      }
    } else {
#define EMB_MFMA(J)                                                                            \
  c = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(frag8(u[J]), frag8(v[J]), c, 0, 4, J,   \
                                                       int(tx), J, int(tw));
      EMB_MFMA(0)
      EMB_MFMA(1)
      EMB_MFMA(2)
      EMB_MFMA(3)
#undef EMB_MFMA
    }
  }
  const int64_t n = n0 + r;
  if (n >= w.rows) return;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int mm = q * 4 + i;
    if (mm < m) out[int64_t(mm) * ldo + n] = T(c[i]);
  }
}

size_t align256(size_t x) { return (x + 255) / 256 * 256; }

}  // namespace

namespace {

int64_t padded(int64_t rows) { return (rows + kPad - 1) / kPad * kPad; }

// x's codes and scales, W's scales, in the workspace.
struct ScoreLayout {
  size_t xs, ws, total;
};
// Whether every block rounds x for itself.
bool fused(int32_t m, int32_t k) { return m <= 16 && m * ((k + kGroup - 1) / kGroup) * kGroup <= kFused; }

ScoreLayout score_layout(int32_t m, int64_t n, int32_t k) {
  if (fused(m, k)) return {0, 0, 0};
  const size_t groups = size_t((k + kGroup - 1) / kGroup);
  ScoreLayout L;
  L.xs = align256(size_t(m) * groups * kGroupBytes);
  L.ws = L.xs + size_t(padded(m)) * groups * 4;
  L.total = L.ws + (m > 16 ? size_t(padded(n)) * groups * 4 : 0);
  return L;
}

template <bool X8, int TN, int TM, int WN, int WM, int STAGES, int RESIDENT, class T>
void launch_tile(const uint8_t* xc, const uint32_t* xs, int32_t m, int32_t groups,
                 const Mx4View& w, const uint32_t* ws, T* out, int64_t ldo, hipStream_t st) {
  constexpr int BN = 32 * TN * WN, BM = 32 * TM * WM;
  static_assert(kPad % BN == 0 && kPad % BM == 0, "padded scales");
  constexpr size_t stage = size_t(BN) * (kGroupBytes + 4) + size_t(BM) * (kXRow<X8> + 4);
  constexpr size_t turn = size_t(WN) * WM * 32 * (32 * turn_tiles<T>(TN) + kVec<T>)*sizeof(T);
  constexpr size_t lds = STAGES * stage + turn;
  static_assert(lds <= kLdsPerCu / RESIDENT, "blocks that share a compute unit");
  const uint32_t mtiles = uint32_t((m + BM - 1) / BM);
  const uint32_t ntiles = uint32_t((w.rows + BN - 1) / BN);
  auto kernel = scores_tile<X8, TN, TM, WN, WM, STAGES, T>;
  if (lds > 65536)
    (void)hipFuncSetAttribute(reinterpret_cast<const void*>(kernel),
                              hipFuncAttributeMaxDynamicSharedMemorySize, int(lds));
  // As many blocks as fit the chip at once, or as there are tiles.
  const uint32_t range = (mtiles * ntiles + kNumXcd - 1) / kNumXcd;
  const uint32_t per_xcd = kNumCu / kNumXcd * RESIDENT;
  const dim3 grid(kNumXcd * (range < per_xcd ? range : per_xcd));
  hipLaunchKernelGGL(kernel, grid, dim3(WN * WM * kWave), lds, st, xc, xs, padded(m), m, groups, w,
                     ws, padded(w.rows), mtiles, ntiles, out, ldo);
}

template <bool FUSED, class TX, class T>
void launch_direct(const TX* x, int64_t stride, const uint8_t* xc, const uint32_t* xs, int32_t m,
                   int32_t groups, const Mx4View& w, T* out, int64_t ldo, hipStream_t st) {
  for_launches((w.rows + 63) / 64, kBlock, [&](uint32_t first, dim3 grid) {
    hipLaunchKernelGGL((scores_direct<TX, T, FUSED>), grid, dim3(kBlock), 0, st, x, stride, xc, xs,
                       padded(m), w, m, groups, out, ldo, first);
  });
}

// More than 16 rows of x.
template <bool X8, class T>
void launch_tiles(const uint8_t* xc, const uint32_t* xs, const uint32_t* ws, int32_t m,
                  int32_t groups, const Mx4View& w, T* out, int64_t ldo, hipStream_t st) {
  auto tiles = [&](int64_t bn, int64_t bm) {
    return (w.rows + bn - 1) / bn * ((m + bm - 1) / bm);
  };
  auto rounds = [](int64_t t, int64_t resident) { return (t + resident - 1) / resident; };
  // The largest tiles where the chip takes four rounds of them or more and those cost less than the
  // rounds of the next size (a round of 256 of 256 x 256 about 10/7 of one of 512 of
  // 128 x 128); smaller ones while they leave compute units idle.  Measured, us, 256 x 256 /
  // 128 x 128 / 128 x 64 / 64 x 64: 4096 x 65536 x 4096 652 / 847 / 1653 / 1760; 1000 x 131072 x
  // 4096 339 / 449 / 886 / 858; 4096 x 65536 x 256 153 / 180 / 282 / 319; 2000 x 20000 x 1024 57 /
  // 49 / 70 / 73; 1024 x 8192 x 1024 19 / 16 / 18 / 20; 200 x 200003 x 256 42 / 31 / 38 / 41;
  // 64 x 200003 x 1024 55 / 34 / 31 / 36; 512 x 4096 x 4096 31 / 17 / 23 / 20; 300 x 1000 x 4096
  // 55 / 26 / 23 / 19.
  const int64_t big = tiles(256, 256), mid = tiles(128, 128);
  const int64_t big_rounds = rounds(big, kNumCu);
  if constexpr (!kExact<X8, T>) {
    if (m > 512 && big_rounds >= 4 && big_rounds * 10 < rounds(mid, 2 * kNumCu) * 7)
      return launch_tile<X8, 4, 4, 2, 2, X8 ? 2 : 3, 1>(xc, xs, m, groups, w, ws, out, ldo, st);
  }
  if (m > 64 && mid >= kNumCu / 2)
    launch_tile<X8, 2, 2, 2, 2, X8 ? 2 : 3, 2>(xc, xs, m, groups, w, ws, out, ldo, st);
  else if (tiles(128, 64) >= kNumCu)
    launch_tile<X8, 1, 2, 4, 1, 3, 2>(xc, xs, m, groups, w, ws, out, ldo, st);
  else
    launch_tile<X8, 1, 1, 2, 2, X8 ? 3 : 4, X8 ? 2 : 3>(xc, xs, m, groups, w, ws, out, ldo, st);
}

template <class T>
void launch_scores(const uint8_t* xc, const uint32_t* xs, const uint32_t* ws, int32_t m,
                   int32_t groups, const Mx4View& w, T* out, int64_t ldo, hipStream_t st) {
  if (m > 16) return launch_tiles<false>(xc, xs, ws, m, groups, w, out, ldo, st);
  launch_direct<false>(static_cast<const T*>(nullptr), 0, xc, xs, m, groups, w, out, ldo, st);
}

// Scales of both sides in the workspace; none for up to 16 rows, which are read in place.
struct Score8Layout {
  size_t ws, total;
};
Score8Layout score8_layout(int32_t m, int64_t n, int32_t k) {
  if (m <= 16) return {0, 0};
  const size_t groups = size_t((k + kGroup - 1) / kGroup);
  Score8Layout L;
  L.ws = size_t(padded(m)) * groups * 4;
  L.total = L.ws + size_t(padded(n)) * groups * 4;
  return L;
}

template <class T>
void launch_scores8(const uint8_t* xc, const uint32_t* xs, int32_t m, int32_t groups, const Mx4View& w,
                    T* out, int64_t ldo, char* ws, hipStream_t st) {
  if (m <= 16) {
    for_launches((w.rows + 63) / 64, kBlock, [&](uint32_t first, dim3 grid) {
      if (m * groups * 128 <= kStaged)
        hipLaunchKernelGGL((scores8_direct<T, true>), grid, dim3(kBlock), 0, st, xc, xs, w, m, groups, out,
                           ldo, first);
      else
        hipLaunchKernelGGL((scores8_direct<T, false>), grid, dim3(kBlock), 0, st, xc, xs, w, m, groups, out,
                           ldo, first);
    });
    return;
  }
  uint32_t* xst = reinterpret_cast<uint32_t*>(ws);
  uint32_t* wst = reinterpret_cast<uint32_t*>(ws + score8_layout(m, w.rows, w.dim).ws);
  const uint32_t xblocks = uint32_t((m + kWave - 1) / kWave);
  const uint32_t wblocks = uint32_t((w.rows + kWave - 1) / kWave);
  for_launches(int64_t(xblocks) + wblocks, kBlock, [&](uint32_t first, dim3 grid) {
    hipLaunchKernelGGL(pack_scales, grid, dim3(kBlock), 0, st, xs, int64_t(m), xst, padded(m), xblocks,
                       reinterpret_cast<const uint32_t*>(w.scales), w.rows, wst, padded(w.rows), groups,
                       first);
  });
  launch_tiles<true>(xc, xst, wst, m, groups, w, out, ldo, st);
}

}  // namespace

size_t mx4_matmul_workspace(int32_t m, int64_t n, int32_t k) { return score_layout(m, n, k).total; }

hipError_t launch_mx4_matmul(const void* x, bool x_bf16, int64_t x_stride, int32_t m,
                             const Mx4View& w, void* out, bool out_bf16, int64_t out_stride,
                             char* ws, hipStream_t st) {
  if (m == 0) return hipSuccess;
  const int groups = (w.dim + kGroup - 1) / kGroup;
  const ScoreLayout L = score_layout(m, w.rows, w.dim);
  uint8_t* xc = reinterpret_cast<uint8_t*>(ws);
  uint8_t* xs = xc + L.xs;
  uint32_t* wst = reinterpret_cast<uint32_t*>(ws + L.ws);
  const uint32_t* wsc = reinterpret_cast<const uint32_t*>(w.scales);
  if (fused(m, w.dim)) {
    auto run = [&](auto* xp, auto* op) {
      launch_direct<true>(xp, x_stride, nullptr, nullptr, m, groups, w, op, out_stride, st);
    };
    const auto* xb = static_cast<const __bf16*>(x);
    const auto* xf = static_cast<const float*>(x);
    auto* ob = static_cast<__bf16*>(out);
    auto* of = static_cast<float*>(out);
    if (x_bf16)
      out_bf16 ? run(xb, ob) : run(xb, of);
    else
      out_bf16 ? run(xf, ob) : run(xf, of);
    return hipGetLastError();
  }
  const int64_t units = int64_t(m) * groups * 4;
  const uint32_t xblocks = uint32_t((units + kBlock / 4 - 1) / (kBlock / 4));
  const uint32_t wblocks = m > 16 ? uint32_t((w.rows + kWave - 1) / kWave) : 0u;
  const FastDiv f = fast_div(uint32_t(groups));
  for_launches(int64_t(xblocks) + wblocks, kBlock, [&](uint32_t first, dim3 pgrid) {
    if (x_bf16)
      hipLaunchKernelGGL(pack_x<__bf16>, pgrid, dim3(kBlock), 0, st, static_cast<const __bf16*>(x),
                         x_stride, m, w.dim, f, xc, xs, padded(m), xblocks, wsc, w.rows, wst,
                         padded(w.rows), first);
    else
      hipLaunchKernelGGL(pack_x<float>, pgrid, dim3(kBlock), 0, st, static_cast<const float*>(x),
                         x_stride, m, w.dim, f, xc, xs, padded(m), xblocks, wsc, w.rows, wst,
                         padded(w.rows), first);
  });
  const uint32_t* xsw = reinterpret_cast<const uint32_t*>(xs);
  if (out_bf16)
    launch_scores(xc, xsw, wst, m, groups, w, static_cast<__bf16*>(out), out_stride, st);
  else
    launch_scores(xc, xsw, wst, m, groups, w, static_cast<float*>(out), out_stride, st);
  return hipGetLastError();
}

size_t mx4_matmul_x8_workspace(int32_t m, int64_t n, int32_t k) { return score8_layout(m, n, k).total; }

hipError_t launch_mx4_matmul_x8(const uint8_t* xc, const uint8_t* xs, int32_t m, const Mx4View& w,
                                void* out, bool out_bf16, int64_t out_stride, char* ws,
                                hipStream_t st) {
  if (m == 0) return hipSuccess;
  const int groups = (w.dim + kGroup - 1) / kGroup;
  const uint32_t* xsw = reinterpret_cast<const uint32_t*>(xs);
  if (out_bf16)
    launch_scores8(xc, xsw, m, groups, w, static_cast<__bf16*>(out), out_stride, ws, st);
  else
    launch_scores8(xc, xsw, m, groups, w, static_cast<float*>(out), out_stride, ws, st);
  return hipGetLastError();
}

}  // namespace embbag
