// Tiles of BF16 products through LDS: out[m][n] = sum over k of B[m][k] A[n][k], sums in FP32.
//
// Both sides go from memory straight to LDS, 32 elements of k per step, STAGES steps in turn (the loads
// of a step are issued STAGES - 1 steps ahead), and out of it as the fragments of 32 x 32 x 16 products.
// A side is either rows of k (its row of a step 64 bytes, the 16-byte chunk c of row r at place
// c ^ (r / 4 % 4)) or, turned, rows of n or m, one for each k (chunk c of row k at place c ^ 4 (k % 4)), which
// the transposing LDS read turns around: either way 64 lanes' reads meet all banks.
// Loads are buffer loads: what lies past a side's end is 0.
//
// A block takes tile after tile (every XCD its own range), and the loads run through the steps of all of
// them.  Sides may have planes (numbers split in several BF16 terms): a tile's steps run over pairs of
// planes, the smallest products first.
//
// Bound by the matrix instructions at the clock they leave: of 4096 x 131072 x 2048 the scores' and the
// gradients' tiles (256 x 256, a block per compute unit) keep them busy for 62 to 68 % of the cycles, at 1.75 to 1.8 GHz;
// all four products with their epilogues take 7.1 ms, a library's four alone 6.6.  Six pairs of planes with the
// epilogue that keeps the scores spill in tiles of 256 x 256 (192 bytes a lane, after a tile's last step).
#pragma once

#include <type_traits>

#include "head.hpp"

namespace embbag {
namespace {

typedef float f16v __attribute__((ext_vector_type(16)));
typedef short s4v __attribute__((ext_vector_type(4)));

constexpr int kStepK = 32;              // elements of k per step
constexpr int kStepBytes = kStepK * 2;  // of a row of k
constexpr uint32_t kFar = 0x40000000u;  // an offset that no side's buffer has

// A side of the products.  Bytes from row to row, from plane to plane.  Rows end at multiples of 8
// elements (loads are whole words: what the last ones hold past the counts is a row's own).
struct Side {
  const void* data;
  int64_t pitch;
  int64_t plane;
};

// Splits of a contraction of `steps` steps over tiles that would leave blocks idle: as many as make `blocks`
// of them, of 8 steps at least, and the steps of each.
struct Splits {
  int32_t count, per;
};
__host__ __device__ __forceinline__ Splits split_steps(int64_t tiles, int64_t steps, int32_t blocks) {
  if (steps < 1) steps = 1;
  int64_t s = blocks / (tiles > 0 ? tiles : 1);
  if (s > steps / 8) s = steps / 8;
  if (s < 1) s = 1;
  const int64_t per = (steps + s - 1) / s;
  return {int32_t((steps + per - 1) / per), int32_t(per)};
}

// The problem.  `live`, where not null, holds the number of rows of m (or of k where LIVE_K) in
// memory; the counts given are then upper bounds.
struct Gemm {
  Side a, b;
  int64_t n, m, k;
  const int32_t* live;
  int32_t pairs;   // of planes: 1, 2 (both of b) or 6 (of three each)
  Splits splits;   // of k: how many, and steps per split and pair
  // Where not 0, the splits are found from the tiles of the rows that count instead: split_steps of
  // `steps`.
  int32_t blocks;
  int64_t steps;
  // With pairs == 2: the largest *live for which the second plane is read.
  int32_t few;
};

// Pair number i: the planes of a and b.
__device__ __forceinline__ void planes_of(int pairs, int i, int* pa, int* pb) {
  // Of three planes each: (2,0) (1,1) (0,2) (1,0) (0,1) (0,0).
  *pa = pairs == 6 ? int(0x001012u >> (4 * i) & 15u) : 0;
  *pb = pairs == 6 ? int(0x010210u >> (4 * i) & 15u) : pairs == 2 ? 1 - i : 0;
}

typedef __attribute__((address_space(3))) void* LdsAny;
// (Addresses and sizes are the wavefront's; said so, they stay in scalar registers.)
__device__ __forceinline__ int scalar(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer_of(const void* p, int bytes) {
  const uint64_t a = reinterpret_cast<uint64_t>(p);
  const uint64_t u = uint64_t(uint32_t(scalar(int(a >> 32)))) << 32 | uint32_t(scalar(int(a)));
  return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void*>(u), 0, scalar(bytes), 0x00020000);
}
__device__ __forceinline__ void buffer_to_lds16(__amdgpu_buffer_rsrc_t r, uint32_t voff, uint32_t soff,
                                                void* dst) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (LdsAny)dst, 16, int(voff), int(soff), 0, 0);
}

// Until at most N of this wavefront's loads are on their way, its LDS reads complete.
template <int N>
__device__ __forceinline__ void wait_loads() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N) : "memory");
}
// The block's barrier alone: unlike __syncthreads it leaves loads to LDS on their way.
__device__ __forceinline__ void block_barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// Where a side's loads of a tile come from, one step after the other.
template <bool TURNED, int ROWS, int W>
struct Stream {
  static constexpr int ALL = ROWS / 16;             // loads of 1024 bytes per step
  static constexpr int LOADS = (ALL + W - 1) / W;   // per wavefront (the last ones may come twice)
  static constexpr int PITCH = ROWS * 2;            // bytes of a turned side's row in LDS
  static constexpr int KROWS = 1024 / PITCH;        // of them per load
  static_assert(!TURNED || ROWS >= 64, "swizzle of turned rows");
  const uint8_t* base;
  int64_t left;      // bytes from base to the side's end
  int records;       // of them in the loads' buffer
  uint32_t at;       // bytes from base to the step
  uint32_t step;     // bytes of a step
  uint32_t rows;     // bytes from a load's first row to the next load's
  uint32_t voff;     // of this lane in a load
  int limit;         // rows of k: elements of k from this lane's chunk to the end

  __device__ __forceinline__ int number(int i, int wave) const { return (i * W + wave) % ALL; }
  __device__ __forceinline__ void clamp() {
    const int64_t most = kFar - 1;
    records = int(left < 0 ? 0 : left < most ? left : most);
  }

  // The tile from row r0 of `total`, the steps from k0 of `k` elements on.
  __device__ __forceinline__ void open(const Side& s, int plane, int64_t r0, int64_t total, int64_t k0,
                                       int64_t k, int lane, int wave) {
    const int64_t pitch = s.pitch;
    const uint8_t* p = static_cast<const uint8_t*>(s.data) + plane * s.plane;
    if constexpr (TURNED) {
      base = p + k0 * pitch + r0 * 2;
      left = (k - k0 - 1) * pitch + (total - r0 + 7) / 8 * 16;
      constexpr int PER = 64 / KROWS;  // lanes per row
      const int kk = lane / PER;
      const int sw = KROWS == 8 ? (kk >> 1 & 1) : KROWS == 4 ? kk : (wave & 1) * 2 + kk;
      voff = uint32_t(kk * pitch) + uint32_t((lane % PER) ^ (sw * 4)) * 16;
      static_assert(KROWS > 2 || W % 2 == 0, "a load's parity is its wavefront's");
      step = uint32_t(kStepK * pitch);
      rows = uint32_t(KROWS * pitch);
    } else {
      base = p + r0 * pitch + k0 * 2;
      left = (total - r0 - 1) * pitch + (k - k0 + 7) / 8 * 16;
      const int c = (lane % 4) ^ (lane / 16);
      voff = uint32_t(lane / 4 * pitch) + uint32_t(c) * 16;
      limit = int(k - k0) - c * 8;
      step = kStepBytes;
      rows = uint32_t(16 * pitch);
    }
    if (k <= k0) left = 0;
    at = 0;
    clamp();
  }
  __device__ __forceinline__ void advance() {
    at += step;
    if constexpr (TURNED) {
      if (at >= kFar / 4) {  // (the buffer's offsets and a step's rows stay below kFar)
        base += at;
        left -= at;
        at = 0;
        clamp();
      }
    } else {
      limit -= kStepK;
    }
  }
  __device__ __forceinline__ void load(int i, int wave, uint8_t* dst) const {
    const int l = number(i, wave);
    const uint32_t v = !TURNED && limit <= 0 ? kFar : voff;
    buffer_to_lds16(buffer_of(base, records), v, at + uint32_t(l) * rows, dst + l * 1024);
  }
};

// Tile number id: strips of `width` m tiles, in a strip n tile after n tile.
__device__ __forceinline__ void tile_at(uint32_t id, uint32_t mtiles, uint32_t ntiles, uint32_t strip,
                                        uint32_t* mt, uint32_t* nt) {
  const uint32_t s = id / (strip * ntiles);
  const uint32_t m0 = s * strip, width = min(strip, mtiles - m0);
  const uint32_t in = id - m0 * ntiles;
  *nt = in / width;
  *mt = m0 + in - *nt * width;
}

// WN x WM wavefronts, each TN x TM products of 32 x 32.  After a tile's last step every wavefront hands
// its sums to epi(acc, n, m, m_end, z, scratch): acc[i][j] element q * 4 + e of lane l is row
// m + 32 j + l % 32 and column n + 32 i + 8 q + 4 (l / 32) + e.  epi must not meet a barrier.
template <int TN, int TM, int WN, int WM, int STAGES, bool AT, bool BT, bool LIVE_K, class Epi>
__global__ __launch_bounds__(WN* WM* kWave, 1) void gemm_tiles(Gemm g, Epi epi, uint32_t mtiles_most,
                                                               uint32_t ntiles, uint32_t strip) {
  constexpr int BN = 32 * TN * WN, BM = 32 * TM * WM, W = WN * WM;
  constexpr int STAGE = (BN + BM) * kStepBytes;
  typedef Stream<AT, BN, W> SA;
  typedef Stream<BT, BM, W> SB;
  extern __shared__ __align__(16) uint8_t lds[];
  const int lane = lane_id(), wave = wave_id();
  uint8_t* scratch = lds + STAGES * STAGE + wave * Epi::template kScratch<TN, TM>;

  int64_t m_end = g.m, k_end = g.k;
  int pairs = g.pairs;
  if (g.live != nullptr) {
    const int live = __builtin_amdgcn_readfirstlane(*g.live);
    if constexpr (LIVE_K)
      k_end = live;
    else
      m_end = live;
    if (pairs == 2 && live > g.few) pairs = 1;
  }
  const uint32_t mtiles = LIVE_K ? mtiles_most : uint32_t((m_end + BM - 1) / BM);
  const uint32_t plain = mtiles * ntiles;
  Splits sp = g.splits;
  if (g.blocks != 0) sp = split_steps(plain, g.steps, g.blocks);
  const uint32_t tiles = plain * uint32_t(sp.count);
  const uint32_t range = (tiles + kNumXcd - 1) / kNumXcd, stride = gridDim.x / kNumXcd;
  const uint32_t end = min((blockIdx.x % kNumXcd + 1) * range, tiles);
  uint32_t tile = blockIdx.x % kNumXcd * range + blockIdx.x / kNumXcd;
  if (tile >= end) return;

  // Steps of split z for a pair of planes (one at least, of zeros where there is nothing to add).
  auto steps_of = [&](uint32_t z) {
    const int64_t k0 = int64_t(z) * sp.per * kStepK;
    const int64_t left = (k_end - k0 + kStepK - 1) / kStepK;
    return int(left < 1 ? 1 : left < sp.per ? left : sp.per);
  };
  uint32_t ltile = tile;
  int lstep = 0, lsteps = 0, lpair = 0;
  SA sa;
  SB sb;
  auto open = [&]() {
    const uint32_t z = ltile / plain;
    uint32_t mt, nt;
    tile_at(ltile - z * plain, mtiles, ntiles, strip, &mt, &nt);
    int pa, pb;
    planes_of(pairs, lpair, &pa, &pb);
    const int64_t k0 = int64_t(z) * sp.per * kStepK;
    sa.open(g.a, pa, int64_t(nt) * BN, g.n, k0, k_end, lane, wave);
    sb.open(g.b, pb, int64_t(mt) * BM, m_end, k0, k_end, lane, wave);
    lsteps = steps_of(z);
    lstep = 0;
  };
  open();
  // Before a step's loads.  After the last tile its last pair of planes is loaded again, so that the number
  // of loads on their way is always the same.
  auto next_load = [&]() {
    if (lstep == lsteps) {
      if (++lpair == pairs) {
        if (ltile + stride < end)
          lpair = 0, ltile += stride;
        else
          --lpair;
      }
      open();
    } else if (lstep > 0) {
      sa.advance();
      sb.advance();
    }
    ++lstep;
  };
  constexpr int PER = SA::LOADS + SB::LOADS;
  auto load = [&](uint8_t* dst, int i) {
    if (i < SA::LOADS)
      sa.load(i, wave, dst);
    else
      sb.load(i - SA::LOADS, wave, dst + BN * kStepBytes);
  };

  const int wn = wave % WN, wm = wave / WN;
  const int half = lane / 32, row = lane % 32;
  f16v acc[TN][TM];
  const int at0 = ((2 * half) ^ (row / 4 % 4)) * 16;  // place of part p's chunk: at0 ^ (16 p)
  const int kq = lane % 16 / 4, tcol = lane / 16 % 2 * 32 + lane % 4 * 8;
  constexpr int BOFF = BN * kStepBytes;
  // A fragment of part p: 8 elements of k from 16 (l / 32) + 8 p on, of row l % 32.
  auto fragment = [&](const uint8_t* __restrict__ cur, auto turned, auto rows, int off, int group,
                      int p) {
    if constexpr (turned) {
      constexpr int PITCH = rows * 2;
      const int sw = rows == 64 ? kq >> 1 : kq;
      const uint8_t* q = cur + off + (half * 16 + kq) * PITCH + ((group ^ sw) * 64 + tcol) + p * 8 * PITCH;
      typedef __attribute__((address_space(3))) s4v* lds4;
      const s4v lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)q);
      const s4v hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(q + 4 * PITCH));
      const u2 l2 = __builtin_bit_cast(u2, lo), h2 = __builtin_bit_cast(u2, hi);
      return u4{l2.x, l2.y, h2.x, h2.y};
    } else {
      return *reinterpret_cast<const u4*>(cur + off + (group * 32 + row) * kStepBytes + (at0 ^ (16 * p)));
    }
  };
  u4 a[2][TN] = {}, b[2][TM] = {};
  auto fetch = [&](const uint8_t* __restrict__ cur, int p, int i) {
    if (i < TM)
      b[p][i] = fragment(cur, std::integral_constant<bool, BT>(), std::integral_constant<int, BM>(), BOFF,
                         wm * TM + i, p);
    else
      a[p][i - TM] = fragment(cur, std::integral_constant<bool, AT>(), std::integral_constant<int, BN>(), 0,
                              wn * TN + i - TM, p);
  };
  // The products of part p, and after every one of them what a wavefront alone on its SIMD can issue while
  // it runs (an instruction per 4 cycles, a product takes 32): in the first half the reads of the next part's
  // fragments (part `next` of `cur`), in the second half that half step's loads of a later step, which go to
  // `nxt`.
  auto part = [&](const uint8_t* __restrict__ cur, uint8_t* __restrict__ nxt, int p, int next) {
    constexpr int N = TN + TM, SLOTS = TN * TM, EARLY = SLOTS > 1 ? SLOTS / 2 : 1, LATE = SLOTS - SLOTS / 2;
    constexpr int HALF = (PER + 1) / 2;
#pragma unroll
    for (int s = 0; s < SLOTS; ++s) {
      const int i = s / TM, j = s % TM;
      acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf8, a[p][i]),
                                                          __builtin_bit_cast(bf8, b[p][j]), acc[i][j], 0,
                                                          0, 0);
      if (next < 0) continue;
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int r = 0; r < N; ++r)
        if (r * EARLY / N == s) fetch(cur, next, r);
#pragma unroll
      for (int l = 0; l < PER; ++l)
        if (l / HALF == next && SLOTS / 2 + l % HALF * LATE / HALF == s) load(nxt, l);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
#pragma unroll
  for (int i = 0; i < STAGES - 1; ++i) {
    next_load();
#pragma unroll
    for (int l = 0; l < PER; ++l) load(lds + i * STAGE, l);
  }
  int cur = 0;
  for (;; tile += stride) {
#pragma unroll
    for (int i = 0; i < TN; ++i)
#pragma unroll
      for (int j = 0; j < TM; ++j) acc[i][j] = f16v{};
    const uint32_t z = tile / plain;
    const int steps = steps_of(z) * pairs;
    for (int step = 0; step < steps; ++step) {
      next_load();
      // This step is in LDS (the next STAGES - 2 may be on their way), and every wavefront holds the
      // last fragments of the stage before, which the next load overwrites.
      wait_loads<(STAGES - 2) * PER>();
      block_barrier();
      const int free = cur == 0 ? STAGES - 1 : cur - 1;
      part(lds + cur * STAGE, lds + free * STAGE, 1, 0);
      part(lds + cur * STAGE, lds + free * STAGE, 0, 1);
      cur = cur == STAGES - 1 ? 0 : cur + 1;
    }
    part(lds, lds, 1, -1);
    // (The next tile's first products take no fragments.)
#pragma unroll
    for (int i = 0; i < TN; ++i) a[1][i] = u4{0u, 0u, 0u, 0u};
#pragma unroll
    for (int i = 0; i < TM; ++i) b[1][i] = u4{0u, 0u, 0u, 0u};
    uint32_t mt, nt;
    tile_at(tile - z * plain, mtiles, ntiles, strip, &mt, &nt);
    epi.template operator()<TN, TM>(acc, int64_t(nt) * BN + wn * TN * 32, int64_t(mt) * BM + wm * TM * 32,
                                    m_end, int(z), scratch);
    if (tile + stride >= end) break;
  }
  // No load to LDS outlives the block.
  wait_loads<0>();
}

// Launches a shape.  RESIDENT blocks share a compute unit.
template <int TN, int TM, int WN, int WM, int STAGES, int RESIDENT, bool AT, bool BT, bool LIVE_K, class Epi>
void launch_gemm(const Gemm& g, const Epi& epi, uint32_t strip, hipStream_t st) {
  constexpr int BN = 32 * TN * WN, BM = 32 * TM * WM, W = WN * WM;
  constexpr int lds = STAGES * (BN + BM) * kStepBytes + W * Epi::template kScratch<TN, TM>;
  static_assert(lds <= 160 * 1024 / RESIDENT, "blocks that share a compute unit");
  const uint32_t mtiles = uint32_t((g.m + BM - 1) / BM), ntiles = uint32_t((g.n + BN - 1) / BN);
  if (mtiles == 0 || ntiles == 0) return;
  auto kernel = gemm_tiles<TN, TM, WN, WM, STAGES, AT, BT, LIVE_K, Epi>;
  if (lds > 65536)
    (void)hipFuncSetAttribute(reinterpret_cast<const void*>(kernel),
                              hipFuncAttributeMaxDynamicSharedMemorySize, lds);
  const uint64_t range = (uint64_t(mtiles) * ntiles * uint32_t(g.splits.count) + kNumXcd - 1) / kNumXcd;
  const uint32_t per_xcd = kNumCu / kNumXcd * RESIDENT;
  const uint32_t blocks = g.blocks != 0 ? uint32_t(g.blocks) / kNumXcd : uint32_t(range);
  hipLaunchKernelGGL(kernel, dim3(kNumXcd * (blocks < per_xcd ? blocks : per_xcd)), dim3(W * kWave),
                     lds, st, g, epi, mtiles, ntiles, strip);
}

}  // namespace
}  // namespace embbag
