// Gradient of the scores with respect to x: dx = dy W, W a 4-bit microscaled
// table.
//
// The contraction runs over W's rows, across its blocks: W's values go through the
// BF16 matrix instructions, which hold every code times its scale exactly (an element is
// 0.5 to 6 times a power of two).  A block of 256 threads makes a BK x BM tile of dx^T over a
// range of W's rows, in steps of 64 rows.  Per step, double-buffered:
//   - dy's tile goes to LDS as it is, [BM][64] BF16, the 16-byte place of a row exchanged
//     with the row's number (row % 8) so that fragments spread over the banks;
//   - W's tile is converted on its way, [64][BK] BF16, rows 32 bytes apart in the banks, and is
//     turned around by the transposing LDS read that makes the fragments.
// Where tiles alone leave compute units idle the rows of W are split over blocks as
// well; the FP32 parts are then added in order by a second kernel.
//
// 4096 x 32768 x 1024, BF16: 248 us with the parts' sum, 1.1 PFLOP/s (a BF16 library product of
// these sizes 398 us, 1.4 PFLOP/s for its best shapes, 1.9 from registers on such data).  Bound by
// the products and the LDS traffic between them; without the interleaving of `part` 409 us.
// 200 x 50001 x 256: 22 us, bound by its chain of steps.
//
// An FP32 dy is the sum of three BF16 terms of 8 bits each, by truncation (bits below 2^-133, which no
// BF16 number has, are dropped): three tiles of dy for one of W, whose fragments meet all three (1024 x
// 20000 x 1024 148 us, with a step of its own for each term 317; 64 x 100000 x 256 25, 43).
#include "head.hpp"

namespace embbag {
namespace {

typedef float f16v __attribute__((ext_vector_type(16)));
typedef short s4v __attribute__((ext_vector_type(4)));
typedef u4 u4_el __attribute__((aligned(2)));
typedef f4 f4_el __attribute__((aligned(4)));

constexpr int kRows = 64;                   // rows of W per step
constexpr int kYRow = kRows * 2;            // bytes of a row of dy's tile

template <int BK>
constexpr int kWRow = BK * 2 + 32;          // bytes of a row of W's tile
template <int BK, int BM, int TERMS>
constexpr int kStage = TERMS * BM * kYRow + kRows * kWRow<BK>;

// x as the sum of three terms: its 8 highest bits, the next 8, the rest, as BF16 patterns in the upper
// halves.  An infinity or a NaN is its own first term and leaves nothing.
__device__ __forceinline__ void bf16_terms(float x, uint32_t (&t)[3]) {
  uint32_t u = __float_as_uint(x);
  const bool special = (u & 0x7F800000u) == 0x7F800000u;
  if (special) u |= (u & 0x007FFFFFu) != 0u ? 0x00400000u : 0u;
  t[0] = u & 0xFFFF0000u;
  const float rest = special ? 0.f : __uint_as_float(u) - __uint_as_float(t[0]);
  t[1] = __float_as_uint(rest) & 0xFFFF0000u;
  t[2] = __float_as_uint(rest - __uint_as_float(t[1])) & 0xFFFF0000u;
}

// 8 elements of a row of dy on their way to LDS, and as BF16 (three terms of FP32 ones).
struct Raw16 {
  u4 v;
};
struct Raw32 {
  f4 a, b;
};
__device__ __forceinline__ Raw16 load8(const __bf16* p) {
  return {*reinterpret_cast<const u4_el*>(p)};
}
__device__ __forceinline__ Raw32 load8(const float* p) {
  return {*reinterpret_cast<const f4_el*>(p), *reinterpret_cast<const f4_el*>(p + 4)};
}
__device__ __forceinline__ void to_bf16(const Raw16& r, u4 (&t)[1]) { t[0] = r.v; }
__device__ __forceinline__ void to_bf16(const Raw32& r, u4 (&t)[3]) {
  const float x[8] = {r.a.x, r.a.y, r.a.z, r.a.w, r.b.x, r.b.y, r.b.z, r.b.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t lo[3], hi[3];
    bf16_terms(x[2 * i], lo);
    bf16_terms(x[2 * i + 1], hi);
#pragma unroll
    for (int q = 0; q < 3; ++q) t[q][i] = lo[q] >> 16 | hi[q];
  }
}
// A word of codes as 8 BF16 values.
__device__ __forceinline__ u4 bf16_values8(uint32_t c, float scale) {
  return u4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 0)),
            __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 1)),
            __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 2)),
            __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 3))};
}

// WK x WM wavefronts, each TK x TM products of 32 x 32.  Block: split z of the rows of W
// (`per` steps each), k tile, m tile, from block `first` of them on.  `dx` is the output, or part z of
// the parts.
//
// The last rows of all may be less than a step.  dy's 8 columns of a load that would pass its row
// are then the row's last 8: W's tile takes the same rows there, without those that
// an earlier load has brought.  Their columns of dy become 0 as well, since an infinity among them would
// make NaN of W's zeros.  A block takes its last rows first, so that this is done once, before its loop
// (in the loop it cost 2%: 1024 x 20000 x 1024 with FP32 dy 146.5 us, here 143).
template <int TK, int TM, int WK, int WM, class TY, class TX>
__global__ __launch_bounds__(kBlock, 1) void grad_tile(const TY* __restrict__ dy, int64_t ldy,
                                                       int32_t m, Mx4View w, uint32_t ktiles,
                                                       uint32_t mtiles, int32_t per,
                                                       TX* __restrict__ dx, int64_t ldx,
                                                       int64_t part_stride, uint32_t first) {
  static_assert(WK * WM == kWavesPerBlock, "four wavefronts");
  constexpr int BK = 32 * TK * WK, BM = 32 * TM * WM;
  constexpr int YL = BM / 32;              // loads of dy per thread
  constexpr int WL = kRows * BK / 32 / kBlock;  // blocks of W per thread
  static_assert(WL >= 1 && YL >= 1, "a load of each per thread");
  constexpr int TERMS = sizeof(TY) == 4 ? 3 : 1;
  constexpr int STAGE = kStage<BK, BM, TERMS>;
  extern __shared__ __align__(16) uint8_t lds[];

  const int lane = lane_id(), wave = wave_id();
  const uint32_t id = first + xcd_remap(blockIdx.x, gridDim.x);
  const uint32_t tiles = ktiles * mtiles;
  const uint32_t z = id / tiles, tile = id - z * tiles;
  const uint32_t mt = tile / ktiles, kt = tile - mt * ktiles;
  const int m0 = int(mt) * BM, k0 = int(kt) * BK;
  const int64_t n0 = int64_t(z) * per * kRows;
  const int rows = int(min(w.rows - n0, int64_t(per) * kRows));  // of W, in this block (>= 1)
  const int steps = (rows + kRows - 1) / kRows;
  const int nb = mx4_blocks(w.dim), sb = mx4_scale_bytes(w.dim);

  // dy: load i of this thread is 8 columns (8 * yc ..) of row i * 32 + threadIdx.x / 8.
  const int yr = threadIdx.x / 8, yc = threadIdx.x % 8;
  const TY* ysrc[YL];
#pragma unroll
  for (int i = 0; i < YL; ++i)
    ysrc[i] = dy + int64_t(min(m0 + i * 32 + yr, m - 1)) * ldy + n0;
  // W: block i of this thread is number wb + PER * i (of the tile's BK/32) of row wr.
  constexpr int PER = kBlock / kRows;  // threads per row
  const int wr = threadIdx.x / PER, wb = threadIdx.x % PER;
  decltype(load8(dy)) yv[YL];
  u4 wv[WL];
  uint32_t ws[WL];
  int64_t wrow = 0;
  int ycol = 0;
  bool win = false;

  // Places of step s's loads.
  const int last = rows - 8;  // of the last 8 rows, the first (in the split before, if rows < 8)
  auto place = [&](int s) {
    const int r0 = s * kRows;
    ycol = min(r0 + yc * 8, last);
    const int c = r0 + wr / 8 * 8;  // the first row of wr's 8
    const int r = min(c, last) + wr % 8;
    win = r >= c && r < rows;
    wrow = n0 + (win ? r : 0);
  };
  auto load_y = [&](int i) { yv[i] = load8(ysrc[i] + ycol); };
  auto load_w = [&](int i) {
    const int b = min(k0 / kMxBlock + wb + PER * i, nb - 1);
    wv[i] = *reinterpret_cast<const u4*>(w.codes + (wrow * nb + b) * 16);
    ws[i] = w.scales[wrow * sb + b];
  };
  bool in = false;  // whether the loads that are stored next were of a row to be added
  auto store_y = [&](uint8_t* st, int i) {
    u4 t[TERMS];
    to_bf16(yv[i], t);
#pragma unroll
    for (int q = 0; q < TERMS; ++q)
      *reinterpret_cast<u4*>(st + (q * BM + i * 32 + yr) * kYRow + (yc ^ (yr & 7)) * 16) = t[q];
  };
  auto store_w = [&](uint8_t* st, int i) {
    const float s = mx4_scale(in ? ws[i] : 0u);
    u4* p = reinterpret_cast<u4*>(st + TERMS * BM * kYRow + wr * kWRow<BK> + (wb + PER * i) * 64);
    p[0] = bf16_values8(in ? wv[i].x : 0u, s);
    p[1] = bf16_values8(in ? wv[i].y : 0u, s);
    p[2] = bf16_values8(in ? wv[i].z : 0u, s);
    p[3] = bf16_values8(in ? wv[i].w : 0u, s);
  };

  const int wk = wave % WK, wm = wave / WK;
  const int row = lane % 32, half = lane / 32;
  f16v acc[TK][TM];
#pragma unroll
  for (int i = 0; i < TK; ++i)
#pragma unroll
    for (int j = 0; j < TM; ++j) acc[i][j] = f16v{};

  // Fragments of part p (rows 16 p .. 16 p + 15): lane l holds column l % 32 and 8 rows from
  // 8 * (l / 32).  W's come from two transposing reads: 16 lanes bring 4 rows of 16 columns
  // and each leaves with its column.
  const int yfrag = (wm * TM * 32 + row) * kYRow;
  const int wfrag = TERMS * BM * kYRow + (half * 8 + (lane % 16) / 4) * kWRow<BK> +
                    (wk * TK * 32 + (lane / 16 % 2) * 16 + (lane % 4) * 4) * 2;
  constexpr int YF = TERMS * TM;  // fragments of dy
  u4 a[2][TK] = {}, b[2][YF] = {};
  auto fetch = [&](const uint8_t* st, int p, int i) {
    if (i < YF) {
      b[p & 1][i] = *reinterpret_cast<const u4*>(st + yfrag + (i / TM * BM + i % TM * 32) * kYRow +
                                                 ((p * 2 + half) ^ (row & 7)) * 16);
    } else {
      const uint8_t* q = st + wfrag + p * 16 * kWRow<BK> + (i - YF) * 64;
      typedef __attribute__((address_space(3))) s4v* lds4;
      const s4v lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)q);
      const s4v hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(q + 4 * kWRow<BK>));
      const u2 l2 = __builtin_bit_cast(u2, lo), h2 = __builtin_bit_cast(u2, hi);
      a[p & 1][i - YF] = u4{l2.x, l2.y, h2.x, h2.y};
    }
  };
  // The products of part p, and between their rows: the reads of the next part's fragments
  // (part `next` of `cur`), and in the first three parts of a step the stores of the next
  // stage, each followed by the load that takes its registers.
  auto part = [&](const uint8_t* cur, uint8_t* nxt, int p, int next, int turn) {
    constexpr int N = TK + YF, READS = TK > 1 ? TK - 1 : 1;
    constexpr int MOVES = YL + WL, SLOTS = 3 * TK;
#pragma unroll
    for (int i = 0; i < TK; ++i) {
#pragma unroll
      for (int j = 0; j < YF; ++j)
        acc[i][j % TM] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
            __builtin_bit_cast(bf8, a[p & 1][i]), __builtin_bit_cast(bf8, b[p & 1][j]),
            acc[i][j % TM], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int r = 0; r < N; ++r)
        if (r * READS / N == i) fetch(cur, next, r);
#pragma unroll
      for (int q = 0; q < MOVES; ++q) {
        if (turn < 3 && q * SLOTS / MOVES == turn * TK + i) {
          if (q < WL)
            store_w(nxt, q), load_w(q);
          else
            store_y(nxt, q - WL), load_y(q - WL);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  };

  // The columns of dy that this thread has stored and that a load before it brought as well (its first
  // ones), or that lie past the end (all 8).
  auto clear_y = [&](uint8_t* st) {
    const int c = (steps - 1) * kRows + yc * 8;
    const int again = min(c - min(c, last), 8);
    if (again == 0) return;
    u4 keep;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      keep[e] = again > 2 * e + 1 ? 0u : again > 2 * e ? 0xFFFF0000u : 0xFFFFFFFFu;
#pragma unroll 1
    for (int i = 0; i < TERMS * YL; ++i) {
      u4* p = reinterpret_cast<u4*>(st + (i / YL * BM + i % YL * 32 + yr) * kYRow +
                                    (yc ^ (yr & 7)) * 16);
      *p &= keep;
    }
  };

  place(steps - 1);
  in = win;
#pragma unroll
  for (int i = 0; i < YL; ++i) load_y(i);
#pragma unroll
  for (int i = 0; i < WL; ++i) load_w(i);
#pragma unroll
  for (int i = 0; i < YL; ++i) store_y(lds, i);
#pragma unroll
  for (int i = 0; i < WL; ++i) store_w(lds, i);
  if (rows % kRows != 0) clear_y(lds);
  place(0);
  in = win;
#pragma unroll
  for (int i = 0; i < YL; ++i) load_y(i);
#pragma unroll
  for (int i = 0; i < WL; ++i) load_w(i);
  for (int s = 0; s < steps; ++s) {
    uint8_t* cur = lds + (s & 1) * STAGE;
    uint8_t* nxt = lds + (~s & 1) * STAGE;
    // The stage is in LDS, and every wavefront holds the last fragments of the other one.
    __syncthreads();
    place(min(s + 1, steps - 1));  // (What the last two turns load is not used.)
    part(cur, nxt, 3, 0, 0);
    part(cur, nxt, 0, 1, 1);
    part(cur, nxt, 1, 2, 2);
    part(cur, nxt, 2, 3, 3);
    in = win;
  }
  part(lds, lds, 3, 0, 3);

  TX* out = dx + int64_t(z) * part_stride;
#pragma unroll
  for (int j = 0; j < TM; ++j) {
    const int mm = m0 + (wm * TM + j) * 32 + row;
    if (mm >= m) continue;
#pragma unroll
    for (int i = 0; i < TK; ++i)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int k = k0 + (wk * TK + i) * 32 + q * 8 + half * 4;
        if (k < w.dim)
          store4(out + int64_t(mm) * ldx + k,
                 f4{acc[i][j][q * 4], acc[i][j][q * 4 + 1], acc[i][j][q * 4 + 2],
                    acc[i][j][q * 4 + 3]});
      }
  }
}

// dx = the sum of the parts [splits][m][k], in order.
template <class TX>
__global__ __launch_bounds__(kBlock) void grad_join(const float* __restrict__ parts, int32_t splits,
                                                    int32_t m, FastDiv k4, TX* __restrict__ dx,
                                                    int64_t ldx) {
  const int64_t n = int64_t(m) * k4.div;
  const int64_t i = int64_t(blockIdx.x) * kBlock + threadIdx.x;
  if (i >= n) return;
  f4 s = load4(parts + i * 4);
  for (int z = 1; z < splits; ++z) s += load4(parts + (z * n + i) * 4);
  const uint32_t row = quotient(uint32_t(i), k4);
  store4(dx + int64_t(row) * ldx + (uint32_t(i) - row * k4.div) * 4, s);
}

// The same where there are many parts of few elements: a wavefront adds every WAVES-th part,
// then the first adds the wavefronts' sums in order.
template <class TX>
__global__ __launch_bounds__(1024) void grad_join_many(const float* __restrict__ parts,
                                                       int32_t splits, int32_t m, FastDiv k4,
                                                       TX* __restrict__ dx, int64_t ldx) {
  constexpr int WAVES = 16;
  __shared__ f4 sums[WAVES][kWave];
  const int64_t n = int64_t(m) * k4.div;
  const int64_t i = int64_t(blockIdx.x) * kWave + lane_id();
  const int wave = wave_id();
  f4 s = {0.f, 0.f, 0.f, 0.f};
  if (i < n) {
#pragma unroll 4
    for (int z = wave; z < splits; z += WAVES) s += load4(parts + (z * n + i) * 4);
  }
  sums[wave][lane_id()] = s;
  __syncthreads();
  if (wave != 0 || i >= n) return;
#pragma unroll
  for (int w = 1; w < WAVES; ++w) s += sums[w][lane_id()];
  const uint32_t row = quotient(uint32_t(i), k4);
  store4(dx + int64_t(row) * ldx + (uint32_t(i) - row * k4.div) * 4, s);
}

// Tables of fewer than 8 rows, which the tiles' loads of 8 columns would pass.  The launch begins with
// block `first`.
template <class TY, class TX>
__global__ __launch_bounds__(kBlock) void grad_few(const TY* __restrict__ dy, int64_t ldy, int32_t m,
                                                   Mx4View w, TX* __restrict__ dx, int64_t ldx,
                                                   uint32_t first) {
  const int64_t k4 = w.dim / 4;
  const int64_t i = (int64_t(first) + blockIdx.x) * kBlock + threadIdx.x;
  if (i >= m * k4) return;
  const int64_t row = i / k4;
  const int e0 = int(i - row * k4) * 4;
  f4 s = {0.f, 0.f, 0.f, 0.f};
  for (int j = 0; j < int(w.rows); ++j) {
    const uint32_t c = *reinterpret_cast<const uint16_t*>(
        w.codes + int64_t(j) * mx4_blocks(w.dim) * 16 + e0 / 2);
    float v[8];
    mx4_values8(c, mx4_scale(w.scales[int64_t(j) * mx4_scale_bytes(w.dim) + e0 / kMxBlock]), v);
    const float y = to_f32(dy[row * ldy + j]);
    s += f4{y * v[0], y * v[1], y * v[2], y * v[3]};
  }
  store4(dx + row * ldx + e0, s);
}

// Tile and split of a gradient.
struct GradPlan {
  int bk, bm;
  uint32_t ktiles, mtiles, splits;
  int32_t per;  // steps per split
};
GradPlan grad_plan(int32_t m, int64_t n, int32_t k, bool y_bf16) {
  GradPlan p = {};
  if (m == 0 || n < 8) return p;
  // 256 or 128 rows of x per tile where the product is large, which read W and its LDS tile less often;
  // else 64 or 32, which leave more blocks and fewer bytes of parts.  Measured, us, 64 / 128 / 256: 1000
  // x 10007 x 300 26 / 27 / 32; 4000 x 10000 x 256 42 / 38 / 48; 300 x 100000 x 768 80 / 72 / 80; 2000 x
  // 20000 x 1024 123 / 95 / 91; 4096 x 32768 x 512 223 / 160 / 145.
  // 256 columns, but 128 where such tiles, split to 4 steps each, leave compute units idle (100 x
  // 5000 x 512: 256 12.6 us, 128 10.8; 64 x 50000 x 1024 22.4 and 22.4; 1 x 200003 x 1024 32 and 35).
  p.bk = k > 128 ? 256 : 128;
  // An FP32 dy has three tiles of its rows in LDS, and products, for each: 64 rows.
  const double products = double(m) * double(n) * k;
  p.bm = m <= 32 ? 32 : m <= 64 || products <= 7e9 || !y_bf16 ? 64 : products <= 3e10 ? 128 : 256;
  p.mtiles = uint32_t((m + p.bm - 1) / p.bm);
  const int64_t steps = (n + kRows - 1) / kRows;
  if (p.bm < 128 && steps / 4 * p.mtiles * ((k + 255) / 256) < kNumCu) p.bk = 128;
  p.ktiles = uint32_t((k + p.bk - 1) / p.bk);
  const int64_t tiles = int64_t(p.ktiles) * p.mtiles;
  // One block per compute unit, two where their LDS lets them share it.
  const int stage = (y_bf16 ? 1 : 3) * p.bm * kYRow + kRows * (p.bk * 2 + 32);
  int64_t splits = kNumCu * (4 * stage <= 160 * 1024 ? 2 : 1) / tiles;
  if (splits > steps / 4) splits = steps / 4;
  if (splits < 1) splits = 1;
  // (Ranges of rows fit 31 bits.)
  while (steps / splits > (int64_t(1) << 24)) ++splits;
  p.per = int32_t((steps + splits - 1) / splits);
  p.splits = uint32_t((steps + p.per - 1) / p.per);
  return p;
}

template <int TK, int TM, int WK, int WM, class TY, class TX>
void launch_tile(const GradPlan& p, const void* dy, int64_t ldy, int32_t m, const Mx4View& w,
                 TX* dx, int64_t ldx, int64_t part_stride, hipStream_t st) {
  auto kernel = grad_tile<TK, TM, WK, WM, TY, TX>;
  constexpr int lds = 2 * kStage<32 * TK * WK, 32 * TM * WM, sizeof(TY) == 4 ? 3 : 1>;
  if (lds > 65536)
    (void)hipFuncSetAttribute(reinterpret_cast<const void*>(kernel),
                              hipFuncAttributeMaxDynamicSharedMemorySize, lds);
  for_launches(int64_t(p.ktiles) * p.mtiles * p.splits, kBlock, [&](uint32_t first, dim3 grid) {
    hipLaunchKernelGGL(kernel, grid, dim3(kBlock), lds, st, static_cast<const TY*>(dy), ldy, m, w,
                       p.ktiles, p.mtiles, p.per, dx, ldx, part_stride, first);
  });
}

template <class TY, class TX>
void launch_plan(const GradPlan& p, const void* dy, int64_t ldy, int32_t m, const Mx4View& w,
                 TX* dx, int64_t ldx, int64_t ps, hipStream_t st) {
  if constexpr (sizeof(TY) == 2) {
    if (p.bm == 256 && p.bk == 256)
      return launch_tile<4, 4, 2, 2, TY>(p, dy, ldy, m, w, dx, ldx, ps, st);
    if (p.bm == 256) return launch_tile<2, 4, 2, 2, TY>(p, dy, ldy, m, w, dx, ldx, ps, st);
    if (p.bm == 128 && p.bk == 256)
      return launch_tile<2, 4, 4, 1, TY>(p, dy, ldy, m, w, dx, ldx, ps, st);
    if (p.bm == 128) return launch_tile<1, 4, 4, 1, TY>(p, dy, ldy, m, w, dx, ldx, ps, st);
  }
  if (p.bm == 64 && p.bk == 256)
    launch_tile<2, 2, 4, 1, TY>(p, dy, ldy, m, w, dx, ldx, ps, st);
  else if (p.bm == 64)
    launch_tile<1, 2, 4, 1, TY>(p, dy, ldy, m, w, dx, ldx, ps, st);
  else if (p.bk == 256)
    launch_tile<2, 1, 4, 1, TY>(p, dy, ldy, m, w, dx, ldx, ps, st);
  else
    launch_tile<1, 1, 4, 1, TY>(p, dy, ldy, m, w, dx, ldx, ps, st);
}

template <class TX>
void launch_grad(const GradPlan& p, const void* dy, bool dy_bf16, int64_t ldy, int32_t m,
                 const Mx4View& w, TX* dx, int64_t ldx, float* parts, hipStream_t st) {
  if (p.splits == 0) {  // fewer than 8 rows
    const int64_t blocks = (int64_t(m) * (w.dim / 4) + kBlock - 1) / kBlock;
    for_launches(blocks, kBlock, [&](uint32_t first, dim3 grid) {
      if (dy_bf16)
        hipLaunchKernelGGL((grad_few<__bf16, TX>), grid, dim3(kBlock), 0, st,
                           static_cast<const __bf16*>(dy), ldy, m, w, dx, ldx, first);
      else
        hipLaunchKernelGGL((grad_few<float, TX>), grid, dim3(kBlock), 0, st,
                           static_cast<const float*>(dy), ldy, m, w, dx, ldx, first);
    });
    return;
  }
  if (p.splits == 1) {
    if (dy_bf16)
      launch_plan<__bf16>(p, dy, ldy, m, w, dx, ldx, 0, st);
    else
      launch_plan<float>(p, dy, ldy, m, w, dx, ldx, 0, st);
    return;
  }
  const int64_t ps = int64_t(m) * w.dim;
  if (dy_bf16)
    launch_plan<__bf16>(p, dy, ldy, m, w, parts, w.dim, ps, st);
  else
    launch_plan<float>(p, dy, ldy, m, w, parts, w.dim, ps, st);
  const int64_t n = ps / 4;
  if (p.splits > 8) {
    hipLaunchKernelGGL(grad_join_many<TX>, dim3(unsigned((n + kWave - 1) / kWave)), dim3(1024), 0, st,
                       parts, int32_t(p.splits), m, fast_div(uint32_t(w.dim / 4)), dx, ldx);
    return;
  }
  hipLaunchKernelGGL(grad_join<TX>, dim3(unsigned((n + kBlock - 1) / kBlock)), dim3(kBlock), 0, st,
                     parts, int32_t(p.splits), m, fast_div(uint32_t(w.dim / 4)), dx, ldx);
}

}  // namespace

size_t mx4_matmul_grad_workspace(int32_t m, int64_t n, int32_t k) {
  const uint32_t splits = max(grad_plan(m, n, k, true).splits, grad_plan(m, n, k, false).splits);
  return splits > 1 ? (size_t(splits) * size_t(m) * size_t(k) * 4 + 255) / 256 * 256 : 0;
}

hipError_t launch_mx4_matmul_grad(const void* dy, bool dy_bf16, int64_t dy_stride, int32_t m,
                                  const Mx4View& w, void* dx, bool dx_bf16, int64_t dx_stride,
                                  char* ws, hipStream_t st) {
  if (m == 0) return hipSuccess;
  const GradPlan p = grad_plan(m, w.rows, w.dim, dy_bf16);
  float* parts = reinterpret_cast<float*>(ws);
  if (dx_bf16)
    launch_grad(p, dy, dy_bf16, dy_stride, m, w, static_cast<__bf16*>(dx), dx_stride, parts, st);
  else
    launch_grad(p, dy, dy_bf16, dy_stride, m, w, static_cast<float*>(dx), dx_stride, parts, st);
  return hipGetLastError();
}

}  // namespace embbag
