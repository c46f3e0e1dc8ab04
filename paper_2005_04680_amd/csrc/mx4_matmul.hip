// Scores of all rows of a 4-bit microscaled table: out = q(x) W^T.
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

// x rounded to the storage of the table: codes [m][groups2 * 64], rows of whole steps of
// 256 elements (zeros past k), scales as words of 4 blocks [groups][m].  Four lanes per block, as
// mx4_quantize.  Blocks from `xblocks` on copy W's scales to words [groups][n].
template <class T>
__global__ __launch_bounds__(kBlock) void pack_x(const T* __restrict__ x, int64_t stride, int32_t m,
                                                 int32_t k, FastDiv groups2, int32_t groups,
                                                 uint8_t* __restrict__ codes,
                                                 uint8_t* __restrict__ scales, uint32_t xblocks,
                                                 const uint32_t* __restrict__ ws, int64_t n,
                                                 uint32_t* __restrict__ ws_out) {
  if (blockIdx.x >= xblocks) {
    // 64 rows, a quarter of the groups for each wavefront, 4 groups at a time.
    const int64_t row = int64_t(blockIdx.x - xblocks) * kWave + lane_id();
    if (row >= n) return;
    const uint32_t* src = ws + row * groups;
    for (int g = wave_id() * 4; g < groups; g += kWavesPerBlock * 4) {
      uint32_t v[4];
      if (groups % 4 == 0) {
        const u4 q = *reinterpret_cast<const u4_word*>(src + g);
        v[0] = q.x, v[1] = q.y, v[2] = q.z, v[3] = q.w;
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = g + i < groups ? src[g + i] : 0u;
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (g + i < groups) ws_out[(g + i) * n + row] = v[i];
    }
    return;
  }
  const int64_t u = int64_t(blockIdx.x) * (kBlock / 4) + threadIdx.x / 4;
  const int part = threadIdx.x % 4;
  const int64_t g4 = u / 4;
  if (g4 >= int64_t(m) * groups2.div) return;
  const uint32_t row = quotient(uint32_t(g4), groups2);
  const int g = int(uint32_t(g4) - row * groups2.div), j = int(u % 4);
  const int e0 = g * 128 + j * kMxBlock + part * 8;
  const T* p = x + int64_t(row) * stride + e0;
  const f4 zero = {0.f, 0.f, 0.f, 0.f};
  const f4 x0 = e0 < k ? load4(p) : zero;
  const f4 x1 = e0 + 4 < k ? load4(p + 4) : zero;
  float y[8] = {x0.x, x0.y, x0.z, x0.w, x1.x, x1.y, x1.z, x1.w};
  uint32_t amax = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) amax = max(amax, __float_as_uint(y[i]) & 0x7FFFFFFFu);
  amax = max(amax, uint32_t(__shfl_xor(int(amax), 1, 4)));
  amax = max(amax, uint32_t(__shfl_xor(int(amax), 2, 4)));
  float factor;
  const uint32_t byte = mx4_scale_of(amax, &factor);
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] *= factor;
  const uint32_t c = byte == 255u ? 0u : mx4_codes8(y);
  *reinterpret_cast<uint32_t*>(codes + (int64_t(row) * groups2.div + g) * 64 + j * 16 + part * 4) = c;
  if (part == 0 && g < groups) scales[(int64_t(g) * m + row) * 4 + j] = uint8_t(byte);
}

constexpr int kStepBytes = 128;  // a row's codes per step: 256 elements, 8 blocks

// 16 bytes per lane from memory to LDS, lane l's at `dst` + 16 l.
__device__ __forceinline__ void to_lds16(const uint8_t* src, uint8_t* dst) {
  __builtin_amdgcn_global_load_lds(
      (const __attribute__((address_space(1))) void*)src,
      (__attribute__((address_space(3))) void*)dst, 16, 0, 0);
}

// Until this wavefront's loads to LDS and reads from it are complete.
__device__ __forceinline__ void wait_loads() {
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
}

// A BN x BM tile of out^T (BN rows of W, BM of x); WN x WM wavefronts, each TN x TM
// products of 32 x 32.
//
// Per step of 256 elements the tile's codes go from memory to LDS, double-buffered: a
// wavefront's load brings 8 rows of 128 bytes, and the lane of row r and place j fetches
// block j ^ (r % 8), so that the fragments' reads (32 rows, one block) spread over the
// banks.  Lane l's row is l % 32; product j of a step takes block 4 (l / 32) + j, whose
// scale is byte j of the word of group 2 * step + l / 32.
template <int TN, int TM, int WN, int WM, class T>
__global__ __launch_bounds__(WN* WM* kWave, 1) void scores_tile(
    const uint8_t* __restrict__ xc, const uint32_t* __restrict__ xs, int32_t m, int32_t groups,
    Mx4View w, const uint32_t* __restrict__ ws, int64_t ws_row, int64_t ws_group, uint32_t mtiles,
    T* __restrict__ out, int64_t ldo) {
  constexpr int BN = 32 * TN * WN, BM = 32 * TM * WM, W = WN * WM;
  constexpr int LOADS = (BN + BM) / 8 / W;  // per wavefront and step
  static_assert((BN + BM) % (8 * W) == 0 && BN % 8 == 0, "whole loads");
  constexpr int STAGE = (BN + BM) * kStepBytes;
  extern __shared__ __align__(16) uint8_t lds[];

  const int lane = lane_id(), wave = wave_id();
  const uint32_t tile = xcd_remap(blockIdx.x, gridDim.x);
  const uint32_t nt = tile / mtiles, mt = tile - nt * mtiles;
  const int64_t n0 = int64_t(nt) * BN;
  const int m0 = int(mt) * BM;
  const int nb = mx4_blocks(w.dim);
  const int steps = (groups + 1) / 2;
  const int64_t xrow = int64_t(steps) * kStepBytes, wrow = int64_t(nb) * 16;

  // Loads: number i of this wavefront brings rows 8 * (i * W + wave) .. + 7 of the stage (W's
  // rows, then x's); rows past the end repeat the last one.
  const int c = (lane % 8) ^ (lane / 8);
  const uint8_t* wbase = w.codes + n0 * wrow;
  const uint8_t* xbase = xc + int64_t(m0) * xrow;
  uint32_t off[LOADS];
#pragma unroll
  for (int i = 0; i < LOADS; ++i) {
    const int r = 8 * (i * W + wave) + lane / 8;
    off[i] = r < BN ? uint32_t(min(int64_t(r), w.rows - 1 - n0) * wrow)
                    : uint32_t(min(r - BN, m - 1 - m0) * xrow + c * 16);
  }
  auto load = [&](int step, uint8_t* dst) {
    // (A block past W's row is its last one: x's codes are 0 there.)
    const uint32_t wk = uint32_t(min(step * 8 + c, nb - 1)) * 16;
    const uint32_t xk = uint32_t(step) * kStepBytes;
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int r0 = 8 * (i * W + wave);
      const uint8_t* src = r0 < BN ? wbase + (off[i] + wk) : xbase + (off[i] + xk);
      to_lds16(src, dst + r0 * kStepBytes);
    }
  };

  const int wn = wave % WN, wm = wave / WN;
  const int half = lane / 32, row = lane % 32;
  const uint32_t* wsp[TN];
  const uint32_t* xsp[TM];
#pragma unroll
  for (int i = 0; i < TN; ++i)
    wsp[i] = ws + min(n0 + (wn * TN + i) * 32 + row, w.rows - 1) * ws_row;
#pragma unroll
  for (int i = 0; i < TM; ++i) xsp[i] = xs + min(m0 + (wm * TM + i) * 32 + row, m - 1);
  uint32_t sw[TN], sx[TM];
  auto load_scales = [&](int step) {
    const int g = 2 * step + half;
    const int64_t gc = min(g, groups - 1);
#pragma unroll
    for (int i = 0; i < TN; ++i) sw[i] = wsp[i][gc * ws_group];
#pragma unroll
    for (int i = 0; i < TM; ++i) sx[i] = xsp[i][gc * m];
    // (Past the last group x's codes are 0: a scale of 0 keeps W's NaN out.)
    if (g >= groups) {
#pragma unroll
      for (int i = 0; i < TN; ++i) sw[i] = 0u;
    }
  };

  f16v acc[TN][TM];
#pragma unroll
  for (int i = 0; i < TN; ++i)
#pragma unroll
    for (int j = 0; j < TM; ++j) acc[i][j] = f16v{};

  load(0, lds);
  load_scales(0);
  const int frag_w = (wn * TN * 32 + row) * kStepBytes;
  const int frag_x = (BN + wm * TM * 32 + row) * kStepBytes;
  const int at0 = ((4 * half) ^ (row & 7)) * 16;  // place of part j's block: at0 ^ (16 j)
  u4 a[2][TN] = {}, b[2][TM] = {};
  uint32_t cw[TN] = {}, cx[TM] = {};
  // The fragments of a part arrive while the products of the part before are issued, those of a
  // step's first part during the last part of the step before.  The next step's codes go to
  // `nxt`, not the memory of `cur`: the reads need not wait for those loads.
  auto fetch = [&](const uint8_t* __restrict__ cur, int j) {
#pragma unroll
    for (int i = 0; i < TN; ++i)
      a[j & 1][i] = *reinterpret_cast<const u4*>(cur + frag_w + i * 32 * kStepBytes + (at0 ^ (16 * j)));
#pragma unroll
    for (int i = 0; i < TM; ++i)
      b[j & 1][i] = *reinterpret_cast<const u4*>(cur + frag_x + i * 32 * kStepBytes + (at0 ^ (16 * j)));
    __builtin_amdgcn_sched_barrier(0);
  };
#define EMB_ROW(J, I)                                                                        \
  _Pragma("unroll") for (int j = 0; j < TM; ++j) acc[I][j] =                                 \
      __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(frag8(a[J & 1][I]), frag8(b[J & 1][j]), \
                                                      acc[I][j], 4, 4, J, int(cw[I]), J,     \
                                                      int(cx[j]));
// (The reads come after the first products: the wait for those products' fragments is
// then no wait for the reads.)
#define EMB_PART(J, READS)                                                                   \
  {                                                                                          \
    EMB_ROW(J, 0)                                                                            \
    __builtin_amdgcn_sched_barrier(0);                                                       \
    READS;                                                                                   \
    __builtin_amdgcn_sched_barrier(0);                                                       \
    _Pragma("unroll") for (int i = 1; i < TN; ++i) { EMB_ROW(J, i) }                         \
    __builtin_amdgcn_sched_barrier(0);                                                       \
  }
  auto step_of = [&](const uint8_t* __restrict__ cur, uint8_t* __restrict__ nxt, int step) {
    if (step + 1 < steps) load(step + 1, nxt);
    EMB_PART(3, fetch(cur, 0))
#pragma unroll
    for (int i = 0; i < TN; ++i) cw[i] = sw[i];
#pragma unroll
    for (int i = 0; i < TM; ++i) cx[i] = sx[i];
    load_scales(min(step + 1, steps - 1));
    EMB_PART(0, fetch(cur, 1))
    EMB_PART(1, fetch(cur, 2))
    EMB_PART(2, fetch(cur, 3))
  };
  for (int step = 0; step < steps; ++step) {
    // This step's codes are in LDS, and every wavefront holds the last fragments of the
    // other stage.
    wait_loads();
    __syncthreads();
    step_of(lds + (step & 1) * STAGE, lds + (~step & 1) * STAGE, step);
  }
  EMB_PART(3, )
#undef EMB_PART
#undef EMB_ROW

  // Each wavefront turns 32 rows of x at a time around in LDS (lane: row of x lane % 32, four
  // consecutive rows of W per quarter of its registers), then stores whole rows.
  constexpr int COLS = 32 * TN;
  constexpr int V = kVec<T>;
  constexpr int PITCH = COLS + V;
  T* turn = reinterpret_cast<T*>(lds) + wave * 32 * PITCH;
  const int64_t nw = n0 + wn * COLS;
#pragma unroll
  for (int j = 0; j < TM; ++j) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < TN; ++i)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        store4(turn + row * PITCH + i * 32 + q * 8 + half * 4,
               f4{acc[i][j][q * 4], acc[i][j][q * 4 + 1], acc[i][j][q * 4 + 2],
                  acc[i][j][q * 4 + 3]});
    __syncthreads();
    constexpr int PER_ROW = COLS / V, ROWS = kWave / PER_ROW;
#pragma unroll
    for (int r0 = 0; r0 < 32; r0 += ROWS) {
      const int r = r0 + lane / PER_ROW, col = lane % PER_ROW * V;
      const int mm = m0 + (wm * TM + j) * 32 + r;
      if (mm >= m || nw + col >= w.rows) continue;
      T* p = out + int64_t(mm) * ldo + nw + col;
      const T* q = turn + r * PITCH + col;
      if (nw + col + V <= w.rows) {
        const u4 v = *reinterpret_cast<const u4*>(q);
        store16(p, v);
      } else {
        for (int e = 0; e < V && nw + col + e < w.rows; ++e) p[e] = q[e];
      }
    }
  }
}

// One wavefront per 16 rows of W and 16 of x, straight from memory: lane l holds
// row l % 16, and of every 4 groups of 128 elements the group l / 16; the four blocks
// of its group go through four products whose scales are the bytes of one word.
template <class T>
__global__ __launch_bounds__(kBlock) void scores_direct(const uint8_t* __restrict__ xc,
                                                        const uint32_t* __restrict__ xs,
                                                        Mx4View w, int32_t m, int32_t groups,
                                                        uint32_t ntiles, T* __restrict__ out,
                                                        int64_t ldo) {
  const int lane = lane_id(), r = lane % 16, q = lane / 16;
  const uint32_t nt = blockIdx.x % ntiles, mt = blockIdx.x / ntiles;
  const int64_t n0 = (int64_t(nt) * kWavesPerBlock + wave_id()) * 16;
  if (n0 >= w.rows) return;
  const int m0 = int(mt) * 16;
  const int nb = mx4_blocks(w.dim);
  const int64_t wn = min(n0 + r, w.rows - 1);
  const int xm = min(m0 + r, m - 1);
  const uint8_t* wc = w.codes + wn * nb * 16;
  const uint32_t* wsc = reinterpret_cast<const uint32_t*>(w.scales) + wn * groups;
  const uint8_t* xcr = xc + int64_t(xm) * ((groups + 1) / 2) * kStepBytes;
  f4 c = {0.f, 0.f, 0.f, 0.f};
  for (int g0 = 0; g0 < groups; g0 += 4) {
    const int g = g0 + q;
    const bool in = g < groups;
    const uint32_t sw = in ? wsc[g] : 0u;
    const uint32_t sx = in ? xs[int64_t(g) * m + xm] : 0u;
    u4 a[4], b[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const u4 none = {0u, 0u, 0u, 0u};
      a[j] = in ? *reinterpret_cast<const u4*>(xcr + (g * 4 + j) * 16) : none;
      b[j] = g * 4 + j < nb ? *reinterpret_cast<const u4*>(wc + (g * 4 + j) * 16) : none;
    }
#define EMB_MFMA(J)                                                                       \
  {                                                                                       \
    const i8v av = {int(a[J].x), int(a[J].y), int(a[J].z), int(a[J].w), 0, 0, 0, 0};      \
    const i8v bv = {int(b[J].x), int(b[J].y), int(b[J].z), int(b[J].w), 0, 0, 0, 0};      \
    c = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(av, bv, c, 4, 4, J, int(sx), J,  \
                                                         int(sw));                        \
  }
    EMB_MFMA(0);
    EMB_MFMA(1);
    EMB_MFMA(2);
    EMB_MFMA(3);
#undef EMB_MFMA
  }
  const int64_t n = n0 + r;
  if (n >= w.rows) return;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int mm = m0 + q * 4 + i;
    if (mm < m) out[int64_t(mm) * ldo + n] = T(c[i]);
  }
}

size_t align256(size_t x) { return (x + 255) / 256 * 256; }

}  // namespace

namespace {

struct ScoreLayout {
  size_t xs, ws, total;
};
ScoreLayout score_layout(int32_t m, int64_t n, int32_t k) {
  const size_t groups = size_t((k + 127) / 128);
  ScoreLayout L;
  L.xs = align256(size_t(m) * ((groups + 1) / 2) * kStepBytes);
  L.ws = L.xs + align256(size_t(m) * groups * 4);
  L.total = L.ws + align256(size_t(n) * groups * 4);
  return L;
}

template <int TN, int TM, int WN, int WM, class T>
void launch_tile(const uint8_t* xc, const uint32_t* xs, int32_t m, int32_t groups,
                 const Mx4View& w, const uint32_t* ws, int64_t ws_row, int64_t ws_group, T* out,
                 int64_t ldo, hipStream_t st) {
  constexpr int BN = 32 * TN * WN, BM = 32 * TM * WM;
  constexpr size_t stage = size_t(BN + BM) * kStepBytes;
  constexpr size_t turn = size_t(WN) * WM * 32 * (32 * TN + kVec<T>)*sizeof(T);
  constexpr size_t lds = 2 * stage > turn ? 2 * stage : turn;
  const uint32_t mtiles = uint32_t((m + BM - 1) / BM);
  const uint32_t ntiles = uint32_t((w.rows + BN - 1) / BN);
  auto kernel = scores_tile<TN, TM, WN, WM, T>;
  if (lds > 65536)
    (void)hipFuncSetAttribute(reinterpret_cast<const void*>(kernel),
                              hipFuncAttributeMaxDynamicSharedMemorySize, int(lds));
  hipLaunchKernelGGL(kernel, dim3(mtiles * ntiles), dim3(WN * WM * kWave), lds, st, xc, xs, m,
                     groups, w, ws, ws_row, ws_group, mtiles, out, ldo);
}

template <class T>
void launch_scores(const uint8_t* xc, const uint32_t* xs, const uint32_t* ws, int32_t m,
                   int32_t groups, const Mx4View& w, T* out, int64_t ldo, hipStream_t st) {
  if (m > 16) {
    launch_tile<4, 4, 2, 2>(xc, xs, m, groups, w, ws, 1, w.rows, out, ldo, st);
    return;
  }
  const uint32_t ntiles = uint32_t((w.rows + 63) / 64);
  const dim3 grid(ntiles * unsigned((m + 15) / 16));
  hipLaunchKernelGGL(scores_direct<T>, grid, dim3(kBlock), 0, st, xc, xs, w, m, groups, ntiles, out,
                     ldo);
}

}  // namespace

size_t mx4_matmul_workspace(int32_t m, int64_t n, int32_t k) { return score_layout(m, n, k).total; }

hipError_t launch_mx4_matmul(const void* x, bool x_bf16, int64_t x_stride, int32_t m,
                             const Mx4View& w, void* out, bool out_bf16, int64_t out_stride,
                             char* ws, hipStream_t st) {
  if (m == 0) return hipSuccess;
  const int groups = (w.dim + 127) / 128, groups2 = (groups + 1) / 2 * 2;
  const ScoreLayout L = score_layout(m, w.rows, w.dim);
  uint8_t* xc = reinterpret_cast<uint8_t*>(ws);
  uint8_t* xs = xc + L.xs;
  uint32_t* wst = reinterpret_cast<uint32_t*>(ws + L.ws);
  const uint32_t* wsc = reinterpret_cast<const uint32_t*>(w.scales);
  const int64_t units = int64_t(m) * groups2 * 4;
  const uint32_t xblocks = uint32_t((units + kBlock / 4 - 1) / (kBlock / 4));
  const uint32_t wblocks = m > 16 ? uint32_t((w.rows + kWave - 1) / kWave) : 0u;
  const dim3 pgrid(xblocks + wblocks);
  const FastDiv f = fast_div(uint32_t(groups2));
  if (x_bf16)
    hipLaunchKernelGGL(pack_x<__bf16>, pgrid, dim3(kBlock), 0, st, static_cast<const __bf16*>(x),
                       x_stride, m, w.dim, f, groups, xc, xs, xblocks, wsc, w.rows, wst);
  else
    hipLaunchKernelGGL(pack_x<float>, pgrid, dim3(kBlock), 0, st, static_cast<const float*>(x),
                       x_stride, m, w.dim, f, groups, xc, xs, xblocks, wsc, w.rows, wst);
  const uint32_t* xsw = reinterpret_cast<const uint32_t*>(xs);
  if (out_bf16)
    launch_scores(xc, xsw, wst, m, groups, w, static_cast<__bf16*>(out), out_stride, st);
  else
    launch_scores(xc, xsw, wst, m, groups, w, static_cast<float*>(out), out_stride, st);
  return hipGetLastError();
}

}  // namespace embbag
