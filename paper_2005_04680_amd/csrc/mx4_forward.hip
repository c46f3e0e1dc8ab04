// Pooled forward (Algorithm 1 with Section II's weights or mean) from 4-bit
// microscaled tables.
//
// A row of E elements is nb = ceil(E/32) blocks of 16 bytes; LPR lanes read it, 8
// bytes (16 elements, half a block) and their block's scale byte each, so a
// wavefront holds 64/LPR rows at once.  `split` row groups share a bag: group j
// takes its look-ups j, j + split, ..., and their sums are added in a fixed tree.
// A lane converts its codes with the block's scale in the conversion (exact) and
// sums in FP32: 16 additions per look-up are what the vector units do here, and FP64
// ones would take twice the time of the bytes.  The order of the additions follows
// from the sizes alone.
//
// Bound by the row reads and these additions about alike: 6.6M look-ups of E = 256 140 us (0.9 GB
// of codes and scales, 6.4 TB/s with what the L2s hold).  Each XCD walks its own range of bags, so
// that a table's hot rows stay in one L2 (8 tables of 1M x 64, 819K look-ups: 14.6 us,
// in dispatch order 18.4).  16 elements per lane and 4 rows in flight were the best of 16 or 32
// and 4 or 8 (9000 weighted bags of 40, E = 100: 12.4, 15.3, 13.5, 17.3).
#include <type_traits>

#include "head.hpp"

namespace embbag {
namespace {

constexpr int kEl = 16;  // elements per lane

template <int LPR, int MODE, class T>
__global__ __launch_bounds__(kBlock) void mx4_forward_kernel(
    TableDesc d, const int32_t* __restrict__ I, const int32_t* __restrict__ O, int32_t NS,
    int32_t B, float inv_b, int32_t split, int32_t bags, T* __restrict__ Y,
    int32_t* __restrict__ status, const float* __restrict__ A) {
  constexpr int R = kWave / LPR;
  constexpr int U = 4;  // rows in flight per lane
  __shared__ TableLds tl;
  stage_tables(d, tl);
  __syncthreads();
  const int lane = lane_id();
  const int rg = lane / LPR, rl = lane % LPR;
  const int per_wave = R / split;  // bags of a wavefront
  const int64_t first =
      (int64_t(xcd_remap(blockIdx.x, gridDim.x)) * (blockDim.x / kWave) + wave_id()) * per_wave;
  const int64_t k64 = first + rg / split;
  const bool live = k64 < bags;
  const int k = live ? int(k64) : bags - 1;
  const int part = rg % split;
  const int t = table_of_bag(uint32_t(k), B, inv_b);
  const uint32_t M = tl.rowbase[t + 1] - tl.rowbase[t];
  const int nb = mx4_blocks(d.dim);
  const int sb = mx4_scale_bytes(d.dim);
  const uint32_t row_bytes = uint32_t(nb) * 16u;
  const auto* codes = table_elem<const uint8_t, uint8_t>(tl.w[t], 0);
  const auto* scales = table_elem<const uint8_t, uint8_t>(tl.lo[t], 0);
  // Lanes past the row's end re-read its last half block.
  const int half = min(rl, nb * 2 - 1);

  int err = 0;
  int s0 = O[k], s1 = O[k + 1];
  if (s0 < 0 || s1 > NS || s0 > s1 || (k == 0 && s0 != 0) || (k == bags - 1 && s1 != NS)) {
    err = EMBBAG_ERR_OFFSETS;
    s0 = s1 = 0;
  }
  const int n = s1 - s0;
  float acc[kEl];
#pragma unroll
  for (int i = 0; i < kEl; ++i) acc[i] = 0.f;

  // Look-up s0 + part + split * i for i = 0 .. mine - 1; past them a slot reads its
  // group's last look-up again and adds nothing.
  // (Unsigned: a bag may hold 2^31 - 1 look-ups.)
  const uint32_t step = uint32_t(split), from = uint32_t(s0 + part);
  const uint32_t mine = n > part ? (uint32_t(n - part) + step - 1u) / step : 0u;
  auto index_at = [&](uint32_t i) { return I[from + step * min(i, mine - 1u)]; };
  int idx[U];
  if (mine > 0) {
#pragma unroll
    for (int u = 0; u < U; ++u) idx[u] = index_at(uint32_t(u));
  }
  // A batch of U look-ups from number i on, of which all exist where `kAll`.  An index outside
  // its table reads row 0 (the output is unspecified then).
  auto batch = [&](uint32_t i, auto all) {
    constexpr bool kAll = decltype(all)::value;
    u2 v[U];
    uint32_t sc[U];
    float a[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const bool ok = uint32_t(idx[u]) < M;
      if (!ok) err = min(err, EMBBAG_ERR_INDEX_RANGE);
      const uint64_t row = ok ? uint32_t(idx[u]) : 0u;
      v[u] = *(const __attribute__((address_space(1))) u2*)(codes + (row * row_bytes + half * 8));
      sc[u] = scales[row * uint32_t(sb) + half / 2];
      if constexpr (MODE == kPoolWeighted) a[u] = A[from + step * (kAll ? i + u : min(i + u, mine - 1u))];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) idx[u] = index_at(i + U + u);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      // A slot past the bag's end must not add NaN either: its codes and scale become 0.
      const bool use = kAll || i + u < mine;
      const float s = mx4_scale(use ? sc[u] : 0u);
      float x[8], y[8];
      mx4_values8(use ? v[u].x : 0u, s, x);
      mx4_values8(use ? v[u].y : 0u, s, y);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if constexpr (MODE == kPoolWeighted) {
          const float w = use ? a[u] : 0.f;
          acc[e] = fmaf(w, x[e], acc[e]);
          acc[8 + e] = fmaf(w, y[e], acc[8 + e]);
        } else {
          acc[e] += x[e];
          acc[8 + e] += y[e];
        }
      }
    }
  };
  uint32_t i = 0;
  for (; i + U <= mine; i += U) batch(i, std::true_type{});
  if (i < mine) batch(i, std::false_type{});
  for (int j = LPR; j < LPR * split; j *= 2) {
#pragma unroll
    for (int e = 0; e < kEl; ++e) acc[e] += __shfl_xor(acc[e], j, kWave);
  }
  if (live && part == 0) {
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const int e0 = rl * kEl + c * 4;
      f4 r = {acc[c * 4], acc[c * 4 + 1], acc[c * 4 + 2], acc[c * 4 + 3]};
      if constexpr (MODE == kPoolMean) {
        if (n > 0) r = r / float(n);
      }
      if (e0 < d.dim) store4(Y + int64_t(k) * d.dim + e0, r);
    }
  }
  if (live && err != 0 && rl == 0 && status != nullptr) atomicMin(status, err);
}

// T*B == 0: the only data check left is offsets[0] == 0 == num_indices.
__global__ void mx4_empty_check(const int32_t* __restrict__ O, int32_t NS,
                                int32_t* __restrict__ status) {
  if (threadIdx.x == 0 && status != nullptr && (O[0] != 0 || NS != 0))
    atomicMin(status, EMBBAG_ERR_OFFSETS);
}

template <int MODE, class T>
void dispatch(int lpr, dim3 grid, hipStream_t st, const TableDesc& d, const int32_t* I,
              const int32_t* O, int32_t NS, int32_t B, int32_t split, int32_t bags, T* Y,
              int32_t* status, const float* A) {
  const float inv_b = 1.f / float(B);
#define EMB_MX4(L)                                                                             \
  case L:                                                                                      \
    hipLaunchKernelGGL((mx4_forward_kernel<L, MODE, T>), grid, dim3(kBlock), 0, st, d, I, O, NS, \
                       B, inv_b, split, bags, Y, status, A);                                   \
    break
  switch (lpr) {
    EMB_MX4(2);
    EMB_MX4(4);
    EMB_MX4(8);
    EMB_MX4(16);
    EMB_MX4(32);
    EMB_MX4(64);
  }
#undef EMB_MX4
}

template <class T>
void dispatch_mode(int mode, int lpr, dim3 grid, hipStream_t st, const TableDesc& d,
                   const int32_t* I, const int32_t* O, int32_t NS, int32_t B, int32_t split,
                   int32_t bags, T* Y, int32_t* status, const float* A) {
  if (mode == kPoolWeighted)
    dispatch<kPoolWeighted>(lpr, grid, st, d, I, O, NS, B, split, bags, Y, status, A);
  else if (mode == kPoolMean)
    dispatch<kPoolMean>(lpr, grid, st, d, I, O, NS, B, split, bags, Y, status, A);
  else
    dispatch<kPoolPlain>(lpr, grid, st, d, I, O, NS, B, split, bags, Y, status, A);
}

}  // namespace

hipError_t launch_mx4_forward(const TableDesc& d, int32_t B, const int32_t* I, const int32_t* O,
                              int64_t NS, void* Y, bool y_bf16, int32_t* status,
                              const PoolArgs& pool, hipStream_t st) {
  const int64_t bags = int64_t(d.num_tables) * B;
  if (bags == 0) {
    hipLaunchKernelGGL(mx4_empty_check, dim3(1), dim3(kWave), 0, st, O, int32_t(NS), status);
    return hipGetLastError();
  }
  int lpr = 2;
  while (lpr < mx4_blocks(d.dim) * 2) lpr *= 2;
  const int groups = kWave / lpr;
  // Groups that share a bag: two for 9 look-ups or more, four for 17 and so on, while the
  // wavefronts do not fill the chip's slots.  Measured, us, shared / not: 512 bags of 32, E = 64
  // 7.5 / 10.8; 64 of 100, E = 1024 12.3 / 17.2; 9000 of 40, E = 100, weighted 12.4 / 15.3; 33K of 10,
  // E = 16, shared by four 9.6, not 8.1.
  const int64_t avg = NS / bags;
  int split = 1;
  while (split < groups && avg > int64_t(split) * 8 && bags * split * lpr < int64_t(kNumCu) * 32 * kWave)
    split *= 2;
  const int64_t per_block = int64_t(kWavesPerBlock) * (groups / split);
  const dim3 grid(unsigned((bags + per_block - 1) / per_block));
  if (y_bf16)
    dispatch_mode(pool.mode, lpr, grid, st, d, I, O, int32_t(NS), B, split, int32_t(bags),
                  static_cast<__bf16*>(Y), status, pool.weights);
  else
    dispatch_mode(pool.mode, lpr, grid, st, d, I, O, int32_t(NS), B, split, int32_t(bags),
                  static_cast<float*>(Y), status, pool.weights);
  return hipGetLastError();
}

}  // namespace embbag
