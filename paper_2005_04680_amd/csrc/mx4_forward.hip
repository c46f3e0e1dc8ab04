// Pooled forward (Algorithm 1 with Section II's weights or mean) from 4-bit
// microscaled tables.
//
// A row of E elements is nb = ceil(E/32) blocks of 16 bytes with a scale byte each.  Lanes
// next to each other read a row, a wavefront several rows at once.  `split` row groups share a bag: group
// j takes its look-ups j, j + split, ..., and their sums are added in a fixed tree.  Sums are FP32;
// the order of the additions follows from the sizes alone.
//
// Sums and means go through the scaled matrix instructions, which take the stored bytes as they are
// (mx4_sum_kernel); 16 additions and 8 conversions per look-up and lane kept the vector units busy for four
// fifths of the time.  An FP32 weight per look-up is no power of two: weighted sums convert and add in the
// vector units (mx4_weighted_kernel).
//
// 6.6M look-ups of E = 256 123 us (in the vector units 141): bound by the rows, 0.9 GB of codes and scales, of
// which 0.52 GB miss the L2s, and 67 MB of outputs: 4.8 TB/s beyond the L2s.  Others, us, before and
// now: 26 tables, 8192 of 1, E = 128 40.4 / 27.2; 2 tables, 8192 of 100, E = 512 60 / 45; 64 of 100, E = 1024 13.1 /
// 8.4; 300 of 3000, E = 64 38.4 / 28.  Each XCD walks its own range of bags, so that a table's hot rows
// stay in one L2 (8 tables of 1M x 64, 819K look-ups, in the vector units: 14.6 us, in dispatch order 18.4).
#include <type_traits>

#include "head.hpp"

namespace embbag {
namespace {

typedef int i8v __attribute__((ext_vector_type(8)));
typedef float f16v __attribute__((ext_vector_type(16)));

constexpr int kEl = 16;  // elements per lane of the weighted sums

// Weighted sums.  LPR lanes read a row, 8 bytes (16 elements, half a block) and their block's scale byte
// each; a lane converts its codes with the block's scale in the conversion (exact) and adds with the
// weight.  16 elements per lane and 4 rows in flight were the best of 16 or 32 and 4 or 8 (9000 bags
// of 40, E = 100: 12.4, 15.3, 13.5, 17.3).
template <int LPR, class T>
__global__ __launch_bounds__(kBlock) void mx4_weighted_kernel(
    TableDesc d, const int32_t* __restrict__ I, const int32_t* __restrict__ O, int32_t NS,
    int32_t B, float inv_b, int32_t split, int32_t bags, T* __restrict__ Y,
    int32_t* __restrict__ status, const float* __restrict__ A, uint32_t first_block) {
  constexpr int R = kWave / LPR;
  constexpr int U = 4;  // rows in flight per lane
  __shared__ TableLds tl;
  stage_tables(d, tl);
  __syncthreads();
  const int lane = lane_id();
  const int rg = lane / LPR, rl = lane % LPR;
  const int per_wave = R / split;  // bags of a wavefront
  const int64_t first =
      (int64_t(first_block + xcd_remap(blockIdx.x, gridDim.x)) * (blockDim.x / kWave) + wave_id()) *
      per_wave;
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
      a[u] = A[from + step * (kAll ? i + u : min(i + u, mine - 1u))];
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
        const float w = use ? a[u] : 0.f;
        acc[e] = fmaf(w, x[e], acc[e]);
        acc[8 + e] = fmaf(w, y[e], acc[8 + e]);
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
      const f4 r = {acc[c * 4], acc[c * 4 + 1], acc[c * 4 + 2], acc[c * 4 + 3]};
      if (e0 < d.dim) store4(Y + int64_t(k) * d.dim + e0, r);
    }
  }
  if (live && err != 0 && rl == 0 && status != nullptr) atomicMin(status, err);
}

// Sums and means: a column of a scaled matrix product holds a block of 32 elements of a bag,
// D[e][c] += sum over k of A[e][k] B[k][c], where B's column is the codes of that block of two
// look-ups (k = 0 .. 31 and 32 .. 63, with a scale each) and A two identities side by side: the
// products are the elements, their sum is the bag's.  Lane l brings block l % P of its row group's
// look-up number 2 i + l / 32: 16 bytes and a scale; P lanes per row, 32 / P row groups.
template <int P, int U, int MODE, class T>
__global__ __launch_bounds__(kBlock) void mx4_sum_kernel(
    TableDesc d, const int32_t* __restrict__ I, const int32_t* __restrict__ O, int32_t NS,
    int32_t B, float inv_b, int32_t split, int32_t bags, T* __restrict__ Y,
    int32_t* __restrict__ status, uint32_t first_block) {
  constexpr int R = 32 / P;
  __shared__ TableLds tl;
  stage_tables(d, tl);
  __syncthreads();
  const int lane = lane_id();
  const int col = lane % 32, half = lane / 32;
  const int rg = col / P, b = col % P;
  const int per_wave = R / split;  // bags of a wavefront
  const int64_t first =
      (int64_t(first_block + xcd_remap(blockIdx.x, gridDim.x)) * (blockDim.x / kWave) + wave_id()) *
      per_wave;
  const int64_t k64 = first + rg / split;
  const bool live = k64 < bags;
  const int k = live ? int(k64) : bags - 1;
  const int part = rg % split;
  const int t = table_of_bag(uint32_t(k), B, inv_b);
  const uint32_t M = tl.rowbase[t + 1] - tl.rowbase[t];
  const int nb = mx4_blocks(d.dim);
  const int sb = mx4_scale_bytes(d.dim);
  // Lanes past the row's end re-read its last block.
  const int block = min(b, nb - 1);
  const auto* codes = table_elem<const uint8_t, uint8_t>(tl.w[t], 0) + block * 16;
  const auto* scales = table_elem<const uint8_t, uint8_t>(tl.lo[t], 0) + block;

  int err = 0;
  int s0 = O[k], s1 = O[k + 1];
  if (s0 < 0 || s1 > NS || s0 > s1 || (k == 0 && s0 != 0) || (k == bags - 1 && s1 != NS)) {
    err = EMBBAG_ERR_OFFSETS;
    s0 = s1 = 0;
  }
  const int n = s1 - s0;
  // This lane's look-ups are s0 + split * half + part + 2 split * i for i = 0 .. mine - 1; past them it
  // reads the last again and adds nothing.  (Unsigned: a bag may hold 2^31 - 1 look-ups.)
  const uint32_t step = 2u * uint32_t(split), skip = uint32_t(split * half + part);
  const uint32_t from = uint32_t(s0) + skip;
  const uint32_t mine = uint32_t(n) > skip ? (uint32_t(n) - skip + step - 1u) / step : 0u;
  auto index_at = [&](uint32_t i) { return I[from + step * min(i, mine - 1u)]; };
  int idx[U];
#pragma unroll
  for (int u = 0; u < U; ++u) idx[u] = mine > 0 ? index_at(uint32_t(u)) : 0;

  // The identity: element col of each half is 1 (code 2).
  i8v one = {};
#pragma unroll
  for (int q = 0; q < 4; ++q) one[q] = col / 8 == q ? 2 << (col % 8 * 4) : 0;
  f16v acc = {};
  // A batch of U look-ups from number i on, of which all exist in every lane where `kAll`.  An index
  // outside its table reads row 0 (the output is unspecified then).
  auto batch = [&](uint32_t i, auto all) {
    constexpr bool kAll = decltype(all)::value;
    u4 v[U];
    uint32_t sc[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const bool ok = uint32_t(idx[u]) < M;
      if (!ok) err = min(err, EMBBAG_ERR_INDEX_RANGE);
      const uint64_t row = ok ? uint32_t(idx[u]) : 0u;
      // (A slot past the bag's end must not add NaN either: its codes and scale are 0.)
      v[u] = u4{0u, 0u, 0u, 0u};
      sc[u] = 0u;
      if (kAll || i + u < mine) {
        v[u] = *(const __attribute__((address_space(1))) u4*)(codes + row * uint32_t(nb * 16));
        sc[u] = scales[row * uint32_t(sb)];
      }
    }
    if (kAll || i + U < mine) {
#pragma unroll
      for (int u = 0; u < U; ++u) idx[u] = index_at(i + U + u);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const i8v x = {int(v[u].x), int(v[u].y), int(v[u].z), int(v[u].w), 0, 0, 0, 0};
      acc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(one, x, acc, 4, 4, 0, 127, 0, int(sc[u]));
    }
  };
  // The products take all lanes: as many batches as the wavefront's longest list has.
  uint32_t least = mine, most = mine;
  for (int j = P; j < kWave; j *= 2) {
    least = min(least, uint32_t(__shfl_xor(int(least), j, kWave)));
    most = max(most, uint32_t(__shfl_xor(int(most), j, kWave)));
  }
  least = __builtin_amdgcn_readfirstlane(least);
  most = __builtin_amdgcn_readfirstlane(most);
  uint32_t i = 0;
  for (; i + U <= least; i += U) batch(i, std::true_type{});
  for (; i < most; i += U) batch(i, std::false_type{});

  for (int j = P; j < P * split; j *= 2) {
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[e] += __shfl_xor(acc[e], j, kWave);
  }
  if (live && part == 0) {
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const int e0 = b * 32 + c * 8 + half * 4;
      f4 r = {acc[c * 4], acc[c * 4 + 1], acc[c * 4 + 2], acc[c * 4 + 3]};
      if constexpr (MODE == kPoolMean) {
        if (n > 0) r = r / float(n);
      }
      if (e0 < d.dim) store4(Y + int64_t(k) * d.dim + e0, r);
    }
  }
  if (live && err != 0 && b == 0 && status != nullptr) atomicMin(status, err);
}

// T*B == 0: the only data check left is offsets[0] == 0 == num_indices.
__global__ void mx4_empty_check(const int32_t* __restrict__ O, int32_t NS,
                                int32_t* __restrict__ status) {
  if (threadIdx.x == 0 && status != nullptr && (O[0] != 0 || NS != 0))
    atomicMin(status, EMBBAG_ERR_OFFSETS);
}

template <int MODE, class T>
void dispatch(int lpr, bool four, dim3 grid, hipStream_t st, const TableDesc& d, const int32_t* I,
              const int32_t* O, int32_t NS, int32_t B, int32_t split, int32_t bags, T* Y,
              int32_t* status, const float* A, uint32_t first) {
  const float inv_b = 1.f / float(B);
#define EMB_MX4(L)                                                                               \
  case L:                                                                                        \
    if constexpr (MODE == kPoolWeighted)                                                         \
      hipLaunchKernelGGL((mx4_weighted_kernel<L, T>), grid, dim3(kBlock), 0, st, d, I, O,   \
                         NS, B, inv_b, split, bags, Y, status, A, first);                        \
    else if (four)                                                                               \
      hipLaunchKernelGGL((mx4_sum_kernel<L / 2, 4, MODE, T>), grid, dim3(kBlock), 0, \
                         st, d, I, O, NS, B, inv_b, split, bags, Y, status, first);              \
    else                                                                                         \
      hipLaunchKernelGGL((mx4_sum_kernel<L / 2, 2, MODE, T>), grid, dim3(kBlock), 0, st, d, I,   \
                         O, NS, B, inv_b, split, bags, Y, status, first);                        \
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
void dispatch_mode(int mode, int lpr, bool four, dim3 grid, hipStream_t st, const TableDesc& d,
                   const int32_t* I, const int32_t* O, int32_t NS, int32_t B, int32_t split,
                   int32_t bags, T* Y, int32_t* status, const float* A, uint32_t first) {
  if (mode == kPoolWeighted)
    dispatch<kPoolWeighted>(lpr, four, grid, st, d, I, O, NS, B, split, bags, Y, status, A, first);
  else if (mode == kPoolMean)
    dispatch<kPoolMean>(lpr, four, grid, st, d, I, O, NS, B, split, bags, Y, status, A, first);
  else
    dispatch<kPoolPlain>(lpr, four, grid, st, d, I, O, NS, B, split, bags, Y, status, A, first);
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
  // Groups that share a bag: two for `list` look-ups or more each, four for twice that and so on, while
  // the wavefronts do not fill the chip's slots.  Lists of 8, but of 16 in the sums, which take two
  // look-ups at a time, once there are two wavefronts for each vector unit.  Measured, us, 8 / 16: 64
  // ragged bags of 32 in each of 8 tables, E = 64 5.4 / 6.2; 9000 of 40, E = 100 11.7 / 9.5; 8 x 2048
  // ragged of 32, E = 128 11.5 / 10.4.
  const int64_t avg = NS / bags;
  int split = 1;
  auto few = [&]() { return bags * split * lpr < int64_t(kNumCu) * 8 * kWave; };
  auto list = [&]() { return pool.mode == kPoolWeighted || few() ? 8 : 16; };
  while (split < groups && avg > split * list() && bags * split * lpr < int64_t(kNumCu) * 32 * kWave)
    split *= 2;
  // Rows in flight per lane of the sums: four, two where lists are short or rows narrow (which leaves
  // more wavefronts on a unit) unless there are few.  Measured, us, four / two: 8 tables, 8192 bags of
  // 100, E = 256 123.5 / 127; 26 tables, 8192 of 1, E = 128 30.5 / 27.8; 8192 of 100 among 18M rows, E =
  // 64 19.8 / 18.5; 8 x 64 ragged of 32, E = 64 5.4 / 6.0.
  const bool four = avg > 4 * split && (lpr > 4 || few());
  const int64_t per_block = int64_t(kWavesPerBlock) * (groups / split);
  for_launches((bags + per_block - 1) / per_block, kBlock, [&](uint32_t first, dim3 grid) {
    if (y_bf16)
      dispatch_mode(pool.mode, lpr, four, grid, st, d, I, O, int32_t(NS), B, split, int32_t(bags),
                    static_cast<__bf16*>(Y), status, pool.weights, first);
    else
      dispatch_mode(pool.mode, lpr, four, grid, st, d, I, O, int32_t(NS), B, split, int32_t(bags),
                    static_cast<float*>(Y), status, pool.weights, first);
  });
  return hipGetLastError();
}

}  // namespace embbag
