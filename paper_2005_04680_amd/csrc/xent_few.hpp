// The products of a wide table (dim > 128) in FP32 with few rows (few_wide): the table is read as it stands, once
// for the scores, which stay in the workspace (few rows of them are small beside the table), and once for dx;
// its three BF16 terms are made in registers.  The tiles of gemm.hpp need the terms packed: 6 bytes written
// and 12 read per element and product.  Measured, us, the whole call with those / these: 6 x 37169 x 2664
// 1295 / 368, 77 x 13117 x 3584 776 / 314, 251 x 5383 x 1468 286 / 161, 380 x 13000 x 1000 373 / 314, without
// gradients 64 x 100000 x 512 219 / 75; past the rule 250 x 30000 x 256 173 / 180.
// Bound by the table's way from memory: of 6 x 37169 x 2664 (396 MB) dx runs at 5.1 TB/s, the scores at 2.9 (their
// blocks are 1.1 rounds of the chip), dW's tiles write at 2.8.
#pragma once

#include "gemm.hpp"
#include "xent.hpp"

namespace embbag {
namespace {

constexpr int kFewBlock = 128;  // rows of x per block at most
// Where the table's bytes are more than what is written of scores and D.
inline bool few_wide(int32_t rows, int32_t dim) { return rows > 0 && rows <= 512 && rows <= dim / 2 + 64; }

// acc += a b of three terms each, the smallest products first.
__device__ __forceinline__ void six_products(const u4 (&a)[3], const u4 (&b)[3], f16v& acc) {
#pragma unroll
  for (int i = 0; i < 6; ++i) {
    constexpr int A[6] = {2, 1, 0, 1, 0, 0}, B[6] = {0, 1, 2, 0, 1, 0};
    acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf8, a[A[i]]),
                                                  __builtin_bit_cast(bf8, b[B[i]]), acc, 0, 0, 0);
  }
}

// Rows that count, in three terms, in the order in which the products take them: 16 elements of k after the
// other, of each 32 rows after the other, 64 lanes' 16 bytes per term.  (Rows as they stand make a load of 64
// lines; 77 x 13117 x 3584: scores 176 us, 105 this way, dx 119, 112.)
struct Fragments {
  const __bf16* data;
  int32_t tiles;  // of 32 rows
  __device__ __forceinline__ int64_t at(int64_t k, int tile, int lane) const {
    return ((k / 16 * tiles + tile) * 3 * kWave + lane) * 8;
  }
  __device__ __forceinline__ void load(int64_t k, int tile, int lane, u4 (&t)[3]) const {
#pragma unroll
    for (int p = 0; p < 3; ++p) t[p] = *reinterpret_cast<const u4*>(data + at(k, tile, lane) + p * kWave * 8);
  }
  // 8 elements of a row from k on.
  __device__ __forceinline__ void store(int64_t k, int row, const u4 (&t)[3]) const {
    __bf16* to = const_cast<__bf16*>(data) + at(k, row / 32, row % 32 + int(k % 16 / 8) * 32);
#pragma unroll
    for (int p = 0; p < 3; ++p) *reinterpret_cast<u4*>(to + p * kWave * 8) = t[p];
  }
};

// x's terms from their planes.
__global__ __launch_bounds__(kBlock) void few_x(const __bf16* __restrict__ x, int64_t plane, FastDiv chunks,
                                                const int32_t* __restrict__ rows, Fragments to) {
  const uint32_t i = blockIdx.x * kBlock + threadIdx.x, at = quotient(i, chunks);
  if (int(at) >= *rows) return;
  const int padded = int(chunks.div) * 8, k = int(i - at * chunks.div) * 8;
  u4 t[3];
#pragma unroll
  for (int p = 0; p < 3; ++p) t[p] = *reinterpret_cast<const u4*>(x + p * plane + int64_t(at) * padded + k);
  to.store(k, int(at), t);
}

// 4 elements on their way (zeros past the row), untouched until values().
template <class T>
struct Four;
template <>
struct Four<float> {
  f4 v;
  __device__ __forceinline__ void load(const float* p, bool in) { v = in ? load4(p) : f4{0.f, 0.f, 0.f, 0.f}; }
  __device__ __forceinline__ f4 values() const { return v; }
};
template <>
struct Four<__bf16> {
  u2 v;
  __device__ __forceinline__ void load(const __bf16* p, bool in) {
    v = in ? *reinterpret_cast<const u2*>(p) : u2{0u, 0u};
  }
  __device__ __forceinline__ f4 values() const { return f4{bf16_lo(v.x), bf16_hi(v.x), bf16_lo(v.y), bf16_hi(v.y)}; }
};

// A block: 32 rows of the table, TM tiles of 32 rows of x.  Its wavefronts take 32 elements of k in turn, so
// that together they read 512 bytes of each row, a load 128 of 8 rows: in the products' own layout a load is
// 16 bytes of 64 lines, which leave the first cache before the next load comes for the rest of them (6 x 37169 x
// 2664: 143 us, 131 this way).  A wavefront's own LDS turns them (chunk c of row r at place c ^ r % 8).  The
// sums are joined in order, one tile by each wavefront, which hands it to `stats`.
template <int TM, class TW, class Stats>
__global__ __launch_bounds__(kBlock) void few_scores(const TW* __restrict__ w, int64_t stride, int64_t vocab,
                                                     int32_t dim, Fragments x, const int32_t* __restrict__ rows,
                                                     float* __restrict__ scores, int64_t pitch, uint32_t blocks,
                                                     Stats stats) {
  __shared__ f4 shared[kWavesPerBlock][TM][4][kWave];
  __shared__ f4 turn[kWavesPerBlock][32][8];
  const int lane = lane_id(), wave = wave_id(), row = lane % 32, half = lane / 32;
  const int row0 = int(blockIdx.x / blocks) * kFewBlock, live = scalar(*rows) - row0;
  if (live <= 0) return;
  const int64_t n0 = int64_t(blockIdx.x % blocks) * 32;
  // Load i: rows 8 i to 8 i + 7, 8 lanes each.
  const TW* p[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int64_t n = n0 + 8 * i + lane / 8;
    p[i] = w + (n < vocab ? n : vocab - 1) * stride + lane % 8 * 4;
  }
  f16v acc[TM];
#pragma unroll
  for (int j = 0; j < TM; ++j) acc[j] = f16v{};
  Four<TW> next[4];
  auto fetch = [&](int k0) {
    const bool in = k0 + lane % 8 * 4 < dim;
#pragma unroll
    for (int i = 0; i < 4; ++i) next[i].load(p[i] + k0, in);
  };
  constexpr int STEP = 32 * kWavesPerBlock;
  fetch(32 * wave);
  for (int k0 = 32 * wave; k0 < dim; k0 += STEP) {
    // (Loads return in order: x's, which this step waits for, before the table's of the next step.)
    u4 b[2][TM][3];
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int j = 0; j < TM; ++j)
        if (j * 32 < live) x.load(k0 + 16 * s, row0 / 32 + j, lane, b[s][j]);
#pragma unroll
    for (int i = 0; i < 4; ++i) turn[wave][8 * i + lane / 8][lane % 8 ^ lane / 8] = next[i].values();
    __builtin_amdgcn_sched_barrier(0);
    fetch(k0 + STEP);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const int c = 4 * s + 2 * half;
      const f4 lo = turn[wave][row][c ^ row % 8], hi = turn[wave][row][(c + 1) ^ row % 8];
      const float v[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
      u4 a[3];
      nearest_terms(v, a);
#pragma unroll
      for (int j = 0; j < TM; ++j)
        if (j * 32 < live) six_products(a, b[s][j], acc[j]);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
#pragma unroll
  for (int j = 0; j < TM; ++j)
#pragma unroll
    for (int q = 0; q < 4; ++q)
      shared[wave][j][q][lane] = f4{acc[j][4 * q], acc[j][4 * q + 1], acc[j][4 * q + 2], acc[j][4 * q + 3]};
  __syncthreads();
  if (wave >= TM || wave * 32 >= live) return;
  f16v sum[1][1];
  const int at = wave * 32 + row;  // from row0
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    f4 s = shared[0][wave][q][lane];
#pragma unroll
    for (int k = 1; k < kWavesPerBlock; ++k) s += shared[k][wave][q][lane];
    if (scores != nullptr && at < live) store4(scores + (row0 + at) * pitch + n0 + 8 * q + 4 * half, s);
#pragma unroll
    for (int r = 0; r < 4; ++r) sum[0][0][4 * q + r] = s[r];
  }
  stats.template operator()<1, 1>(sum, n0, row0 + wave * 32, row0 + live, 0, nullptr);
}

// D of the rows that count, in three terms, from their scores: 8 columns per thread, zeros past the table.  In
// fragments for dx's product above (`f` not empty); `planes` planes of it for the tiles' (`d` not null).
__global__ __launch_bounds__(kBlock) void few_d(const float* __restrict__ scores, FastDiv chunks, int64_t vocab,
                                                const Token* __restrict__ tokens, float unit,
                                                const int32_t* __restrict__ rows, __bf16* __restrict__ d,
                                                int64_t plane, int planes, Fragments f) {
  const uint32_t chunk = blockIdx.x * kBlock + threadIdx.x, q = quotient(chunk, chunks);
  if (int(q) >= *rows) return;
  const int64_t at = q, pitch = int64_t(chunks.div) * 8, n = int64_t(chunk - q * chunks.div) * 8;
  const Token t = tokens[at];
  const float c = t.inv * t.ratio;
  const f4 lo = load4(scores + at * pitch + n), hi = load4(scores + at * pitch + n + 4);
  float v[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float e = exp2_of(__builtin_fmaf(v[i], unit, -t.top));
    v[i] = n + i >= vocab ? 0.f : n + i == t.label ? (e * t.inv - 1.f) * t.ratio : e * c;
  }
  u4 terms[3];
  if (planes == 3) {
    nearest_terms(v, terms);
  } else {  // (Two terms: a NaN has to be in the first.)
    terms[0] = pack16(v);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] -= (i % 2 ? bf16_hi : bf16_lo)(terms[0][i / 2]);
    terms[1] = terms[2] = pack16(v);
  }
  if (f.data != nullptr) f.store(n, int(at), terms);
  if (d == nullptr) return;
#pragma unroll
  for (int k = 0; k < 3; ++k)
    if (k < planes) *reinterpret_cast<u4*>(d + k * plane + at * pitch + n) = terms[k];
}

// N elements of a row.
__device__ __forceinline__ void load_some(const float* p, float (&v)[4]) {
  unpack16(*reinterpret_cast<const u4*>(p), v);
}
__device__ __forceinline__ void load_some(const __bf16* p, float (&v)[4]) {
  const f4 x = load4(p);
  v[0] = x.x, v[1] = x.y, v[2] = x.z, v[3] = x.w;
}
__device__ __forceinline__ void load_some(const float* p, float (&v)[2]) {
  typedef float f2 __attribute__((ext_vector_type(2)));
  const f2 x = *reinterpret_cast<const f2*>(p);
  v[0] = x.x, v[1] = x.y;
}
__device__ __forceinline__ void load_some(const __bf16* p, float (&v)[2]) {
  const uint32_t x = *reinterpret_cast<const uint32_t*>(p);
  v[0] = bf16_lo(x), v[1] = bf16_hi(x);
}

// A part of `count` of dx = D W: 32 TN columns of the table, `per` chunks of 16 of its rows, which the wavefronts
// take in turn.  A lane's TN elements are of TN tiles (tile t's row i is column TN i + t), so that a row is read
// in wide pieces; the wavefronts' sums are joined in order.
template <int TM, int TN, class TW>
__global__ __launch_bounds__(kBlock) void few_dx(const TW* __restrict__ w, int64_t stride, int64_t vocab,
                                                 int32_t dim, Fragments d, const int32_t* __restrict__ rows,
                                                 int32_t per, float* __restrict__ parts, int64_t part,
                                                 uint32_t columns, uint32_t count) {
  constexpr int GROUP = 4 / TN;  // tiles of rows that are joined at a time
  static_assert(TN <= 4 && TM % GROUP == 0, "join");
  __shared__ f4 shared[kWavesPerBlock][GROUP][TN][4][kWave];
  const int lane = lane_id(), wave = wave_id(), row = lane % 32, half = lane / 32;
  const uint32_t z = blockIdx.x / columns % count;
  const int row0 = int(blockIdx.x / columns / count) * kFewBlock, live = scalar(*rows) - row0;
  if (live <= 0) return;
  const int e0 = int(blockIdx.x % columns) * 32 * TN, e = e0 + row * TN;
  const bool in = e < dim;
  const int64_t first = int64_t(z) * per * 16;
  const int64_t end = first + int64_t(per) * 16 < vocab ? first + int64_t(per) * 16 : vocab;
  const TW* p = w + (in ? e : 0);
  f16v acc[TN][TM];
#pragma unroll
  for (int t = 0; t < TN; ++t)
#pragma unroll
    for (int j = 0; j < TM; ++j) acc[t][j] = f16v{};
  float next[8][TN];
  auto fetch = [&](int64_t v0) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int64_t v = v0 + 8 * half + i;
#pragma unroll
      for (int t = 0; t < TN; ++t) next[i][t] = 0.f;
      if (in && v < end) load_some(p + v * stride, next[i]);
    }
  };
  fetch(first + wave * 16);
  for (int64_t v0 = first + wave * 16; v0 < end; v0 += 16 * kWavesPerBlock) {
    u4 a[TN][3], b[TM][3];
#pragma unroll
    for (int j = 0; j < TM; ++j)
      if (j * 32 < live) d.load(v0, row0 / 32 + j, lane, b[j]);
    float now[TN][8];
#pragma unroll
    for (int t = 0; t < TN; ++t)
#pragma unroll
      for (int i = 0; i < 8; ++i) now[t][i] = next[i][t];
    __builtin_amdgcn_sched_barrier(0);
    fetch(v0 + 16 * kWavesPerBlock);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int t = 0; t < TN; ++t) nearest_terms(now[t], a[t]);
#pragma unroll
    for (int j = 0; j < TM; ++j)
      if (j * 32 < live) {
#pragma unroll
        for (int t = 0; t < TN; ++t) six_products(a[t], b[j], acc[t][j]);
      }
  }
  float* out = parts + z * part;
#pragma unroll
  for (int g = 0; g < TM; g += GROUP) {
    if (g * 32 >= live) break;
    if (g > 0) __syncthreads();
#pragma unroll
    for (int j = 0; j < GROUP; ++j)
#pragma unroll
      for (int t = 0; t < TN; ++t)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const f16v& s = acc[t][g + j];
          shared[wave][j][t][q][lane] = f4{s[4 * q], s[4 * q + 1], s[4 * q + 2], s[4 * q + 3]};
        }
    __syncthreads();
    // Wavefront q joins the tiles' rows 8 q to 8 q + 7.
#pragma unroll
    for (int j = 0; j < GROUP; ++j) {
      float s[4 * TN];
#pragma unroll
      for (int t = 0; t < TN; ++t) {
        f4 x = shared[0][j][t][wave][lane];
#pragma unroll
        for (int k = 1; k < kWavesPerBlock; ++k) x += shared[k][j][t][wave][lane];
#pragma unroll
        for (int r = 0; r < 4; ++r) s[r * TN + t] = x[r];
      }
      const int at = (g + j) * 32 + row, c = e0 + (8 * wave + 4 * half) * TN;
#pragma unroll
      for (int i = 0; i < 4 * TN; i += 4)
        if (at < live && c + i < dim)
          store4(out + int64_t(row0 + at) * dim + c + i, f4{s[i], s[i + 1], s[i + 2], s[i + 3]});
    }
  }
}

// Parts of dx: two blocks per compute unit, 8 chunks for each wavefront, and no more than a quarter of the
// table's bytes written in them.
inline int32_t few_parts(int32_t rows, int64_t vocab, int32_t dim) {
  const int64_t columns = rows > 32 ? 64 : 128;
  int64_t z = 2 * kNumCu / ((dim + columns - 1) / columns * ((rows + kFewBlock - 1) / kFewBlock));
  if (z > vocab / 512) z = vocab / 512;
  if (z > vocab / (4 * int64_t(rows))) z = vocab / (4 * int64_t(rows));
  if (z < 1) z = 1;
  const int64_t chunks = (vocab + 15) / 16, per = (chunks + z - 1) / z;
  return int32_t((chunks + per - 1) / per);
}

template <class TW, class Stats>
void launch_few_scores(const TW* w, int64_t stride, int64_t vocab, int32_t dim, int32_t rows, const Fragments& x,
                       const int32_t* live, float* scores, int64_t pitch, const Stats& stats, hipStream_t st) {
  const uint32_t blocks = uint32_t((vocab + 31) / 32);
  const dim3 grid(blocks * uint32_t((rows + kFewBlock - 1) / kFewBlock));
  auto run = [&](auto tm) {
    hipLaunchKernelGGL((few_scores<tm.value, TW, Stats>), grid, dim3(kBlock), 0, st, w, stride, vocab, dim, x, live,
                       scores, pitch, blocks, stats);
  };
  if (rows > 64)
    run(std::integral_constant<int, 4>());
  else if (rows > 32)
    run(std::integral_constant<int, 2>());
  else
    run(std::integral_constant<int, 1>());
}

template <class TW>
void launch_few_dx(const TW* w, int64_t stride, int64_t vocab, int32_t dim, int32_t rows, const Fragments& d,
                   const int32_t* live, int32_t count, float* parts, int64_t part, hipStream_t st) {
  const int64_t chunks = (vocab + 15) / 16;
  const int32_t per = int32_t((chunks + count - 1) / count);
  auto run = [&](auto tm, auto tn) {
    constexpr int COLUMNS = 32 * tn.value;
    const uint32_t columns = uint32_t((dim + COLUMNS - 1) / COLUMNS);
    const dim3 grid(columns * uint32_t(count) * uint32_t((rows + kFewBlock - 1) / kFewBlock));
    hipLaunchKernelGGL((few_dx<tm.value, tn.value, TW>), grid, dim3(kBlock), 0, st, w, stride, vocab, dim, d, live, per,
                       parts, part, columns, uint32_t(count));
  };
  if (rows > 64)
    run(std::integral_constant<int, 4>(), std::integral_constant<int, 2>());
  else if (rows > 32)
    run(std::integral_constant<int, 2>(), std::integral_constant<int, 2>());
  else
    run(std::integral_constant<int, 1>(), std::integral_constant<int, 4>());
}

}  // namespace
}  // namespace embbag
