// Softmax cross entropy of the scores over a table, with the gradients of the scores' inputs and
// of the table; the scores are kept only where they are small.
//
// z = scale x W^T, loss = w (log sum exp z - z[label]), D = softmax(z) - onehot(label):
//   dx = scale w D W,   dW = scale (w D)^T x.
// 1. The rows that count (a label, a weight) are packed: x as BF16, rows that are left out are not
//    computed with.
// 2. The scores' tiles leave, for every row and 128 columns, their largest score and the sum of the
//    exponentials; the parts are joined in order.
// 3. Piece by piece of the vocabulary the tiles are computed again, now as D times w / (largest w),
//    rounded to BF16 in the workspace, and that piece's two products follow: dx is added up in FP32, dW
//    of the piece is final.
// All sums are in orders that the sizes determine; there are no atomics on them.
//
// BF16 operands are taken as they are.  D is rounded to BF16 (2^-8 of each element at most, as the
// gradients' own rounding; two terms of it where few rows count, so that the products do not bound the call, or the
// table is small).
// With the weights' ratio in D, equal weights leave the label's element, next to -1, almost exact.  FP32
// operands, and D with them, are the sum of three BF16 terms, of whose nine products six are taken: what
// is left out is below 2^-22 of each product.  Where scores cost more to compute again than to keep (FP32 sides,
// few rows) and fit in 512 MB, they stay in FP32 and D is made of them.
//
// Four products, 8 N V E operations, where 6 N V E would do if the scores were kept: at 4096 x 131072 x 2048
// they would be 2.1 GB written and read in FP32.  Bound by the products, with few rows by W's bytes.  Measured, us:
// 4096 x 131072 x 2048 BF16 7060, 1999 x 50001 x 300 (1200 rows count) 279, 2048 x 100003 x 512 (205 count, two terms
// of D) 292, 1 x 200003 x 1024 without gradients 85 (410 MB at 4.8 TB/s).
#include "gemm.hpp"
#include "xent.hpp"
#include "xent_few.hpp"

namespace embbag {
namespace {

constexpr int64_t kPieceBytes = int64_t(512) << 20;   // of D, W's terms, the sums' parts or kept scores: at most, each
constexpr int kRowsAtOnce = 4096;                     // rows whose places 1024 threads find in a round
constexpr int64_t kMaxPitch = int64_t(1) << 19;       // elements of a row of D

// 8 elements of a row from e on (zeros past dim; dim % 4 == 0) times the sign as BF16 terms to `dst`.
template <int TERMS, class T>
__device__ __forceinline__ void pack8(const T* row, int e, int dim, float sign, __bf16* dst, int64_t plane) {
  const f4 zero = {0.f, 0.f, 0.f, 0.f};
  const f4 p = e < dim ? load4(row + e) : zero;
  const f4 q = e + 4 < dim ? load4(row + e + 4) : zero;
  const float v[8] = {p.x * sign, p.y * sign, p.z * sign, p.w * sign,
                      q.x * sign, q.y * sign, q.z * sign, q.w * sign};
  if constexpr (TERMS == 1) {
    store16(dst, pack16(v));
  } else {
    u4 t[3];
    nearest_terms(v, t);
#pragma unroll
    for (int k = 0; k < 3; ++k) store16(dst + k * plane, t[k]);
  }
}

// Which rows count, their places in order, and the largest weight, by the threads of one block of 1024.
// `writes`: whether the block stores them; `place` is stored for rows from `low` to `high` alone
// and may be in LDS (its entry 0 is row `low`).  The losses of the rows that do not count are 0.
struct RowSums {
  int counts[16];
  float tops[16];
};
__device__ __forceinline__ void find_rows(const int32_t* __restrict__ labels, const float* __restrict__ weights,
                                          int32_t rows, int32_t vocab, float scale, const Rows& out,
                                          int32_t* place, int32_t low_row, int32_t high_row, bool writes,
                                          float* __restrict__ loss, int32_t* __restrict__ status,
                                          RowSums& shared) {
  const int lane = lane_id(), wave = wave_id();
  int base = 0;
  float top = 0.f;
  bool bad = false;
  for (int r0 = 0; r0 < rows; r0 += kRowsAtOnce) {
    int label[4], n = 0;
    float w[4];
    bool in[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = r0 + threadIdx.x * 4 + i;
      label[i] = r < rows ? labels[r] : -1;
      w[i] = r < rows && weights != nullptr ? weights[r] : 1.f;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      bad = bad || label[i] >= vocab;
      in[i] = label[i] >= 0 && label[i] < vocab && w[i] != 0.f;
      n += in[i];
      if (in[i]) top = fmaxf(top, fabsf(w[i]));
    }
    int before = n;
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) {
      const int v = __shfl_up(before, d, kWave);
      if (lane >= d) before += v;
    }
    __syncthreads();  // (the counts of the round before have been read)
    if (lane == kWave - 1) shared.counts[wave] = before;
    __syncthreads();
    int at = base + before - n, all = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      if (i < wave) at += shared.counts[i];
      all += shared.counts[i];
    }
    base += all;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = r0 + threadIdx.x * 4 + i;
      if (r >= rows) continue;
      if (r >= low_row && r < high_row) place[r - low_row] = in[i] ? at : -1;
      if (in[i]) {
        if (writes) {
          out.row[at] = r;
          Token t = {0.f, 0.f, w[i], label[i]};
          out.tokens[at] = t;
        }
        ++at;
      } else if (writes) {
        loss[r] = 0.f;
      }
    }
  }
  if (!writes) return;
  if (bad && status != nullptr) atomicMin(status, EMBBAG_ERR_INDEX_RANGE);
#pragma unroll
  for (int d = 1; d < kWave; d *= 2) top = fmaxf(top, __shfl_xor(top, d, kWave));
  if (lane == 0) shared.tops[wave] = top;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int i = 1; i < 16; ++i) top = fmaxf(top, shared.tops[i]);
    out.head->live = base;
    out.head->largest = top;
    out.head->factor = scale * top;
    out.head->factor_w = fabsf(scale) * top;
  }
}

__global__ __launch_bounds__(1024) void xent_rows(const int32_t* __restrict__ labels,
                                                  const float* __restrict__ weights, int32_t rows,
                                                  int32_t vocab, float scale, Rows out,
                                                  float* __restrict__ loss, int32_t* __restrict__ status) {
  __shared__ RowSums shared;
  find_rows(labels, weights, rows, vocab, scale, out, out.place, 0, rows, true, loss, status, shared);
}

// Row r of x, times the sign, as TERMS planes at its place among the rows that count; dx's row as zeros if
// it does not.  By a wavefront.
template <int TERMS, class T>
__device__ __forceinline__ void pack_row(const T* __restrict__ x, int64_t stride, int r, int at, int32_t dim,
                                         int32_t padded, float sign, __bf16* __restrict__ out, int64_t plane,
                                         T* __restrict__ dx, int64_t dx_stride) {
  if (at < 0) {
    if (dx == nullptr) return;
    for (int e = lane_id() * 4; e < dim; e += kWave * 4)
      store4(dx + r * dx_stride + e, f4{0.f, 0.f, 0.f, 0.f});
    return;
  }
  for (int e = lane_id() * 8; e < padded; e += kWave * 8)
    pack8<TERMS>(x + r * stride, e, dim, sign, out + int64_t(at) * padded + e, plane);
}

template <int TERMS, class T>
__global__ __launch_bounds__(kBlock) void xent_pack_x(const T* __restrict__ x, int64_t stride,
                                                      int32_t rows, int32_t dim, int32_t padded, float sign,
                                                      const int32_t* __restrict__ place,
                                                      __bf16* __restrict__ out, int64_t plane,
                                                      T* __restrict__ dx, int64_t dx_stride) {
  const int r = blockIdx.x * kWavesPerBlock + wave_id();
  if (r >= rows) return;
  pack_row<TERMS>(x, stride, r, scalar(place[r]), dim, padded, sign, out, plane, dx, dx_stride);
}

// Both for up to kRowsAtOnce rows: every block finds the places for itself and packs 16 rows (a launch
// less: 33 x 32001 x 128 4 us).
template <int TERMS, class T>
__global__ __launch_bounds__(1024) void xent_rows_pack(const int32_t* __restrict__ labels,
                                                       const float* __restrict__ weights, int32_t rows,
                                                       int32_t vocab, float scale, Rows found,
                                                       float* __restrict__ loss, int32_t* __restrict__ status,
                                                       const T* __restrict__ x, int64_t stride, int32_t dim,
                                                       int32_t padded, float sign, __bf16* __restrict__ out,
                                                       int64_t plane, T* __restrict__ dx, int64_t dx_stride) {
  __shared__ RowSums shared;
  __shared__ int32_t place[16];
  const int r0 = blockIdx.x * 16, r = r0 + wave_id();
  find_rows(labels, weights, rows, vocab, scale, found, place, r0, r0 + 16, blockIdx.x == 0, loss, status, shared);
  __syncthreads();
  if (r >= rows) return;
  pack_row<TERMS>(x, stride, r, scalar(place[wave_id()]), dim, padded, sign, out, plane, dx, dx_stride);
}

// Rows of W as TERMS planes [rows][padded].
template <int TERMS, class T>
__global__ __launch_bounds__(kBlock) void xent_pack_w(const T* __restrict__ w, int64_t stride,
                                                      int64_t rows, int32_t dim, FastDiv chunks,
                                                      __bf16* __restrict__ out, int64_t plane) {
  const int64_t i = int64_t(blockIdx.x) * kBlock + threadIdx.x;
  if (i >= rows * chunks.div) return;
  const uint32_t r = quotient(uint32_t(i), chunks);
  const int e = int(uint32_t(i) - r * chunks.div) * 8;
  pack8<TERMS>(w + int64_t(r) * stride, e, dim, 1.f, out + i * 8, plane);
}

// A tile's parts: of each row and the wavefront's 32 TN columns the exponent of the largest score, rounded,
// and the sum of the exponentials beside exactly that.
template <bool KEEP>
struct StatsEpi {
  float2* parts;         // [the piece's columns / (32 TN)][pitch]
  int64_t pitch;
  const Token* tokens;
  float* target;
  float unit;
  int64_t first;         // the piece's first column
  int64_t columns;       // of the piece
  float* scores;         // [live][scores_pitch], with KEEP
  int64_t scores_pitch;
  template <int TN, int TM>
  static constexpr int kScratch = 0;

  template <int TN, int TM>
  __device__ __forceinline__ void operator()(f16v (&acc)[TN][TM], int64_t n, int64_t m, int64_t m_end, int,
                                             uint8_t*) const {
    const int row = lane_id() % 32, half = lane_id() / 32;
    if constexpr (KEEP) {
#pragma unroll
      for (int j = 0; j < TM; ++j) {
        const int64_t at = m + j * 32 + row;
        float* to = scores + at * scores_pitch + n + half * 4;
        const int64_t left = at < m_end ? scores_pitch - n - half * 4 : 0;
#pragma unroll
        for (int i = 0; i < TN; ++i)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const int c = i * 32 + q * 8;
            if (c < left)
              store4(to + c, f4{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]});
          }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
#pragma unroll
    for (int j = 0; j < TM; ++j) {
      const int64_t at = m + j * 32 + row;
      const bool in = at < m_end;
      if (n + 32 * TN > columns) {
        const int64_t left = columns - n - half * 4;
#pragma unroll
        for (int i = 0; i < TN; ++i)
#pragma unroll
          for (int r = 0; r < 16; ++r)
            acc[i][j][r] = i * 32 + r / 4 * 8 + r % 4 < left ? acc[i][j][r] : low();
      }
      float top = low();
#pragma unroll
      for (int i = 0; i < TN; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) top = fmaxf(top, acc[i][j][r]);
      top = fmaxf(top, __shfl_xor(top, 32, kWave));
      const float ref = top == low() ? 0.f : -(top * unit);
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < TN; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) sum += exp2_of(__builtin_fmaf(acc[i][j][r], unit, ref));
      sum += __shfl_xor(sum, 32, kWave);
      const int label = in ? tokens[at].label : -1;
      const int64_t place = label - first - n - half * 4;  // of the label among the lane's columns
      if (place >= 0 && place < 32 * TN && place / 4 % 2 == 0) {
        float z = 0.f;
#pragma unroll
        for (int i = 0; i < TN; ++i)
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if (int(place) == i * 32 + r / 4 * 8 + r % 4) z = acc[i][j][r];
        target[at] = z;
      }
      if (in && half == 0 && n < columns) parts[n / (32 * TN) * pitch + at] = float2{top * unit, sum};
    }
  }
};

// Joins the parts of TOKENS rows per block to what the pieces before have left (none if `first`) in top and
// inv; after the `last` piece losses, and what the backward needs.
template <int TOKENS>
__global__ __launch_bounds__(1024) void xent_join(const float2* __restrict__ parts, int64_t pitch,
                                                  int32_t count, bool first, bool last, float unit,
                                                  Rows rows, float* __restrict__ loss) {
  constexpr int SLICES = 1024 / TOKENS;
  __shared__ float2 shared[SLICES][TOKENS + 1];
  const int live = rows.head->live;
  const int t = threadIdx.x % TOKENS, slice = threadIdx.x / TOKENS;
  const int at = blockIdx.x * TOKENS + t;
  if (int(blockIdx.x) * TOKENS >= live) return;
  float top = low(), sum = 0.f;
  auto add = [&](float2 p) {
    const float m = fmaxf(top, p.x), ref = m == low() ? 0.f : m;
    sum = sum * exp2_of(top - ref) + p.y * exp2_of(p.x - ref);
    top = m;
  };
  if (at < live) {
#pragma unroll 4
    for (int i = slice; i < count; i += SLICES) add(parts[int64_t(i) * pitch + at]);
  }
  shared[slice][t] = float2{top, sum};
  __syncthreads();
  for (int d = SLICES / 2; d > 0; d /= 2) {
    if (slice < d) {
      add(shared[slice + d][t]);
      shared[slice][t] = float2{top, sum};
    }
    __syncthreads();
  }
  if (slice != 0 || at >= live) return;
  Token k = rows.tokens[at];
  if (!first) add(float2{k.top, k.inv});
  if (!last) {
    k.top = top, k.inv = sum;
    rows.tokens[at] = k;
    return;
  }
  const float w = k.ratio;
  const int r = rows.row[at];
  loss[r] = w * (__builtin_fmaf(-rows.target[at], unit, top) * kLn2 + __builtin_logf(sum));
  k.top = top, k.inv = 1.f / sum, k.ratio = w / rows.head->largest;
  rows.tokens[at] = k;
}

// Rows of a tile turned around in a wavefront's own LDS: 32 rows of m, 128 bytes of each.
template <class T>
constexpr int kTurnTiles = 128 / 32 / int(sizeof(T)) < 1 ? 1 : 128 / 32 / int(sizeof(T));
template <class T, int TN>
constexpr int kTiles = kTurnTiles<T> < TN ? kTurnTiles<T> : TN;
template <class T, int TN>
constexpr int kTurnPitch = 32 * kTiles<T, TN> + kVec<T>;

// Stores 32 rows of m and kTiles * 32 columns from `turn`: `put(row of the 32, column, 16 bytes)`.
template <class T, int TN, class Put>
__device__ __forceinline__ void stored_rows(const T* turn, Put put) {
  constexpr int V = kVec<T>, PITCH = kTurnPitch<T, TN>, PER_ROW = 32 * kTiles<T, TN> / V;
  constexpr int ROWS = kWave / PER_ROW;
  const int r = lane_id() / PER_ROW, c = lane_id() % PER_ROW * V;
#pragma unroll
  for (int q = 0; q < 32 / ROWS; ++q)
    put(r + q * ROWS, c, *reinterpret_cast<const u4*>(turn + (r + q * ROWS) * PITCH + c));
}
template <class T, int TN, int TM>
__device__ __forceinline__ void turn_rows(T* turn, const f16v (&acc)[TN][TM], int h, int j) {
  const int row = lane_id() % 32, half = lane_id() / 32;
#pragma unroll
  for (int i = 0; i < kTiles<T, TN>; ++i)
#pragma unroll
    for (int q = 0; q < 4; ++q)
      store4(turn + row * kTurnPitch<T, TN> + i * 32 + q * 8 + half * 4,
             f4{acc[h + i][j][q * 4], acc[h + i][j][q * 4 + 1], acc[h + i][j][q * 4 + 2],
                acc[h + i][j][q * 4 + 3]});
}

// A tile of D (times the weights' ratio): TERMS planes [live][pitch], zeros in the columns past the
// vocabulary.  Of two the second is stored only where at most `few` rows count.
template <int TERMS>
struct GradEpi {
  __bf16* d;
  int64_t pitch, plane;
  const Token* tokens;
  float unit;
  int64_t first, columns;
  const int32_t* live;
  int32_t few;
  template <int TN, int TM>
  static constexpr int kScratch = 32 * kTurnPitch<__bf16, TN> * 2;

  template <int TN, int TM>
  __device__ __forceinline__ void operator()(f16v (&acc)[TN][TM], int64_t n, int64_t m, int64_t m_end, int,
                                             uint8_t* scratch) const {
    const int row = lane_id() % 32, half = lane_id() / 32;
    __bf16* turn = reinterpret_cast<__bf16*>(scratch);
    const bool one = TERMS == 2 && scalar(*live) > few;
#pragma unroll
    for (int j = 0; j < TM; ++j) {
      const int64_t at = m + j * 32 + row;
      const Token t = at < m_end ? tokens[at] : Token{0.f, 0.f, 0.f, -1};
      const float c = t.inv * t.ratio;
      const int64_t place = t.label - first - n - half * 4;  // of the label among the lane's columns
      const bool mine = place >= 0 && place < 32 * TN && place / 4 % 2 == 0;
      if (__builtin_amdgcn_ballot_w64(mine) != 0ull) {
#pragma unroll
        for (int i = 0; i < TN; ++i)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const float e = exp2_of(__builtin_fmaf(acc[i][j][r], unit, -t.top));
            const bool label = mine && int(place) == i * 32 + r / 4 * 8 + r % 4;
            acc[i][j][r] = label ? (e * t.inv - 1.f) * t.ratio : e * c;
          }
      } else {
#pragma unroll
        for (int i = 0; i < TN; ++i)
#pragma unroll
          for (int r = 0; r < 16; ++r)
            acc[i][j][r] = exp2_of(__builtin_fmaf(acc[i][j][r], unit, -t.top)) * c;
      }
      if (n + 32 * TN > columns) {
        const int64_t left = columns - n - half * 4;
#pragma unroll
        for (int i = 0; i < TN; ++i)
#pragma unroll
          for (int r = 0; r < 16; ++r)
            acc[i][j][r] = i * 32 + r / 4 * 8 + r % 4 < left ? acc[i][j][r] : 0.f;
      }
#pragma unroll
      for (int h = 0; h < TN; h += kTiles<__bf16, TN>) {
#pragma unroll
        for (int k = 0; k < TERMS; ++k) {
          turn_rows<__bf16, TN, TM>(turn, acc, h, j);
          stored_rows<__bf16, TN>(turn, [&](int r, int c, const u4& v) {
            const int64_t to = m + j * 32 + r;
            if (to < m_end && n + h * 32 + c < pitch)
              *reinterpret_cast<u4*>(d + k * plane + to * pitch + n + h * 32 + c) = v;
          });
          if (one) break;
          if (k + 1 < TERMS) {
#pragma unroll
            for (int i = 0; i < kTiles<__bf16, TN>; ++i)
#pragma unroll
              for (int r = 0; r < 16; ++r) {
                const float x = acc[h + i][j][r], rest = x - float(__bf16(x));
                acc[h + i][j][r] = rest;
              }
          }
        }
      }
    }
  }
};

// Sums times `factor` into rows of `out`, or into part z of parts [rows of m][pitch] (`part` elements
// each; of the rows that count where that is negative), where `add` adds to what they hold.
template <class T>
struct StoreEpi {
  T* out;
  int64_t pitch;
  int64_t columns;
  const float* factor;
  int64_t part;
  bool add;
  template <int TN, int TM>
  static constexpr int kScratch = 32 * kTurnPitch<T, TN> * int(sizeof(T));

  template <int TN, int TM>
  __device__ __forceinline__ void operator()(f16v (&acc)[TN][TM], int64_t n, int64_t m, int64_t m_end, int z,
                                             uint8_t* scratch) const {
    constexpr int V = kVec<T>;
    T* turn = reinterpret_cast<T*>(scratch);
    const float f = factor != nullptr ? *factor : 1.f;
#pragma unroll
    for (int j = 0; j < TM; ++j) {
      if (factor != nullptr) {
#pragma unroll
        for (int i = 0; i < TN; ++i)
#pragma unroll
          for (int r = 0; r < 16; ++r) acc[i][j][r] *= f;
      }
#pragma unroll
      for (int h = 0; h < TN; h += kTiles<T, TN>) {
        turn_rows<T, TN, TM>(turn, acc, h, j);
        stored_rows<T, TN>(turn, [&](int r, int c, const u4& v) {
          const int64_t at = m + j * 32 + r, col = n + h * 32 + c;
          if (at >= m_end || col >= columns) return;
          T* p = out + z * (part < 0 ? m_end * pitch : part) + at * pitch + col;
          if (col + V <= columns) {
            if (sizeof(T) == 4 && add) {
              float x[kVec<T>], y[kVec<T>];
              unpack16(v, x);
              unpack16(load16(p), y);
#pragma unroll
              for (int e = 0; e < V; ++e) x[e] += y[e];
              store16(p, pack16(x));
            } else {
              store16(p, v);
            }
          } else {  // 4 BF16 elements: columns % 4 == 0
            *reinterpret_cast<u2*>(p) = u2{v.x, v.y};
          }
        });
      }
    }
  }
};

// The parts [splits][rows of m][dim] added up, times the factor, into the rows that `map` names: SLICES
// threads for 4 elements add every SLICES-th part each, then their sums are added in order.
struct PartCount {
  int32_t count;
  int64_t part;  // elements of a part
  // Where not 0, both are those of a product whose splits are found from the rows that count.
  int32_t blocks, bm, ntiles;
  int64_t steps;
};
template <int SLICES, class T>
__global__ __launch_bounds__(kBlock) void xent_join_parts(const float* __restrict__ parts, PartCount pc,
                                                          const int32_t* __restrict__ live,
                                                          int64_t rows, FastDiv d4,
                                                          const int32_t* __restrict__ map,
                                                          const float* __restrict__ factor,
                                                          T* __restrict__ out, int64_t pitch,
                                                          int64_t row0) {
  constexpr int EACH = kBlock / SLICES;
  __shared__ f4 sums[SLICES > 1 ? SLICES : 1][EACH];
  const int t = threadIdx.x % EACH, slice = threadIdx.x / EACH;
  const int64_t i = int64_t(blockIdx.x) * EACH + t;
  const uint32_t q = quotient(uint32_t(i), d4);
  const int64_t at = row0 + q;
  const int c = int(uint32_t(i) - q * d4.div) * 4;
  const int64_t end = live != nullptr ? int64_t(*live) : rows;
  int32_t splits = pc.count;
  int64_t part = pc.part;
  if (pc.blocks != 0) {
    splits = split_steps((end + pc.bm - 1) / pc.bm * pc.ntiles, pc.steps, pc.blocks).count;
    part = end * (int64_t(d4.div) * 4);
  }
  const bool in = i < (rows - row0) * int64_t(d4.div) && at < end;
  f4 s = {0.f, 0.f, 0.f, 0.f};
  if (in) {
    const float* p = parts + at * (int64_t(d4.div) * 4) + c;
#pragma unroll 8
    for (int z = slice; z < splits; z += SLICES) s += load4(p + z * part);
  }
  if constexpr (SLICES > 1) {
    sums[slice][t] = s;
    __syncthreads();
    if (slice != 0) return;
#pragma unroll
    for (int k = 1; k < SLICES; ++k) s += sums[k][t];
  }
  if (!in) return;
  const float f = *factor;
  store4(out + (map != nullptr ? int64_t(map[at]) : at) * pitch + c, s * f);
}
// Slices where the parts are many: their loads are a chain otherwise (33 rows of 128 from 250 parts: 18 us
// with one).
template <class T>
void launch_join_parts(const float* parts, const PartCount& pc, const int32_t* live, int64_t rows, int32_t dim,
                       const int32_t* map, const float* factor, T* out, int64_t pitch, int64_t row0,
                       hipStream_t st) {
  const int64_t n = (rows - row0) * (dim / 4);
  const FastDiv d = fast_div(uint32_t(dim / 4));
  auto run = [&](auto slices) {
    constexpr int S = decltype(slices)::value;
    hipLaunchKernelGGL((xent_join_parts<S, T>), dim3(unsigned((n + kBlock / S - 1) / (kBlock / S))),
                       dim3(kBlock), 0, st, parts, pc, live, rows, d, map, factor, out, pitch, row0);
  };
  if (pc.count > 32)
    run(std::integral_constant<int, 32>());
  else if (pc.count > 4)
    run(std::integral_constant<int, 4>());
  else
    run(std::integral_constant<int, 1>());
}

size_t align256(size_t x) { return (x + 255) / 256 * 256; }
int64_t up(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Tile shapes: columns and rows.
struct Shape {
  int bn, bm;
  // Columns of a wavefront, which a part of a row's sum covers.
  int part() const { return bn == 256 ? 128 : bm == 128 ? 64 : 32; }
};

// Everything that the sizes decide.
struct Plan {
  bool narrow;         // the products of xent_narrow.hip
  Narrow nar;
  bool f32;            // three terms of everything
  int terms;           // of D
  int pairs;           // of planes, in the gradients' products
  int32_t few;         // of two terms the second is dropped where more rows count
  bool pack;           // whether W is packed
  bool few_wide;       // the products of xent_few.hpp
  bool keep;           // whether the scores stay in the workspace
  int32_t padded;      // elements of a packed row
  int64_t piece;       // columns of the vocabulary at a time (a multiple of 256)
  Shape scores, dx, dw;
  Splits dx_splits, dw_splits;
  int32_t few_parts;   // of dx, with few_wide
  // Workspace.
  size_t place, row, tokens, target, x, parts, xf, z, df, w, d, dxp, dwp, total;
};

// Tiles of 256 x 256 (one block per compute unit) or 128 x 128 (two, of which one's products run while the
// other stores), by their estimated time in units of 1000 cycles: a round of the chip of `steps` steps takes
// 1.65 or 1.11 of them each and what an epilogue of the larger tile shows.  Measured, us, the whole call with
// 256 / 128: scores, 2000 x 50000 x 512 551 / 518, 4096 x 131072 x 2048 7153 / 8545, FP32 500 x
// 30000 x 256 267 / 281; dW, 1999 x 50001 x 300 340 / 319, 100 x 50000 x 1024 180 / 163, 2000 x 50000 x 512
// 551 / 562.
Shape cheaper(int64_t m, int64_t n, int64_t steps, double epilogue) {
  if (m <= 128 || n <= 128) return {128, 128};
  const double big = double(up(up(m, 256) * up(n, 256), kNumCu)) * (1.65 * steps + epilogue);
  const double small = double(up(up(m, 128) * up(n, 128), kNumCu)) / 2 * (1.11 * steps + 0.35 * epilogue);
  return big <= small ? Shape{256, 256} : Shape{128, 128};
}
Shape few_rows(int64_t m) { return m <= 32 ? Shape{128, 32} : Shape{128, 64}; }
int blocks_of(Shape s) { return s.bn == 256 ? kNumCu : 2 * kNumCu; }
int64_t tiles_of(Shape s, int64_t m, int64_t n) { return up(m, s.bm) * up(n, s.bn); }

Plan plan_of(int32_t rows, int64_t vocab, int32_t dim, bool f32, bool backward) {
  Plan p = {};
  p.f32 = f32;
  const int planes = f32 ? 3 : 1;
  p.terms = f32 ? 3 : 2;
  p.few = few_of(vocab);
  p.pairs = f32 ? 6 : 2;
  // Rows of D's planes in all: a second term is that of at most `few` rows, which come first.
  const int64_t d_rows = f32 ? int64_t(rows) * 3 : int64_t(rows) + (rows < p.few ? rows : p.few);
  p.narrow = dim <= kNarrow;
  p.few_wide = f32 && !p.narrow && few_wide(rows, dim) && vocab <= kMaxPitch &&
               (!backward || rows * up(vocab, 256) * 256 * 6 <= kPieceBytes);
  p.pack = (f32 || dim % 8 != 0) && !p.few_wide;
  p.padded = (dim + kStepK - 1) / kStepK * kStepK;
  size_t at = 256;
  auto take = [&](size_t bytes) {
    const size_t was = at;
    at += align256(bytes);
    return was;
  };
  p.place = take(size_t(rows) * 4);
  p.row = take(size_t(rows) * 4);
  p.tokens = take(size_t(rows) * sizeof(Token));
  p.target = take(size_t(rows) * 4);
  if (p.narrow) {
    p.padded = dim <= 64 ? 64 : 128;
    p.x = take(size_t(rows) * size_t(p.padded) * 2 * planes);
    p.nar = narrow_plan(rows, vocab, dim, f32);
    const size_t parts = size_t(p.nar.splits) * p.nar.parts;
    p.parts = take(parts * size_t(rows) * sizeof(float2));
    if (backward) {
      p.dxp = take(parts * size_t(rows) * size_t(dim) * 4);
      if (p.nar.dw_splits > 1) p.dwp = take(size_t(p.nar.dw_splits) * size_t(vocab) * size_t(dim) * 4);
    }
    p.total = at;
    return p;
  }
  int64_t piece = up(vocab, 256) * 256;
  auto at_most = [&](int64_t v) {
    v = v / 256 * 256;
    if (v < 256) v = 256;
    if (piece > v) piece = v;
  };
  at_most(kMaxPitch);
  if (backward) at_most(kPieceBytes / (int64_t(rows > 0 ? rows : 1) * 2 * (f32 ? 3 : rows <= p.few ? 2 : 1)));
  if (p.pack) at_most(kPieceBytes / (int64_t(p.padded) * 2 * planes));
  // The parts of the rows' sums, of 32 columns each at least (few rows) or 64: the only limit of many rows without
  // gradients (2^20 x 2^20: 32 GB otherwise).
  at_most(kPieceBytes / (int64_t(rows > 0 ? rows : 1) * int64_t(sizeof(float2))) * (rows <= 64 ? 32 : 64));
  const int64_t pieces = up(vocab, piece);
  p.piece = up(up(vocab, pieces), 256) * 256;  // pieces of one size
  p.x = take(size_t(rows) * size_t(p.padded) * 2 * planes);
  const int64_t steps = up(dim, kStepK);
  p.scores = rows <= 64 ? few_rows(rows) : cheaper(rows, p.piece, steps * (f32 ? 6 : 1), 16);
  p.parts = take(size_t(up(p.piece, p.few_wide ? 32 : p.scores.part())) * size_t(rows) * sizeof(float2));
  if (p.few_wide) {
    p.xf = take(size_t(up(rows, 32) * 32) * size_t(p.padded) * 6);
    if (backward) {
      p.z = take(size_t(rows) * size_t(p.piece) * 4);
      p.df = take(size_t(up(rows, 32) * 32) * size_t(p.piece) * 6);
    }
  }
  p.w = p.pack ? take(size_t(p.piece) * size_t(p.padded) * 2 * planes) : 0;
  // Six pairs of planes' products again cost more than the scores' way through memory, where they fit: us, again /
  // kept, 1411 x 3929 x 2664 965 / 707, 3615 x 6188 x 724 1030 / 819, 2000 x 20000 x 512 1101 / 1012, x 196 619 / 597.
  // Of BF16 rows that are few beside dim, W's bytes once more do: 16 x 100000 x 512 130 / 114, 100 x 50000 x 1024
  // 164 / 147, 123 x 84048 x 492 209 / 197, 33 x 32001 x 136 45.8 / 45.6.
  p.keep = backward && !p.few_wide && pieces == 1 && rows > 0 &&
           rows * p.piece * 4 <= kPieceBytes && (f32 ? dim >= 192 : rows <= kFew && rows <= dim / 4);
  if (p.keep) p.z = take(size_t(rows) * size_t(p.piece) * 4);
  if (backward) {
    p.d = take(size_t(d_rows) * size_t(p.piece) * 2);
    // dx: the larger tiles where they, split, leave few compute units idle.
    const int64_t psteps = up(p.piece, kStepK);
    p.dx = {256, 256};
    if (rows <= 64)
      p.dx = few_rows(rows);
    else if (rows <= 128 || dim <= 128 ||
             tiles_of(p.dx, rows, dim) * split_steps(tiles_of(p.dx, rows, dim), psteps, kNumCu).count < kNumCu * 3 / 4)
      p.dx = {128, 128};
    p.dx_splits = split_steps(tiles_of(p.dx, rows, dim), psteps, blocks_of(p.dx));
    const int64_t area = int64_t(blocks_of(p.dx)) * p.dx.bm * p.dx.bn, whole = int64_t(rows) * dim;
    p.few_parts = p.few_wide ? few_parts(rows, vocab, dim) : 0;
    p.dxp = take(size_t(p.few_wide ? whole * p.few_parts : area > whole ? area : whole) * 4);
    p.dw = cheaper(p.piece, dim, up(rows, kStepK) * (rows <= p.few ? p.pairs : 1), 8);
    p.dw_splits = split_steps(tiles_of(p.dw, p.piece, dim), up(rows, kStepK), blocks_of(p.dw));
    if (p.dw_splits.count > 1) p.dwp = take(size_t(p.dw_splits.count) * size_t(p.piece) * size_t(dim) * 4);
  }
  p.total = at;
  return p;
}

template <bool AT, bool BT, bool LIVE_K, class Epi>
void run_gemm(const Gemm& g, const Epi& epi, Shape s, hipStream_t st) {
  if (s.bn == 256)
    launch_gemm<4, 4, 2, 2, 4, 1, AT, BT, LIVE_K>(g, epi, 2, st);
  else if (s.bm == 128)
    launch_gemm<2, 2, 2, 2, 3, 2, AT, BT, LIVE_K>(g, epi, 8, st);
  else if constexpr (!BT) {
    if (s.bm == 64)
      launch_gemm<1, 2, 4, 1, 4, 2, AT, BT, LIVE_K>(g, epi, 8, st);
    else
      launch_gemm<1, 1, 4, 1, 4, 2, AT, BT, LIVE_K>(g, epi, 8, st);
  }
}

template <int TERMS, class TX, class TW>
hipError_t launch_types(const embbag_xent_t& a, const Plan& p, char* ws, int32_t* status, hipStream_t st) {
  const int32_t N = a.rows, E = a.dim;
  const int64_t V = a.vocab;
  Head* head = reinterpret_cast<Head*>(ws);
  Rows rows = {head, reinterpret_cast<int32_t*>(ws + p.place), reinterpret_cast<int32_t*>(ws + p.row),
               reinterpret_cast<Token*>(ws + p.tokens), reinterpret_cast<float*>(ws + p.target)};
  __bf16* xp = reinterpret_cast<__bf16*>(ws + p.x);
  float2* parts = reinterpret_cast<float2*>(ws + p.parts);
  __bf16* wp = reinterpret_cast<__bf16*>(ws + p.w);
  __bf16* d = reinterpret_cast<__bf16*>(ws + p.d);
  float* dxp = reinterpret_cast<float*>(ws + p.dxp);
  const TX* x = static_cast<const TX*>(a.x);
  const TW* w = static_cast<const TW*>(a.table);
  TX* dx = static_cast<TX*>(a.grad_x);
  TW* dw = static_cast<TW*>(a.grad_table);
  const float unit = unit_of(a.scale);
  const int64_t xplane = int64_t(N) * p.padded, wplane = p.piece * p.padded;

  if (N > 0 && N <= kRowsAtOnce) {
    hipLaunchKernelGGL((xent_rows_pack<TERMS, TX>), dim3(unsigned(up(N, 16))), dim3(1024), 0, st, a.labels,
                       a.row_weights, N, int32_t(V), a.scale, rows, a.loss, status, x, a.x_stride, E, p.padded,
                       sign_of(a.scale), xp, xplane, dx, a.grad_x_stride);
  } else {
    hipLaunchKernelGGL(xent_rows, dim3(1), dim3(1024), 0, st, a.labels, a.row_weights, N, int32_t(V), a.scale,
                       rows, a.loss, status);
    if (N > 0)
      hipLaunchKernelGGL((xent_pack_x<TERMS, TX>), dim3(unsigned(up(N, kWavesPerBlock))), dim3(kBlock), 0, st,
                         x, a.x_stride, N, E, p.padded, sign_of(a.scale), rows.place, xp, xplane, dx,
                         a.grad_x_stride);
  }

  auto join_sums = [&](int32_t count, bool first, bool last) {
    if (N > 0 && N <= 256)
      hipLaunchKernelGGL(xent_join<4>, dim3(unsigned(up(N, 4))), dim3(1024), 0, st, parts, int64_t(N), count,
                         first, last, unit, rows, a.loss);
    else if (N > 0)
      hipLaunchKernelGGL(xent_join<64>, dim3(unsigned(up(N, 64))), dim3(1024), 0, st, parts, int64_t(N), count,
                         first, last, unit, rows, a.loss);
  };
  auto join_dx = [&](const PartCount& pc) {
    const int64_t most = (int64_t(1) << 25) / (E / 4);  // 32 threads for each
    for (int64_t r0 = 0; r0 < N; r0 += most) {
      const int64_t n = N - r0 < most ? N - r0 : most;
      launch_join_parts<TX>(dxp, pc, &head->live, r0 + n, E, rows.row, &head->factor, dx,
                            a.grad_x_stride, r0, st);
    }
  };
  auto join_dw = [&](const float* from, int32_t count, int64_t part, int64_t n, TW* to) {
    const int64_t most = (int64_t(1) << 25) / (E / 4);  // 32 threads for each
    for (int64_t r0 = 0; r0 < n; r0 += most) {
      const int64_t q = n - r0 < most ? n - r0 : most;
      launch_join_parts<TW>(from, {count, part, 0, 0, 0, 0}, nullptr, r0 + q, E, nullptr, &head->factor_w, to,
                            a.grad_table_stride, r0, st);
    }
  };
  if (p.narrow) {
    NarrowArgs q = {p.nar, p.f32 ? 3 : N <= p.few ? 2 : 1, p.few, w, sizeof(TW) == 2, a.table_stride, xp, xplane, head,
                    rows.tokens, rows.target,
                    unit, parts, dxp, dw, sizeof(TW) == 2, a.grad_table_stride, &head->factor_w};
    hipError_t e = launch_narrow_scores(q, st);
    if (e != hipSuccess) return e;
    join_sums(p.nar.splits * p.nar.parts, true, true);
    if (dx == nullptr && dw == nullptr) return hipGetLastError();
    const bool dw_parts = dw != nullptr && p.nar.dw_splits > 1;
    if (dx == nullptr) q.dx_parts = nullptr;
    if (dw_parts) q.dw = ws + p.dwp, q.dw_bf16 = false, q.dw_stride = E, q.dw_factor = nullptr;
    e = launch_narrow_gradients(q, st);
    if (e != hipSuccess) return e;
    if (dx != nullptr) join_dx({p.nar.splits * p.nar.parts, int64_t(N) * E, 0, 0, 0, 0});
    if (dw_parts) join_dw(reinterpret_cast<float*>(ws + p.dwp), p.nar.dw_splits, V * E, V, dw);
    return hipGetLastError();
  }
  const int64_t xpitch = int64_t(p.padded) * 2;
  const Side xs = {xp, xpitch, xplane * 2};
  int64_t packed = -1;  // the piece that wp holds
  auto side_w = [&](int64_t v0, int64_t n) {
    if (!p.pack) return Side{w + v0 * a.table_stride, a.table_stride * 2, 0};
    if (packed != v0) {
      const FastDiv chunks = fast_div(uint32_t(p.padded / 8));
      hipLaunchKernelGGL((xent_pack_w<TERMS, TW>), dim3(unsigned(up(n * (p.padded / 8), kBlock))),
                         dim3(kBlock), 0, st, w + v0 * a.table_stride, a.table_stride, n, E, chunks, wp,
                         wplane);
      packed = v0;
    }
    return Side{wp, xpitch, wplane * 2};
  };
  const int64_t dplane = int64_t(N) * p.piece;
  const Side ds = {d, p.piece * 2, dplane * 2};
  auto product_dw = [&](int64_t v0, int64_t n) {
    const Gemm g = {xs, ds, E, n, N, &head->live, p.pairs, p.dw_splits, 0, 0, p.few};
    TW* to = dw + v0 * a.grad_table_stride;
    if (p.dw_splits.count == 1) {
      run_gemm<true, true, true>(g, StoreEpi<TW>{to, a.grad_table_stride, E, &head->factor_w, 0, false}, p.dw, st);
    } else {
      float* dwp = reinterpret_cast<float*>(ws + p.dwp);
      run_gemm<true, true, true>(g, StoreEpi<float>{dwp, E, E, nullptr, p.piece * E, false}, p.dw, st);
      join_dw(dwp, p.dw_splits.count, p.piece * E, n, to);
    }
  };
  auto d_of_scores = [&](const float* z, __bf16* to, const Fragments& f) {
    hipLaunchKernelGGL(few_d, dim3(unsigned(up(int64_t(N) * (p.piece / 8), kBlock))), dim3(kBlock), 0, st, z,
                       fast_div(uint32_t(p.piece / 8)), V, rows.tokens, unit, &head->live, to, dplane, p.terms, f);
  };
  if constexpr (TERMS == 3) {
    if (p.few_wide) {
      const bool back = dx != nullptr || dw != nullptr;
      float* z = back ? reinterpret_cast<float*>(ws + p.z) : nullptr;
      const int32_t tiles = int32_t(up(N, 32));
      const Fragments xf = {reinterpret_cast<__bf16*>(ws + p.xf), tiles};
      const Fragments df = {dx != nullptr ? reinterpret_cast<__bf16*>(ws + p.df) : nullptr, tiles};
      hipLaunchKernelGGL(few_x, dim3(unsigned(up(int64_t(N) * (p.padded / 8), kBlock))), dim3(kBlock), 0, st, xp,
                         xplane, fast_div(uint32_t(p.padded / 8)), &head->live, xf);
      launch_few_scores(w, a.table_stride, V, E, N, xf, &head->live, z, p.piece,
                        StatsEpi<false>{parts, N, rows.tokens, rows.target, unit, 0, V, nullptr, 0}, st);
      join_sums(int32_t(up(V, 32)), true, true);
      if (!back) return hipGetLastError();
      d_of_scores(z, dw != nullptr ? d : nullptr, df);
      if (dx != nullptr) {
        launch_few_dx(w, a.table_stride, V, E, N, df, &head->live, p.few_parts, dxp,
                      int64_t(N) * E, st);
        join_dx({p.few_parts, int64_t(N) * E, 0, 0, 0, 0});
      }
      if (dw != nullptr) product_dw(0, V);
      return hipGetLastError();
    }
  }
  const int32_t pairs = TERMS == 3 ? 6 : 1;
  const Shape ss = p.scores;
  float* kept = p.keep && (dx != nullptr || dw != nullptr) ? reinterpret_cast<float*>(ws + p.z) : nullptr;
  for (int64_t v0 = 0; v0 < V; v0 += p.piece) {
    const int64_t n = V - v0 < p.piece ? V - v0 : p.piece;
    const Gemm g = {side_w(v0, n), xs, n, N, E, &head->live, pairs, {1, int32_t(up(E, kStepK))}, 0, 0, 0};
    auto stats = [&](auto keep) {
      run_gemm<false, false, false>(
          g, StatsEpi<keep.value>{parts, N, rows.tokens, rows.target, unit, v0, n, kept, p.piece}, ss, st);
    };
    if (kept != nullptr)
      stats(std::true_type());
    else
      stats(std::false_type());
    join_sums(int32_t(up(n, ss.part())), v0 == 0, v0 + n == V);
  }
  if (dx == nullptr && dw == nullptr) return hipGetLastError();

  for (int64_t v0 = 0; v0 < V; v0 += p.piece) {
    const int64_t n = V - v0 < p.piece ? V - v0 : p.piece;
    const Side wsd = side_w(v0, n);
    const Gemm g = {wsd, xs, n, N, E, &head->live, pairs, {1, int32_t(up(E, kStepK))}, 0, 0, 0};
    auto grad = [&](auto terms) {
      run_gemm<false, false, false>(
          g, GradEpi<terms.value>{d, p.piece, dplane, rows.tokens, unit, v0, n, &head->live, p.few}, ss, st);
    };
    if (kept != nullptr)
      d_of_scores(kept, d, Fragments{nullptr, 0});
    else
      grad(std::integral_constant<int, TERMS == 3 ? 3 : 2>());
    if (dx != nullptr) {
      const Gemm gx = {wsd, ds, E, N, n, &head->live, p.pairs, p.dx_splits, blocks_of(p.dx), up(p.piece, kStepK), p.few};
      run_gemm<true, false, false>(gx, StoreEpi<float>{dxp, E, E, nullptr, -1, v0 > 0}, p.dx, st);
    }
    if (dw != nullptr) product_dw(v0, n);
  }
  if (dx != nullptr)
    join_dx({p.dx_splits.count, 0, blocks_of(p.dx), p.dx.bm, int32_t(up(E, p.dx.bn)), up(p.piece, kStepK)});
  return hipGetLastError();
}

}  // namespace

size_t xent_workspace(int32_t rows, int64_t vocab, int32_t dim, bool f32, bool backward) {
  return plan_of(rows, vocab, dim, f32, backward).total;
}

hipError_t launch_xent(const embbag_xent_t& a, char* ws, int32_t* status, hipStream_t st) {
  if (a.rows == 0 && a.grad_table == nullptr) return hipSuccess;
  const bool xb = a.x_type == EMBBAG_BF16, wb = a.table_type == EMBBAG_BF16;
  const Plan p = plan_of(a.rows, a.vocab, a.dim, !(xb && wb), a.grad_x != nullptr || a.grad_table != nullptr);
  if (xb && wb) return launch_types<1, __bf16, __bf16>(a, p, ws, status, st);
  if (xb) return launch_types<3, __bf16, float>(a, p, ws, status, st);
  if (wb) return launch_types<3, float, __bf16>(a, p, ws, status, st);
  return launch_types<3, float, float>(a, p, ws, status, st);
}

}  // namespace embbag
