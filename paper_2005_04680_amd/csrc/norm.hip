// RMS norm of rows with the residual's addition, into FP32, BF16 or 8-bit
// microscaled rows, and its gradients.
//
// A row lives in the registers of T threads, 8 consecutive elements (a chunk) at a
// time: every input is read once and every output written once.  The sum of
// squares is FP64, so that it neither overflows nor loses small rows (an FP32 square does beyond
// 1.8e19 and below 1e-23).  The forward's outputs are FP64 to their rounding to FP32, from which BF16 and 8-bit
// rows are rounded: an element lies next to a border of E4M3's rounding often enough that the last bits of FP32
// arithmetic move codes (of 16M elements some tens, 2^-4 of the element each; the one rounding to FP32 about 9, which
// then are those of `out` and not of the exact norm).  The gradient works in FP32, its factor 1/sqrt as a power
// of two and a rest: its exponent scales the elements first, which is exact.
//
// Bound by bytes; the next row's loads are on their way during a row (16384 x 4096 BF16 gradient 171 us without,
// 118 with).  Measured, us: 16384 x 4096 BF16 with a residual 102 (537 MB at 5.26 TB/s; a copy 5.24), 4096 x 4096
// BF16 with an FP32 residual into 8 bits 32 (185 MB at 5.8 TB/s, partly from the caches) and 9.5 to read
// back, the gradient of 16384 x 4096 with dsum 118 (4.6 TB/s).  FP64 costs rows of more than 8192 elements 9 %
// (1024 threads, 16 elements each, spill; 4000 x 16384 100 us in FP32, 109) and the others nothing.  The gradient of such
// rows has no room for the next one and spills too: 4000 x 16384 with dsum 192 us, 2.7 TB/s.
#include <type_traits>

#include "head.hpp"

namespace embbag {
namespace {

constexpr int kChunk = 8;  // elements of a thread's loads

// 1/sqrt(mean + eps) = rest * 2^exp, rest in (0.7, 1.5) (0 or NaN where the sum is not finite): the
// FP64 number is split exactly, its mantissa rounded to FP32 once.
struct Inverse {
  float rest;
  int exp;
};
__device__ __forceinline__ Inverse inverse_of(double sum, double per, double eps) {
  const double m = sum * per + eps;
  const int e = __builtin_amdgcn_frexp_exp(m);
  const float f = float(__builtin_amdgcn_frexp_mant(m));  // [0.5, 1)
  const int odd = e & 1;
  return {1.f / sqrtf(odd ? f + f : f), -((e - odd) / 2)};
}
// The same in FP64: a Newton step from FP32's 24 bits.
__device__ __forceinline__ double inverse64_of(double sum, double per, double eps) {
  const double m = sum * per + eps;
  const int e = __builtin_amdgcn_frexp_exp(m);
  const int odd = e & 1;
  const double f = __builtin_amdgcn_frexp_mant(m) * (odd ? 2.0 : 1.0);
  const double r = double(1.f / sqrtf(float(f)));
  return m - m == 0.0 ? ldexp(r * fma(-0.5 * f * r, r, 1.5), -((e - odd) / 2)) : r;  // (0 of an infinity)
}
// x / sqrt(mean + eps).
__device__ __forceinline__ float times(float x, const Inverse& s) { return ldexpf(x, s.exp) * s.rest; }

// 8 elements of a row from chunk c on (zeros past dim; dim % 4 == 0).
template <class T>
__device__ __forceinline__ void load_chunk(const T* row, int c, int dim, float (&v)[8]) {
  Eight<T> x;
  x.load(row + c * kChunk, dim - c * kChunk);
  x.values(v);
}
__device__ __forceinline__ void store_chunk(float* row, int c, int dim, const float (&v)[8]) {
  const int e = c * kChunk;
  if (e < dim) store4(row + e, f4{v[0], v[1], v[2], v[3]});
  if (e + 4 < dim) store4(row + e + 4, f4{v[4], v[5], v[6], v[7]});
}
__device__ __forceinline__ void store_chunk(__bf16* row, int c, int dim, const float (&v)[8]) {
  const int e = c * kChunk;
  const u4 w = pack16(v);
  if (e + 4 < dim)
    store16(row + e, w);
  else if (e < dim)
    *reinterpret_cast<u2*>(row + e) = u2{w.x, w.y};
}

// The weights of a chunk: FP32, BF16 or none (ones).
__device__ __forceinline__ void load_weight(const void* w, bool bf16, int c, int dim, float (&v)[8]) {
  if (w == nullptr) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = 1.f;
  } else if (bf16) {
    load_chunk(static_cast<const __bf16*>(w), c, dim, v);
  } else {
    load_chunk(static_cast<const float*>(w), c, dim, v);
  }
}

// The sum over the T threads of a row of each of v's N numbers, in all of them.  `slots`: N doubles
// per wavefront; two calls in turn need two places.
template <int T, int N>
__device__ __forceinline__ void row_sum(double (&v)[N], double* slots) {
#pragma unroll
  for (int d = 1; d < (T < kWave ? T : kWave); d *= 2)
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += __shfl_xor(v[i], d, kWave);
  if constexpr (T > kWave) {
    constexpr int W = T / kWave;
    if (lane_id() == 0) {
#pragma unroll
      for (int i = 0; i < N; ++i) slots[wave_id() * N + i] = v[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      v[i] = slots[i];
#pragma unroll
      for (int w = 1; w < W; ++w) v[i] += slots[w * N + i];
    }
  }
}

// The scale byte of 32 elements whose largest magnitude has the FP32 bits `amax` and the factor 2^-e:
// the smallest 2^e with amax <= 448 * 2^e (the carry of a mantissa beyond 1.75 raises it).
__device__ __forceinline__ uint32_t mx8_scale_of(uint32_t amax, float* factor) {
  if (amax >= 0x7F800000u) {  // an infinity or a NaN
    *factor = 0.f;
    return 255u;
  }
  const int e = max(int((amax + 0x1FFFFFu) >> 23) - 135, -127);
  *factor = __uint_as_float(uint32_t(127 - e) << 23);
  return amax == 0u ? 0u : uint32_t(e + 127);
}

// 8 elements as E4M3 codes of their block (four neighbouring lanes), nearest, ties to even; no
// element passes 448, the largest code.
__device__ __forceinline__ u2 mx8_codes(const float (&y)[8], uint32_t* byte) {
  uint32_t amax = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) amax = max(amax, __float_as_uint(y[i]) & 0x7FFFFFFFu);
  amax = max(amax, uint32_t(__shfl_xor(int(amax), 1, 4)));
  amax = max(amax, uint32_t(__shfl_xor(int(amax), 2, 4)));
  float f;
  *byte = mx8_scale_of(amax, &f);
  if (*byte == 255u) return u2{0u, 0u};
  int lo = 0, hi = 0;
  lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[0] * f, y[1] * f, lo, false);
  lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[2] * f, y[3] * f, lo, true);
  hi = __builtin_amdgcn_cvt_pk_fp8_f32(y[4] * f, y[5] * f, hi, false);
  hi = __builtin_amdgcn_cvt_pk_fp8_f32(y[6] * f, y[7] * f, hi, true);
  return u2{uint32_t(lo), uint32_t(hi)};
}

template <int T>
constexpr int kNormThreads = T > kBlock ? T : kBlock;

// T threads per row, NC chunks of each.  A block takes every gridDim.x-th group of rows; `out`, the
// 8-bit rows and the sum are each optional, `residual` too.  Inputs may be outputs: a row is read before
// it is written.
template <int T, int NC, class TX, class TR, class TO>
__global__ __launch_bounds__(kNormThreads<T>) void norm_rows(NormArgs a) {
  constexpr int R = kNormThreads<T> / T;  // rows at a time
  __shared__ double slots[2][T > kWave ? T / kWave : 1];
  const int t = threadIdx.x % T;
  const int dim = a.dim, padded = mx4_scale_bytes(dim) * 4;  // chunks of a row of codes
  float w[NC][8];
#pragma unroll
  for (int i = 0; i < NC; ++i) load_weight(a.weight, a.weight_bf16, t + i * T, dim, w[i]);
  // The next row's inputs are on their way while a row is summed and stored.
  Eight<TX> nx[NC];
  Eight<TR> nr[NC];
  auto fetch = [&](int64_t row) {
    const int last = row < a.rows ? dim : 0;
    const int64_t at = row < a.rows ? row : 0;
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      const int e = (t + i * T) * kChunk;
      nx[i].load(static_cast<const TX*>(a.x) + at * a.x_stride + e, last - e);
    }
    if (a.residual == nullptr) return;
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      const int e = (t + i * T) * kChunk;
      nr[i].load(static_cast<const TR*>(a.residual) + at * a.residual_stride + e, last - e);
    }
  };
  fetch(int64_t(blockIdx.x) * R + threadIdx.x / T);
  int turn = 0;
  for (int64_t row0 = int64_t(blockIdx.x) * R; row0 < a.rows; row0 += int64_t(gridDim.x) * R) {
    const int64_t row = row0 + threadIdx.x / T;
    const bool in = row < a.rows;
    const int last = in ? dim : 0;  // (the others of the wavefront need its lanes)
    Eight<TX> cx[NC];
    Eight<TR> cr[NC];
#pragma unroll
    for (int i = 0; i < NC; ++i) cx[i] = nx[i], cr[i] = nr[i];
    if (row0 + int64_t(gridDim.x) * R < a.rows) fetch(row + int64_t(gridDim.x) * R);
    auto sum_of = [&](int i, double (&h)[8]) {
      float x[8], q[8];
      cx[i].values(x);
#pragma unroll
      for (int j = 0; j < 8; ++j) h[j] = double(x[j]);
      if (a.residual == nullptr) return;
      cr[i].values(q);
#pragma unroll
      for (int j = 0; j < 8; ++j) h[j] += double(q[j]);
    };
    double sum[1] = {0.0};
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      double h[8];
      sum_of(i, h);
#pragma unroll
      for (int j = 0; j < 8; ++j) sum[0] = fma(h[j], h[j], sum[0]);
      if (a.sum_out != nullptr) {
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = float(h[j]);
        store_chunk(static_cast<TR*>(a.sum_out) + (in ? row : 0) * a.sum_stride, t + i * T, last, v);
      }
    }
    row_sum<T, 1>(sum, slots[turn]);
    turn ^= 1;
    const double s = inverse64_of(sum[0], a.per, a.eps);
    float y[NC][8];
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      double h[8];
      cx[i].again();
      if (a.residual != nullptr) cr[i].again();
      sum_of(i, h);
#pragma unroll
      for (int j = 0; j < 8; ++j) y[i][j] = float(h[j] * s * double(w[i][j]));
    }
    if (a.out != nullptr) {
      TO* p = static_cast<TO*>(a.out) + (in ? row : 0) * a.out_stride;
#pragma unroll
      for (int i = 0; i < NC; ++i) store_chunk(p, t + i * T, last, y[i]);
    }
    if (a.codes != nullptr) {
#pragma unroll
      for (int i = 0; i < NC; ++i) {
        const int c = t + i * T;
        if (c >= (dim + kChunk - 1) / kChunk) {  // (a NaN of the row makes NaN of zeros)
#pragma unroll
          for (int j = 0; j < 8; ++j) y[i][j] = 0.f;
        }
        uint32_t byte;
        const u2 codes = mx8_codes(y[i], &byte);
        if (!in || c >= padded) continue;
        *reinterpret_cast<u2*>(a.codes + row * padded * kChunk + c * kChunk) = codes;
        if (c % 4 == 0) a.scales[row * (padded / 4) + c / 4] = uint8_t(byte);
      }
    }
  }
}

// Gradients: with n = h / sqrt(mean(h^2) + eps) and g = w dy,
//   dh = (g - n mean(n g)) / sqrt(mean(h^2) + eps) + dsum,   dw = sum over the rows of dy n.
// A thread keeps its columns' share of dw in registers over all of its rows; a block adds its groups' in
// order and writes one row of `parts`, which norm_join adds: no atomics, the same bits in every run.
template <int T, int NC, class TY, class TH>
__global__ __launch_bounds__(kNormThreads<T>) void norm_grad_rows(NormGradArgs a) {
  constexpr int R = kNormThreads<T> / T;
  __shared__ double slots[2][T > kWave ? 2 * (T / kWave) : 2];
  __shared__ __align__(16) float sums[R > 1 ? kBlock * NC * 8 : 4];
  const int t = threadIdx.x % T;
  const int dim = a.dim;
  // 1024 threads have 128 registers each: the weights are loaded again for every row then, and no row ahead.
  constexpr bool ROOM = T < 1024;
  float w[NC][8], dw[NC][8];
#pragma unroll
  for (int i = 0; i < NC; ++i) {
    if (ROOM) load_weight(a.weight, a.weight_bf16, t + i * T, dim, w[i]);
#pragma unroll
    for (int j = 0; j < 8; ++j) dw[i][j] = 0.f;
  }
  // The next row's inputs are on their way while a row is summed and stored.
  Eight<TH> nh[NC], nd[NC];
  Eight<TY> ny[NC];
  auto fetch = [&](int64_t row) {
    const int last = row < a.rows ? dim : 0;
    const int64_t at = row < a.rows ? row : 0;
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      const int e = (t + i * T) * kChunk;
      nh[i].load(static_cast<const TH*>(a.h) + at * a.h_stride + e, last - e);
      ny[i].load(static_cast<const TY*>(a.dy) + at * a.dy_stride + e, last - e);
    }
    if (a.dsum == nullptr) return;
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      const int e = (t + i * T) * kChunk;
      nd[i].load(static_cast<const TH*>(a.dsum) + at * a.dsum_stride + e, last - e);
    }
  };
  if (ROOM) fetch(int64_t(blockIdx.x) * R + threadIdx.x / T);
  int turn = 0;
  for (int64_t row0 = int64_t(blockIdx.x) * R; row0 < a.rows; row0 += int64_t(gridDim.x) * R) {
    const int64_t row = row0 + threadIdx.x / T;
    const bool in = row < a.rows;
    const int last = in ? dim : 0;
    const int64_t at = in ? row : 0;
    if (!ROOM) {
      fetch(row);
#pragma unroll
      for (int i = 0; i < NC; ++i) load_weight(a.weight, a.weight_bf16, t + i * T, dim, w[i]);
    }
    float h[NC][8], y[NC][8];
    Eight<TH> d[NC];
#pragma unroll
    for (int i = 0; i < NC; ++i) nh[i].values(h[i]), ny[i].values(y[i]), d[i] = nd[i];
    if (ROOM && row0 + int64_t(gridDim.x) * R < a.rows) fetch(row + int64_t(gridDim.x) * R);
    double sum[2] = {0.0, 0.0};
#pragma unroll
    for (int i = 0; i < NC; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        sum[0] = fma(double(h[i][j]), double(h[i][j]), sum[0]);
        sum[1] = fma(double(h[i][j]), double(w[i][j] * y[i][j]), sum[1]);
      }
    row_sum<T, 2>(sum, slots[turn]);
    turn ^= 1;
    const Inverse s = inverse_of(sum[0], a.per, a.eps);
    const float k = float(ldexp(sum[1] * a.per * double(s.rest), s.exp));  // mean(n g)
#pragma unroll
    for (int i = 0; i < NC; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float n = times(h[i][j], s);
        dw[i][j] += in ? y[i][j] * n : 0.f;
        h[i][j] = times(w[i][j] * y[i][j] - n * k, s);
      }
    if (a.dsum != nullptr) {
#pragma unroll
      for (int i = 0; i < NC; ++i) {
        float q[8];
        d[i].values(q);
#pragma unroll
        for (int j = 0; j < 8; ++j) h[i][j] += q[j];
      }
    }
    TH* p = static_cast<TH*>(a.dh) + at * a.dh_stride;
#pragma unroll
    for (int i = 0; i < NC; ++i) store_chunk(p, t + i * T, last, h[i]);
  }
  if (a.parts == nullptr) return;
  if constexpr (R > 1) {
#pragma unroll
    for (int i = 0; i < NC; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) sums[(threadIdx.x / T * NC + i) * T * 8 + t * 8 + j] = dw[i][j];
    __syncthreads();
    // Thread u takes float u, u + 256, ... of a row of T * NC chunks.
    for (int u = threadIdx.x; u < dim; u += kBlock) {
      float s = 0.f;
#pragma unroll 4
      for (int r = 0; r < R; ++r) s += sums[r * NC * T * 8 + u];
      a.parts[int64_t(blockIdx.x) * dim + u] = s;
    }
  } else {
#pragma unroll
    for (int i = 0; i < NC; ++i) store_chunk(a.parts + int64_t(blockIdx.x) * dim, t + i * T, dim, dw[i]);
  }
}

// dw = the sum of the parts [blocks][dim]: 8 groups of 4 columns per block, every 128-th part per
// thread, then the threads' sums in order.
template <class TW>
__global__ __launch_bounds__(1024) void norm_join(const float* __restrict__ parts, int32_t blocks,
                                                  int32_t dim, TW* __restrict__ dw) {
  __shared__ f4 sums[128][8];
  const int c = threadIdx.x % 8, p = threadIdx.x / 8;
  const int e = (blockIdx.x * 8 + c) * 4;
  f4 s = {0.f, 0.f, 0.f, 0.f};
  if (e < dim) {
#pragma unroll 4
    for (int b = p; b < blocks; b += 128) s += load4(parts + int64_t(b) * dim + e);
  }
  sums[p][c] = s;
  __syncthreads();
  for (int d = 64; d > 0; d /= 2) {
    if (p < d) sums[p][c] += sums[p + d][c];
    __syncthreads();
  }
  if (p == 0 && e < dim) store4(dw + e, sums[0][c]);
}

// 8-bit rows as values; a thread per 8 elements.
template <class T>
__global__ __launch_bounds__(kBlock) void mx8_read(const uint8_t* __restrict__ codes,
                                                   const uint8_t* __restrict__ scales, int32_t dim,
                                                   int64_t chunks, FastDiv per_row, int64_t row0,
                                                   T* __restrict__ dst, int64_t stride) {
  const int64_t i = int64_t(blockIdx.x) * kBlock + threadIdx.x;
  if (i >= chunks) return;
  const uint32_t q = quotient(uint32_t(i), per_row);
  const int c = int(uint32_t(i) - q * per_row.div);
  const int64_t row = row0 + q;
  const int sb = mx4_scale_bytes(dim);
  const u2 v = *reinterpret_cast<const u2*>(codes + row * sb * 32 + c * kChunk);
  const uint32_t b = scales[row * sb + c / 4];
  const float s = b == 0u ? __uint_as_float(0x00400000u)
                          : b == 255u ? __uint_as_float(0x7FC00000u) : __uint_as_float(b << 23);
  const f2 p0 = __builtin_amdgcn_cvt_pk_f32_fp8(int(v.x), false);
  const f2 p1 = __builtin_amdgcn_cvt_pk_f32_fp8(int(v.x), true);
  const f2 p2 = __builtin_amdgcn_cvt_pk_f32_fp8(int(v.y), false);
  const f2 p3 = __builtin_amdgcn_cvt_pk_f32_fp8(int(v.y), true);
  const float y[8] = {p0.x * s, p0.y * s, p1.x * s, p1.y * s, p2.x * s, p2.y * s, p3.x * s, p3.y * s};
  store_chunk(dst + row * stride, c, dim, y);
}

// Threads per row and chunks per thread: the fewest threads that hold a row (of whole 128-element
// groups where codes are written) in one chunk each up to 64, then in two.
template <class Fn>
void for_shape(int32_t dim, Fn fn) {
  if (dim <= 128)
    fn(std::integral_constant<int, 16>(), std::integral_constant<int, 1>());
  else if (dim <= 256)
    fn(std::integral_constant<int, 32>(), std::integral_constant<int, 1>());
  else if (dim <= 512)
    fn(std::integral_constant<int, 64>(), std::integral_constant<int, 1>());
  else if (dim <= 1024)
    fn(std::integral_constant<int, 64>(), std::integral_constant<int, 2>());
  else if (dim <= 2048)
    fn(std::integral_constant<int, 256>(), std::integral_constant<int, 1>());
  else if (dim <= 4096)
    fn(std::integral_constant<int, 256>(), std::integral_constant<int, 2>());
  else if (dim <= 8192)
    fn(std::integral_constant<int, 512>(), std::integral_constant<int, 2>());
  else
    fn(std::integral_constant<int, 1024>(), std::integral_constant<int, 2>());
}

template <class Fn>
void for_type(bool bf16, Fn fn) {
  if (bf16)
    fn(__bf16());
  else
    fn(float());
}

// Blocks of `rows` rows, `at_once` of them per block: as many as the chip holds at once (2048 threads
// per compute unit), or fewer.
int64_t grid_of(int64_t rows, int at_once, int threads, int share) {
  const int64_t want = (rows + at_once - 1) / at_once;
  const int64_t most = int64_t(kNumCu) * (2048 / threads) / share;
  return want < most ? want : most;
}

// Blocks of the gradient: each writes a row of parts.
int64_t grad_blocks(int64_t rows, int32_t dim) {
  int64_t n = 0;
  for_shape(dim, [&](auto T, auto) {
    constexpr int threads = kNormThreads<T.value>;
    n = grid_of(rows, threads / T.value, threads, 2);
  });
  return n;
}

}  // namespace

hipError_t launch_rmsnorm(const NormArgs& a, bool x_bf16, bool r_bf16, bool out_bf16, hipStream_t st) {
  if (a.rows == 0) return hipSuccess;
  for_shape(a.dim, [&](auto T, auto NC) {
    for_type(x_bf16, [&](auto x) {
      for_type(r_bf16, [&](auto r) {
        for_type(out_bf16, [&](auto o) {
          constexpr int threads = kNormThreads<T.value>;
          hipLaunchKernelGGL((norm_rows<T.value, NC.value, decltype(x), decltype(r), decltype(o)>),
                             dim3(unsigned(grid_of(a.rows, threads / T.value, threads, 1))),
                             dim3(threads), 0, st, a);
        });
      });
    });
  });
  return hipGetLastError();
}

size_t rmsnorm_grad_workspace(int64_t rows, int32_t dim) {
  return (size_t(grad_blocks(rows, dim)) * size_t(dim) * 4 + 255) / 256 * 256;
}

hipError_t launch_rmsnorm_grad(NormGradArgs a, bool y_bf16, bool h_bf16, void* dweight, char* ws,
                               hipStream_t st) {
  a.parts = dweight != nullptr ? reinterpret_cast<float*>(ws) : nullptr;
  const int64_t blocks = grad_blocks(a.rows, a.dim);
  if (blocks > 0) {
    for_shape(a.dim, [&](auto T, auto NC) {
      for_type(y_bf16, [&](auto y) {
        for_type(h_bf16, [&](auto h) {
          hipLaunchKernelGGL((norm_grad_rows<T.value, NC.value, decltype(y), decltype(h)>),
                             dim3(unsigned(blocks)), dim3(kNormThreads<T.value>), 0, st, a);
        });
      });
    });
  }
  if (dweight != nullptr) {
    for_type(a.weight_bf16, [&](auto w) {
      using TW = decltype(w);
      hipLaunchKernelGGL(norm_join<TW>, dim3(unsigned((a.dim + 31) / 32)), dim3(1024), 0, st, a.parts,
                         int32_t(blocks), a.dim, static_cast<TW*>(dweight));
    });
  }
  return hipGetLastError();
}

hipError_t launch_mx8_dequantize(const uint8_t* codes, const uint8_t* scales, int64_t rows,
                                 int32_t dim, void* dst, bool bf16, int64_t dst_stride, hipStream_t st) {
  const int32_t per = (dim + kChunk - 1) / kChunk;
  const int64_t most = ((int64_t(1) << 30) / per);  // rows per launch: chunks are numbered in 31 bits
  for (int64_t row0 = 0; row0 < rows; row0 += most) {
    const int64_t n = rows - row0 < most ? rows - row0 : most;
    for_type(bf16, [&](auto t) {
      using T = decltype(t);
      hipLaunchKernelGGL(mx8_read<T>, dim3(unsigned((n * per + kBlock - 1) / kBlock)), dim3(kBlock), 0,
                         st, codes, scales, dim, n * per, fast_div(uint32_t(per)), row0,
                         static_cast<T*>(dst), dst_stride);
    });
  }
  return hipGetLastError();
}

}  // namespace embbag
