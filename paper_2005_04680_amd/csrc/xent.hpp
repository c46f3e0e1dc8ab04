// What the kernels of the cross entropy share: exponents, BF16 terms, the rows that count.
#pragma once

#include "head.hpp"

namespace embbag {
namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }

// D of BF16 sides has a second term where at most so many rows count, or the table has fewer rows than
// kSmallTable: the few roundings of the labels' elements do not average out, and over a small table such an element,
// 1 - p, is off by as much as p in the same direction in every row.  How many rows count is known on the device.
constexpr int32_t kFew = 256;
constexpr int64_t kSmallTable = 1024;
inline int32_t few_of(int64_t vocab) { return vocab < kSmallTable ? INT32_MAX : kFew; }

// Numbers as sums of three BF16 terms, each the nearest to what is left.  What BF16 cannot hold, beyond its
// largest number (infinities and NaN too), comes in the last term, which meets the other side's first alone.
__device__ __forceinline__ void nearest_terms(const float (&x)[8], u4 (&t)[3]) {
  constexpr float kLargest = 3.3895313892515355e38f;
  float v[8], over[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    v[i] = __builtin_amdgcn_fmed3f(x[i], -kLargest, kLargest);
    over[i] = x[i] - v[i];
  }
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    t[k] = pack16(v);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] -= (i % 2 ? bf16_hi : bf16_lo)(t[k][i / 2]);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] += over[i];
  t[2] = pack16(v);
}

// Scores enter the exponentials as 2^(score * log2(e)), in one FMA: their sums are taken with x times the
// scale's sign, of which `unit` = |scale| log2(e) makes the exponent.  (A scale of 0 makes x 0, and its
// unit is any.)
__host__ __device__ __forceinline__ float sign_of(float scale) {
  return scale > 0.f ? 1.f : scale < 0.f ? -1.f : 0.f;
}
__host__ __device__ __forceinline__ float unit_of(float scale) {
  return scale == 0.f ? 1.f : (scale < 0.f ? -scale : scale) * kLog2e;
}

// What the backward needs of a row that counts.
struct Token {
  float top;    // about its largest score's exponent
  float inv;    // 1 / the sum of 2^(exponent - top)
  float ratio;  // its weight over the largest
  int label;
};

// In the workspace.
struct Head {
  int32_t live;   // rows that count
  float largest;  // of their weights' magnitudes
  float factor;   // scale * largest, of dx
  float factor_w; // |scale| * largest, of dW (x has the scale's sign)
};

struct Rows {
  Head* head;
  int32_t* place;  // [rows]: among the rows that count, or -1
  int32_t* row;    // [live]: the row at a place
  Token* tokens;   // [live]
  float* target;   // [live]: the label's sum
};

}  // namespace

// The products of narrow tables (dim <= kNarrow), whose D stays in registers.  Sizes as xent.hip's plan has
// them.
constexpr int kNarrow = 128;
struct Narrow {
  int32_t rows, dim;
  int64_t vocab;
  int bm;               // rows of x per block
  int32_t splits, per;  // ranges of the vocabulary: blocks of it, and rows of W in each
  int parts;            // parts per range (wavefronts that share a block's rows of x)
  int32_t dw_splits, dw_per;  // ranges of the rows that count, rows in each
};
Narrow narrow_plan(int32_t rows, int64_t vocab, int32_t dim, bool f32);
struct NarrowArgs {
  Narrow n;
  int terms;  // of D (1: 2 where at most `few` rows count); of the sides 3 if that is 3, else 1
  int32_t few;
  const void* table;
  bool table_bf16;
  int64_t table_stride;
  const void* x;       // planes [rows][padded]
  int64_t x_plane;     // elements
  const void* head;    // Head, Token[rows], the labels' sums
  const void* tokens;
  float* target;
  float unit;
  void* sums;          // float2 [splits * parts][rows]: exponents and sums
  float* dx_parts;     // [splits * parts][rows][dim], null if not wanted
  void* dw;            // table's type, or FP32 parts [dw_splits][vocab][dim]; null if not wanted
  bool dw_bf16;
  int64_t dw_stride;
  const float* dw_factor;  // null for parts
};
hipError_t launch_narrow_scores(const NarrowArgs& a, hipStream_t st);
hipError_t launch_narrow_gradients(const NarrowArgs& a, hipStream_t st);

}  // namespace embbag
