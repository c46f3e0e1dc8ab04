// Definitions shared by the kernels of the output head: 4-bit microscaled
// tables, logits and distillation.
#pragma once

#include "common.hpp"

namespace embbag {

constexpr int kMxBlock = 32;         // elements that share a scale
constexpr int kMxMaxDim = 16384;
constexpr int kMaxTeacher = 1024;    // a teacher's entries per row

typedef uint32_t u4 __attribute__((ext_vector_type(4)));
typedef float f2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf8 __attribute__((ext_vector_type(8)));

// Blocks of a row, and bytes of its row of scales (whole words).
__host__ __device__ constexpr int mx4_blocks(int dim) { return (dim + kMxBlock - 1) / kMxBlock; }
__host__ __device__ constexpr int mx4_scale_bytes(int dim) { return (mx4_blocks(dim) + 3) / 4 * 4; }

// A scale byte as the FP32 operand of the conversion instructions, which take
// its exponent field: byte 0 stands for 2^-127, byte 255 for NaN.
__device__ __forceinline__ float mx4_scale(uint32_t byte) { return __uint_as_float(byte << 23); }

// Scale byte of a block whose largest magnitude has the FP32 bits `amax`, and
// the factor 2^-e that brings its elements to the codes' range.  floor(log2) is the
// exponent field (a subnormal's e is below -127 either way).  The factor is a normal
// number: -127 <= e <= 125.
__device__ __forceinline__ uint32_t mx4_scale_of(uint32_t amax, float* factor) {
  if (amax >= 0x7F800000u) {  // an infinity or a NaN
    *factor = 0.f;
    return 255u;
  }
  const int e = max(int(amax >> 23) - 129, -127);
  *factor = __uint_as_float(uint32_t(127 - e) << 23);
  return amax == 0u ? 0u : uint32_t(e + 127);
}

// Codes of 8 elements scaled to the codes' range: nearest, ties to the even code,
// beyond 6 to 6 (the instruction's own rounding).
__device__ __forceinline__ uint32_t mx4_codes8(const float (&y)[8]) {
  uint32_t c = 0;
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, y[0], y[1], 1.0f, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, y[2], y[3], 1.0f, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, y[4], y[5], 1.0f, 2);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, y[6], y[7], 1.0f, 3);
  return c;
}

// The 8 values of a word of codes.
__device__ __forceinline__ void mx4_values8(uint32_t codes, float scale, float (&v)[8]) {
  const f2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 0);
  const f2 b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 1);
  const f2 c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 2);
  const f2 d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 3);
  v[0] = a.x, v[1] = a.y, v[2] = b.x, v[3] = b.y;
  v[4] = c.x, v[5] = c.y, v[6] = d.x, v[7] = d.y;
}

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// Two FP32 values to BF16, nearest, ties to even.
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  const bf2 v = {__bf16(a), __bf16(b)};
  return __builtin_bit_cast(uint32_t, v);
}

// A buffer element as FP32, and back (BF16 to nearest even).
__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__bf16 x) { return float(x); }

// 4 consecutive elements: 16 bytes of FP32, 8 of BF16.
__device__ __forceinline__ f4 load4(const float* p) { return *reinterpret_cast<const f4*>(p); }
__device__ __forceinline__ f4 load4(const __bf16* p) {
  const u2 w = *reinterpret_cast<const u2*>(p);
  return f4{bf16_lo(w.x), bf16_hi(w.x), bf16_lo(w.y), bf16_hi(w.y)};
}
__device__ __forceinline__ void store4(float* p, const f4& v) { *reinterpret_cast<f4*>(p) = v; }
__device__ __forceinline__ void store4(__bf16* p, const f4& v) {
  *reinterpret_cast<u2*>(p) = u2{pack_bf16(v.x, v.y), pack_bf16(v.z, v.w)};
}

// 16 bytes of a row: 4 FP32 or 8 BF16 elements.
template <class T>
constexpr int kVec = 16 / int(sizeof(T));
__device__ __forceinline__ void unpack16(const u4& w, float (&v)[4]) {
  v[0] = __uint_as_float(w.x), v[1] = __uint_as_float(w.y);
  v[2] = __uint_as_float(w.z), v[3] = __uint_as_float(w.w);
}
__device__ __forceinline__ void unpack16(const u4& w, float (&v)[8]) {
  v[0] = bf16_lo(w.x), v[1] = bf16_hi(w.x), v[2] = bf16_lo(w.y), v[3] = bf16_hi(w.y);
  v[4] = bf16_lo(w.z), v[5] = bf16_hi(w.z), v[6] = bf16_lo(w.w), v[7] = bf16_hi(w.w);
}
__device__ __forceinline__ u4 pack16(const float (&v)[4]) {
  return u4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]),
            __float_as_uint(v[3])};
}
__device__ __forceinline__ u4 pack16(const float (&v)[8]) {
  return u4{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]),
            pack_bf16(v[6], v[7])};
}

// 16 bytes to or from a row of any alignment (the hardware takes vector accesses at element
// boundaries).
typedef u4 u4_any __attribute__((aligned(2)));
__device__ __forceinline__ void store16(void* p, const u4& v) { *static_cast<u4_any*>(p) = v; }
__device__ __forceinline__ u4 load16(const void* p) { return *static_cast<const u4_any*>(p); }

__device__ __forceinline__ float low() { return -__builtin_inff(); }

// 16 bytes of a row of which n elements exist: the others become -infinity.
template <class T>
__device__ __forceinline__ u4 load_vec(const T* p, int n) {
  constexpr int V = kVec<T>;
  if (n >= V) return load16(p);
  float v[V];
#pragma unroll
  for (int e = 0; e < V; ++e) v[e] = e < n ? to_f32(p[e]) : low();
  return pack16(v);
}
template <class T>
__device__ __forceinline__ void store_vec(T* p, int n, const float (&v)[kVec<T>]) {
  constexpr int V = kVec<T>;
  if (n >= V) {
    store16(p, pack16(v));
    return;
  }
#pragma unroll
  for (int e = 0; e < V; ++e)
    if (e < n) p[e] = T(v[e]);
}

// u / d for u < 2^31 as a product and a shift; d >= 1.
struct FastDiv {
  uint32_t mul, shift, div;
};
inline FastDiv fast_div(uint32_t d) {
  uint32_t s = 0;
  while ((uint64_t(1) << s) < d) ++s;
  const uint64_t m = ((uint64_t(1) << (31 + s)) + d - 1) / d;  // <= 2^32 - 1 for d >= 1
  return {uint32_t(m), 31 + s, d};
}
__device__ __forceinline__ uint32_t quotient(uint32_t u, const FastDiv& f) {
  return uint32_t((uint64_t(u) * f.mul) >> f.shift);
}

// HIP takes fewer than 2^32 threads a launch.  Calls fn(first block, grid) for the launches, one but for
// the largest sizes, that make up `blocks` blocks.
template <class Fn>
void for_launches(int64_t blocks, int threads, Fn fn) {
  const int64_t most = (int64_t(1) << 31) / threads;
  for (int64_t b = 0; b < blocks; b += most)
    fn(uint32_t(b), dim3(uint32_t(blocks - b < most ? blocks - b : most)));
}

// One microscaled table.
struct Mx4View {
  const uint8_t* codes;
  const uint8_t* scales;
  int64_t rows;
  int32_t dim;
};

hipError_t launch_mx4_quantize(const void* src, bool bf16, int64_t src_stride, int64_t rows,
                               int32_t dim, const int32_t* ids, int64_t num_ids, uint8_t* codes,
                               uint8_t* scales, int32_t* status, hipStream_t st);
hipError_t launch_mx4_dequantize(const Mx4View& w, void* dst, bool bf16, int64_t dst_stride,
                                 hipStream_t st);
// Tables as a TableDesc: w = codes, lo = scales.
hipError_t launch_mx4_forward(const TableDesc& d, int32_t B, const int32_t* I, const int32_t* O,
                              int64_t NS, void* Y, bool y_bf16, int32_t* status,
                              const PoolArgs& pool, hipStream_t st);

size_t mx4_matmul_workspace(int32_t m, int64_t n, int32_t k);
hipError_t launch_mx4_matmul(const void* x, bool x_bf16, int64_t x_stride, int32_t m,
                             const Mx4View& w, void* out, bool out_bf16, int64_t out_stride,
                             char* ws, hipStream_t st);
size_t mx4_matmul_grad_workspace(int32_t m, int64_t n, int32_t k);
hipError_t launch_mx4_matmul_grad(const void* dy, bool dy_bf16, int64_t dy_stride, int32_t m,
                                  const Mx4View& w, void* dx, bool dx_bf16, int64_t dx_stride,
                                  char* ws, hipStream_t st);

hipError_t launch_logits(const embbag_logits_t& a, int32_t* status, hipStream_t st);

size_t distill_workspace(int32_t rows, int32_t vocab, int32_t top);
hipError_t launch_distill(const embbag_distill_t& a, char* ws, int32_t* status, hipStream_t st);

}  // namespace embbag
