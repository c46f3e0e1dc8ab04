// Rows to and from 4-bit microscaled storage (OCP Microscaling Formats v1.0:
// FP4 E2M1 elements, an E8M0 scale for 32 of them).
//
// A block's scale is 2^e, e = floor(log2 of its largest magnitude) - 2, so that the
// largest element lies in [4, 8) before it is rounded (to 4 or 6).  Scaling by
// a power of two is exact: the conversion's rounding is the only one.
//
// Four lanes hold a block, 8 elements each: their maximum takes two exchanges, a
// lane's codes are one word, and a wavefront reads 16 blocks (2 KB of FP32) and
// writes 256 B of codes, all of it in whole lines where rows follow each other.  Bound by memory: 1M
// rows of 256, FP32, 218 us (1.16 GB, 5.3 TB/s), read back as BF16 131 us (648 MB, 4.9 TB/s).
#include "head.hpp"

namespace embbag {
namespace {

// Units (blocks) per launch, four threads each, of which a launch takes fewer than 2^32.  (The kernels
// number them in 31 bits.)
constexpr int64_t kMaxUnits = int64_t(1) << 29;

// Unit u of the launch is block (u + first) % nb of row row0 + (u + first) / nb, or of
// the row that the list names there.
template <class T>
__global__ __launch_bounds__(kBlock) void mx4_quantize_kernel(
    const T* __restrict__ src, int64_t stride, int64_t rows, int32_t dim, FastDiv nb,
    const int32_t* __restrict__ ids, int64_t row0, uint32_t units, uint8_t* __restrict__ codes,
    uint8_t* __restrict__ scales, int32_t* __restrict__ status) {
  const uint32_t u = blockIdx.x * uint32_t(kBlock / 4) + threadIdx.x / 4;
  const int part = threadIdx.x % 4;
  if (u >= units) return;  // whole groups of four lanes leave together
  const uint32_t q = quotient(u, nb);
  const int b = int(u - q * nb.div);
  int64_t row = row0 + q;
  if (ids != nullptr) {
    row = ids[row];
    if (row < 0 || row >= rows) {
      if (b == 0 && part == 0 && status != nullptr) atomicMin(status, EMBBAG_ERR_INDEX_RANGE);
      return;
    }
  }
  const int e0 = b * kMxBlock + part * 8;
  const T* p = src + row * stride + e0;
  const f4 zero = {0.f, 0.f, 0.f, 0.f};
  const f4 x0 = e0 < dim ? load4(p) : zero;
  const f4 x1 = e0 + 4 < dim ? load4(p + 4) : zero;
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
  *reinterpret_cast<uint32_t*>(codes + (row * nb.div + b) * 16 + part * 4) = c;
  // The last block's lanes write the padding of the row of scales as well.
  const int sb = mx4_scale_bytes(dim);
  uint8_t* s = scales + row * sb;
  if (part == 0) s[b] = uint8_t(byte);
  if (b == int(nb.div) - 1 && part > 0 && b + part < sb) s[b + part] = 0;
}

template <class T>
__global__ __launch_bounds__(kBlock) void mx4_dequantize_kernel(
    const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, int32_t dim, FastDiv nb,
    int64_t row0, uint32_t units, T* __restrict__ dst, int64_t stride) {
  const uint32_t u = blockIdx.x * uint32_t(kBlock / 4) + threadIdx.x / 4;
  const int part = threadIdx.x % 4;
  if (u >= units) return;
  const uint32_t q = quotient(u, nb);
  const int b = int(u - q * nb.div);
  const int64_t row = row0 + q;
  const int e0 = b * kMxBlock + part * 8;
  if (e0 >= dim) return;
  const uint32_t c =
      *reinterpret_cast<const uint32_t*>(codes + (row * nb.div + b) * 16 + part * 4);
  float v[8];
  mx4_values8(c, mx4_scale(scales[row * mx4_scale_bytes(dim) + b]), v);
  T* p = dst + row * stride + e0;
  store4(p, f4{v[0], v[1], v[2], v[3]});
  if (e0 + 4 < dim) store4(p + 4, f4{v[4], v[5], v[6], v[7]});
}

// Calls fn(first row, units) for launches of whole rows.
template <class Fn>
void for_rows(int64_t rows, int nb, Fn fn) {
  const int64_t step = kMaxUnits / nb;
  for (int64_t r = 0; r < rows; r += step) {
    const int64_t n = rows - r < step ? rows - r : step;
    fn(r, uint32_t(n * nb));
  }
}

dim3 grid_of(uint32_t units) { return dim3((units + kBlock / 4 - 1) / (kBlock / 4)); }

}  // namespace

hipError_t launch_mx4_quantize(const void* src, bool bf16, int64_t src_stride, int64_t rows,
                               int32_t dim, const int32_t* ids, int64_t num_ids, uint8_t* codes,
                               uint8_t* scales, int32_t* status, hipStream_t st) {
  const int nb = mx4_blocks(dim);
  const FastDiv f = fast_div(uint32_t(nb));
  for_rows(ids != nullptr ? num_ids : rows, nb, [&](int64_t r, uint32_t units) {
    if (bf16)
      hipLaunchKernelGGL(mx4_quantize_kernel<__bf16>, grid_of(units), dim3(kBlock), 0, st,
                         static_cast<const __bf16*>(src), src_stride, rows, dim, f, ids, r, units,
                         codes, scales, status);
    else
      hipLaunchKernelGGL(mx4_quantize_kernel<float>, grid_of(units), dim3(kBlock), 0, st,
                         static_cast<const float*>(src), src_stride, rows, dim, f, ids, r, units,
                         codes, scales, status);
  });
  return hipGetLastError();
}

hipError_t launch_mx4_dequantize(const Mx4View& w, void* dst, bool bf16, int64_t dst_stride,
                                 hipStream_t st) {
  const int nb = mx4_blocks(w.dim);
  const FastDiv f = fast_div(uint32_t(nb));
  for_rows(w.rows, nb, [&](int64_t r, uint32_t units) {
    if (bf16)
      hipLaunchKernelGGL(mx4_dequantize_kernel<__bf16>, grid_of(units), dim3(kBlock), 0, st,
                         w.codes, w.scales, w.dim, f, r, units, static_cast<__bf16*>(dst),
                         dst_stride);
    else
      hipLaunchKernelGGL(mx4_dequantize_kernel<float>, grid_of(units), dim3(kBlock), 0, st,
                         w.codes, w.scales, w.dim, f, r, units, static_cast<float*>(dst),
                         dst_stride);
  });
  return hipGetLastError();
}

}  // namespace embbag
