// Scores of all rows of a 4-bit microscaled table: out = q(x) W^T.
#include "head.hpp"

namespace embbag {
namespace {

typedef int i8v __attribute__((ext_vector_type(8)));

// x rounded to the storage of the table, rows of whole 128-element groups: codes
// [m][groups * 64], scales as words (4 blocks) [groups][m].  Four lanes per block, as
// mx4_quantize.
template <class T>
__global__ __launch_bounds__(kBlock) void pack_x(const T* __restrict__ x, int64_t stride, int32_t m,
                                                 int32_t k, FastDiv groups,
                                                 uint8_t* __restrict__ codes,
                                                 uint8_t* __restrict__ scales) {
  const int64_t u = int64_t(blockIdx.x) * (kBlock / 4) + threadIdx.x / 4;
  const int part = threadIdx.x % 4;
  const int64_t g4 = u / 4;
  if (g4 >= int64_t(m) * groups.div) return;
  const uint32_t row = quotient(uint32_t(g4), groups);
  const int g = int(uint32_t(g4) - row * groups.div), j = int(u % 4);
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
  *reinterpret_cast<uint32_t*>(codes + (int64_t(row) * groups.div + g) * 64 + j * 16 + part * 4) = c;
  if (part == 0) scales[(int64_t(g) * m + row) * 4 + j] = uint8_t(byte);
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
  const uint8_t* xcr = xc + int64_t(xm) * groups * 64;
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

size_t mx4_matmul_workspace(int32_t m, int64_t n, int32_t k) {
  const size_t groups = size_t((k + 127) / 128);
  return align256(size_t(m) * groups * 64) + align256(size_t(m) * groups * 4);
}

hipError_t launch_mx4_matmul(const void* x, bool x_bf16, int64_t x_stride, int32_t m,
                             const Mx4View& w, void* out, bool out_bf16, int64_t out_stride,
                             char* ws, hipStream_t st) {
  if (m == 0 || w.rows == 0) return hipSuccess;
  const int groups = (w.dim + 127) / 128;
  uint8_t* xc = reinterpret_cast<uint8_t*>(ws);
  uint8_t* xs = xc + align256(size_t(m) * groups * 64);
  const int64_t units = int64_t(m) * groups * 4;
  const dim3 pgrid(unsigned((units + kBlock / 4 - 1) / (kBlock / 4)));
  const FastDiv f = fast_div(uint32_t(groups));
  if (x_bf16)
    hipLaunchKernelGGL(pack_x<__bf16>, pgrid, dim3(kBlock), 0, st, static_cast<const __bf16*>(x),
                       x_stride, m, w.dim, f, xc, xs);
  else
    hipLaunchKernelGGL(pack_x<float>, pgrid, dim3(kBlock), 0, st, static_cast<const float*>(x),
                       x_stride, m, w.dim, f, xc, xs);
  const uint32_t ntiles = uint32_t((w.rows + 63) / 64);
  const dim3 grid(ntiles * unsigned((m + 15) / 16));
  const uint32_t* xsw = reinterpret_cast<const uint32_t*>(xs);
  if (out_bf16)
    hipLaunchKernelGGL(scores_direct<__bf16>, grid, dim3(kBlock), 0, st, xc, xsw, w, m, groups,
                       ntiles, static_cast<__bf16*>(out), out_stride);
  else
    hipLaunchKernelGGL(scores_direct<float>, grid, dim3(kBlock), 0, st, xc, xsw, w, m, groups,
                       ntiles, static_cast<float*>(out), out_stride);
  return hipGetLastError();
}

}  // namespace embbag
