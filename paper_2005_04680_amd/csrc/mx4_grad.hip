// Gradient of the scores with respect to x: dx = dy W, W a 4-bit microscaled
// table.
#include "head.hpp"

namespace embbag {
namespace {

constexpr int kRowsPerBlock = 8;  // rows of dy
constexpr int kStep = 64;         // rows of W whose dy a block holds at a time

// A thread holds 8 columns of 8 rows of dx.
template <class TY, class TX>
__global__ __launch_bounds__(kWave) void scores_grad(const TY* __restrict__ dy, int64_t ldy,
                                                     int32_t m, Mx4View w, uint32_t ktiles,
                                                     TX* __restrict__ dx, int64_t ldx) {
  __shared__ float y[kRowsPerBlock][kStep];
  const int nb = mx4_blocks(w.dim), sb = mx4_scale_bytes(w.dim);
  const uint32_t kt = blockIdx.x % ktiles, mt = blockIdx.x / ktiles;
  const int e0 = (int(kt) * kWave + int(threadIdx.x)) * 8;
  const int m0 = int(mt) * kRowsPerBlock;
  const bool in = e0 < w.dim;
  float acc[kRowsPerBlock][8] = {};
  for (int64_t n0 = 0; n0 < w.rows; n0 += kStep) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kRowsPerBlock; ++i) {
      const int64_t n = n0 + threadIdx.x;
      y[i][threadIdx.x] =
          m0 + i < m && n < w.rows ? to_f32(dy[int64_t(m0 + i) * ldy + n]) : 0.f;
    }
    __syncthreads();
    if (!in) continue;
    const int steps = int(min(int64_t(kStep), w.rows - n0));
    for (int j = 0; j < steps; ++j) {
      const int64_t row = n0 + j;
      const uint32_t c = *reinterpret_cast<const uint32_t*>(w.codes + row * nb * 16 + e0 / 2);
      float v[8];
      mx4_values8(c, mx4_scale(w.scales[row * sb + e0 / kMxBlock]), v);
#pragma unroll
      for (int i = 0; i < kRowsPerBlock; ++i) {
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[i][e] = fmaf(y[i][j], v[e], acc[i][e]);
      }
    }
  }
  if (!in) return;
#pragma unroll
  for (int i = 0; i < kRowsPerBlock; ++i) {
    if (m0 + i >= m) break;
    TX* p = dx + int64_t(m0 + i) * ldx + e0;
    store4(p, f4{acc[i][0], acc[i][1], acc[i][2], acc[i][3]});
    if (e0 + 4 < w.dim) store4(p + 4, f4{acc[i][4], acc[i][5], acc[i][6], acc[i][7]});
  }
}

template <class TY, class TX>
void launch_simple(const void* dy, int64_t ldy, int32_t m, const Mx4View& w, void* dx, int64_t ldx,
                   hipStream_t st) {
  const uint32_t ktiles = uint32_t((w.dim + kWave * 8 - 1) / (kWave * 8));
  const dim3 grid(ktiles * unsigned((m + kRowsPerBlock - 1) / kRowsPerBlock));
  hipLaunchKernelGGL((scores_grad<TY, TX>), grid, dim3(kWave), 0, st, static_cast<const TY*>(dy),
                     ldy, m, w, ktiles, static_cast<TX*>(dx), ldx);
}

}  // namespace

size_t mx4_matmul_grad_workspace(int32_t m, int64_t n, int32_t k) { return 256; }

hipError_t launch_mx4_matmul_grad(const void* dy, bool dy_bf16, int64_t dy_stride, int32_t m,
                                  const Mx4View& w, void* dx, bool dx_bf16, int64_t dx_stride,
                                  char* ws, hipStream_t st) {
  if (m == 0) return hipSuccess;
  if (dy_bf16 && dx_bf16)
    launch_simple<__bf16, __bf16>(dy, dy_stride, m, w, dx, dx_stride, st);
  else if (dy_bf16)
    launch_simple<__bf16, float>(dy, dy_stride, m, w, dx, dx_stride, st);
  else if (dx_bf16)
    launch_simple<float, __bf16>(dy, dy_stride, m, w, dx, dx_stride, st);
  else
    launch_simple<float, float>(dy, dy_stride, m, w, dx, dx_stride, st);
  return hipGetLastError();
}

}  // namespace embbag
