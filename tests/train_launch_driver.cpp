// The launches that the norm, the scores from 8-bit rows and the cross entropy make at the sizes the
// header allows.  The launch functions of HIP are defined here (an executable's symbols come before a
// library's), check what they are given and start nothing: the device pointers below are dummies that no
// kernel sees.  Exits 0 if every launch is one that HIP takes (fewer than 2^32 threads, at least one block)
// and no call makes more of them than its sizes need.
#include <hip/hip_runtime.h>

#include <cstdint>
#include <cstdio>

#include "embbag.h"

namespace {

int failures = 0;
uint64_t launches, most;  // of the call
dim3 next_grid, next_block;

void record(const dim3& g, const dim3& b) {
  const uint64_t threads = uint64_t(g.x) * b.x;
  ++launches;
  most = threads > most ? threads : most;
  if (g.x == 0 || g.y != 1 || g.z != 1 || b.x == 0 || b.x > 1024 || threads >= (uint64_t(1) << 32)) {
    std::fprintf(stderr, "a launch of %u x %u blocks of %u threads\n", g.x, g.y, b.x);
    ++failures;
  }
}

template <class T>
T* dev(uintptr_t k) {
  return reinterpret_cast<T*>((uintptr_t(1) << 44) + (k << 41));
}

void expect(const char* what, int status, uint64_t limit) {
  if (status != EMBBAG_OK || launches > limit) {
    std::fprintf(stderr, "%s: status %d, %llu launches, at most %llu expected\n", what, status,
                 (unsigned long long)launches, (unsigned long long)limit);
    ++failures;
  }
  launches = most = 0;
}

}  // namespace

extern "C" {
hipError_t hipLaunchKernel(const void*, dim3 g, dim3 b, void**, size_t, hipStream_t) {
  record(g, b);
  return hipSuccess;
}
hipError_t __hipPushCallConfiguration(dim3 g, dim3 b, size_t, hipStream_t) {
  next_grid = g, next_block = b;
  return hipSuccess;
}
hipError_t __hipPopCallConfiguration(dim3* g, dim3* b, size_t* shared, hipStream_t* st) {
  *g = next_grid, *b = next_block, *shared = 0, *st = nullptr;
  return hipSuccess;
}
hipError_t hipGetLastError(void) { return hipSuccess; }
hipError_t hipFuncSetAttribute(const void*, hipFuncAttribute, int) { return hipSuccess; }
}

int main() {
  const int64_t kRows = 2147483647;
  auto* codes = dev<uint8_t>(0);
  auto* scales = dev<uint8_t>(1);
  void* in = dev<void>(2);
  void* out = dev<void>(3);
  void* sum = dev<void>(4);
  void* ws = dev<void>(5);
  const size_t any = ~size_t(0);

  for (int64_t rows : {int64_t(1), int64_t(7), int64_t(1) << 20, kRows})
    for (int dim : {4, 128, 132, 260, 516, 1028, 2052, 4100, 8196, 16384})
      for (int type : {EMBBAG_F32, EMBBAG_BF16}) {
        embbag_rmsnorm_t n = {};
        n.rows = rows, n.dim = dim, n.eps = 1e-6f, n.x_type = n.residual_type = n.out_type = type;
        n.x = in, n.out = out, n.sum_out = sum, n.x_stride = n.out_stride = n.sum_stride = dim;
        n.codes = codes, n.scales = scales;
        expect("norm", embbag_rmsnorm(&n, nullptr), 1);
        embbag_rmsnorm_grad_t g = {};
        g.rows = rows, g.dim = dim, g.eps = 1e-6f, g.dy_type = g.h_type = type;
        g.dy = in, g.h = sum, g.dh = out, g.dy_stride = g.h_stride = g.dh_stride = dim, g.dweight = in;
        expect("norm's gradient", embbag_rmsnorm_grad(&g, ws, any, nullptr), 2);
        expect("8-bit rows read back", embbag_mx8_dequantize(codes, scales, rows, dim, out, type, dim, nullptr),
               1 + uint64_t(rows) * ((dim + 7) / 8) / (uint64_t(1) << 29));
      }

  for (int64_t n : {int64_t(1000), int64_t(1) << 30, kRows})
    for (int m : {1, 16, 17, 300})
      for (int k : {64, 16384})
        expect("scores from 8-bit rows",
               embbag_mx4_matmul_x8(codes, scales, m, codes, scales, n, k, out, EMBBAG_F32, n, ws, any, nullptr), 12);
  for (int n : {1, 1000, 131072})
    expect("scores of many 8-bit rows", embbag_mx4_matmul_x8(codes, scales, (1 << 23) - 1, codes, scales, n, 16384,
                                                             out, EMBBAG_BF16, n, ws, any, nullptr), 4);

  struct { int rows; int64_t vocab; int dim; } sizes[] = {
      {0, 1, 4}, {1, 1, 4}, {1, kRows, 4}, {1, kRows, 64}, {65, kRows, 128}, {1, kRows, 132}, {500, kRows, 16384},
      {1 << 20, 1, 4}, {1 << 20, 1 << 20, 64}, {1 << 20, 1 << 20, 128}, {1 << 20, 1 << 20, 132},
      {1 << 20, 1000, 16384}, {4096, 131072, 2048}, {4097, 1000, 300}, {512, kRows, 256}, {33, 32001, 128}};
  for (auto z : sizes)
    for (int tx : {EMBBAG_F32, EMBBAG_BF16})
      for (int tw : {EMBBAG_F32, EMBBAG_BF16})
        for (int grads = 0; grads < 4; ++grads) {
          embbag_xent_t a = {};
          a.rows = z.rows, a.dim = z.dim, a.vocab = z.vocab, a.x_type = tx, a.x = in, a.x_stride = z.dim;
          a.table_type = tw, a.table = out, a.table_stride = z.dim, a.labels = dev<int32_t>(6), a.scale = 1.f;
          a.loss = dev<float>(7), a.grad_x_stride = a.grad_table_stride = z.dim;
          if (grads & 1) a.grad_x = sum;
          if (grads & 2) a.grad_table = dev<void>(8);
          // A piece holds 256 columns at least.  Its launches: W packed, scores, their join; W packed, D, dx, dW
          // and its join.
          const uint64_t pieces = (uint64_t(z.vocab) + 255) / 256;
          expect("cross entropy", embbag_xent(&a, ws, any, nullptr, nullptr), 8 * pieces + 600);
        }
  if (failures == 0) std::printf("all launches fit\n");
  return failures != 0;
}
