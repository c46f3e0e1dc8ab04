// The launches that the output head's entry points make at the sizes the header allows.  The launch
// functions of HIP are defined here (an executable's symbols come before a library's), count what they are
// given and start nothing: the device pointers below are dummies that no kernel sees.  Exits 0 if every
// launch is one that HIP takes (fewer than 2^32 threads, at least one block) and every call's blocks add up
// to what its sizes need.
#include <hip/hip_runtime.h>

#include <cstdint>
#include <cstdio>

#include "embbag.h"

namespace {

int failures = 0;
uint64_t blocks, launches, most;  // of the call
dim3 next_grid, next_block;

void record(const dim3& g, const dim3& b) {
  const uint64_t threads = uint64_t(g.x) * b.x;
  ++launches;
  blocks += g.x;
  most = threads > most ? threads : most;
  if (g.x == 0 || g.y != 1 || g.z != 1 || threads >= (uint64_t(1) << 32)) {
    std::fprintf(stderr, "a launch of %u x %u blocks of %u threads\n", g.x, g.y, b.x);
    ++failures;
  }
}

template <class T>
T* dev(uintptr_t k) {
  return reinterpret_cast<T*>((uintptr_t(1) << 44) + (k << 41));
}

uint64_t up(uint64_t a, uint64_t b) { return (a + b - 1) / b; }

void expect(const char* what, int status, uint64_t want) {
  std::printf("%-44s %10llu blocks in %llu launches, at most %llu threads\n", what,
              (unsigned long long)blocks, (unsigned long long)launches, (unsigned long long)most);
  if (status != EMBBAG_OK || (want != 0 && blocks != want)) {
    std::fprintf(stderr, "%s: status %d, %llu blocks, expected %llu\n", what, status,
                 (unsigned long long)blocks, (unsigned long long)want);
    ++failures;
  }
  blocks = launches = most = 0;
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
  auto* ids = dev<int32_t>(2);
  void* in = dev<void>(3);
  void* out = dev<void>(4);
  void* ws = dev<void>(5);
  const size_t any = ~size_t(0);

  // Four threads for each 32 elements.
  for (int type : {EMBBAG_F32, EMBBAG_BF16}) {
    struct { int64_t rows; int dim; } sizes[] = {{1, 4}, {kRows, 4}, {kRows, 32}, {kRows, 260}, {1 << 27, 256},
                                                 {(1 << 27) - 1, 256}, {1 << 30, 4}, {1 << 21, 16384},
                                                 {kRows, 16384}};
    for (auto s : sizes) {
      const uint64_t units = uint64_t(s.rows) * up(s.dim, 32);
      // (Launches of whole rows: a launch may end within a block.)
      const uint64_t least = up(units, 64);
      expect("quantize", embbag_mx4_quantize(in, type, s.dim, s.rows, s.dim, nullptr, 0, codes, scales,
                                             nullptr, nullptr), s.dim <= 256 && s.dim != 260 ? least : 0);
      expect("quantize, listed rows",
             embbag_mx4_quantize(in, type, s.dim, 1000, s.dim, ids, s.rows, codes, scales, nullptr, nullptr),
             s.dim <= 256 ? least : 0);
      expect("dequantize", embbag_mx4_dequantize(codes, scales, s.rows, s.dim, out, type, s.dim, nullptr),
             s.dim <= 256 ? least : 0);
    }
  }

  // Bags of the look-ups: up to 64 tables.
  for (int dim : {4, 64, 516, 1024}) {
    for (int32_t batch : {1, 1 << 20, 33554431}) {
      int64_t rows[64];
      uint8_t *c[64], *s[64];
      for (int t = 0; t < 64; ++t) rows[t] = 100, c[t] = codes, s[t] = scales;
      const embbag_mx4_tables_t tb = {64, dim, rows, c, s};
      for (int64_t n : {int64_t(0), int64_t(1) << 20, kRows})
        for (int mode : {EMBBAG_POOL_SUM, EMBBAG_POOL_MEAN})
          for (const float* a : {(const float*)nullptr, (const float*)dev<float>(6)})
            if (a == nullptr || mode == EMBBAG_POOL_SUM)
              expect("forward", embbag_mx4_forward(&tb, batch, ids, ids, n, a, mode, out, EMBBAG_F32,
                                                   nullptr, nullptr), 0);
    }
  }

  // Scores: one block for 64 rows of W up to 16 rows of x (after the packing of x where it is large).
  for (int64_t n : {int64_t(1000), int64_t(1) << 30, kRows}) {
    expect("scores of one row", embbag_mx4_matmul(in, EMBBAG_BF16, 64, 1, codes, scales, n, 64, out,
                                                  EMBBAG_BF16, n, ws, any, nullptr), up(n, 64));
    expect("scores of 16 wide rows",
           embbag_mx4_matmul(in, EMBBAG_F32, 16384, 16, codes, scales, n, 16384, out, EMBBAG_F32, n, ws, any,
                             nullptr), up(n, 64) + 16 * 128 * 4 / 64);
    expect("scores of 300 rows", embbag_mx4_matmul(in, EMBBAG_F32, 64, 300, codes, scales, n, 64, out,
                                                   EMBBAG_F32, n, ws, any, nullptr), 0);
    expect("gradient of 300 rows", embbag_mx4_matmul_grad(in, EMBBAG_F32, n, 300, codes, scales, n, 64, out,
                                                          EMBBAG_F32, 64, ws, any, nullptr), 0);
  }
  const int32_t kM = (1 << 23) - 1;
  for (int n : {1, 7, 8, 1000, 131072})
    for (int k : {4, 1000, 16384})
      for (int type : {EMBBAG_F32, EMBBAG_BF16}) {
        expect("scores of many rows", embbag_mx4_matmul(in, type, k, kM, codes, scales, n, k, out, type, n, ws,
                                                        any, nullptr), 0);
        expect("gradient of many rows", embbag_mx4_matmul_grad(in, type, n, kM, codes, scales, n, k, out, type,
                                                               k, ws, any, nullptr),
               n < 8 ? up(uint64_t(kM) * (k / 4), 256) : 0);
      }

  // Logits: a block for 4096 of a row; distillation: a block for a row.
  struct { int32_t rows, vocab; } sizes[] = {{1, 1}, {2147483647, 1}, {2147483647, 512}, {1 << 24, 8},
                                             {(1 << 24) - 1, 8}, {1 << 28, 4096}, {1 << 27, 4097}, {1 << 22, 8193},
                                             {1 << 22, 40000}, {1 << 23, 131072}, {512, 2147483647},
                                             {1, 2147483647}, {100, 200003}};
  for (int type : {EMBBAG_F32, EMBBAG_BF16})
    for (auto z : sizes) {
      embbag_logits_t l = {};
      l.rows = z.rows, l.vocab = z.vocab, l.type = type, l.logits = in, l.logits_stride = z.vocab;
      l.out = out, l.out_stride = z.vocab;
      const uint64_t want = uint64_t(z.rows) * up(z.vocab, 4096);
      expect("logits", embbag_logits_process(&l, nullptr, nullptr), want);
      l.seen = ids, l.seen_offsets = ids, l.num_seen = 5;
      expect("logits with seen tokens", embbag_logits_process(&l, nullptr, nullptr), want);
      l.bias_ids = ids, l.bias_offsets = ids, l.biases = dev<float>(6), l.num_biases = 5;
      expect("logits with both lists", embbag_logits_process(&l, nullptr, nullptr), want);
      embbag_distill_t d = {};
      d.rows = z.rows, d.vocab = z.vocab, d.type = type, d.logits = in, d.logits_stride = z.vocab;
      d.top = 8, d.ids = ids, d.teacher = in, d.temperature = 1.f, d.loss = dev<float>(6);
      d.grad = out, d.grad_stride = z.vocab;
      expect("distillation", embbag_distill(&d, ws, any, nullptr, nullptr), z.rows >= 128 ? z.rows : 0);
    }
  if (failures == 0) std::printf("all launches fit\n");
  return failures != 0;
}
