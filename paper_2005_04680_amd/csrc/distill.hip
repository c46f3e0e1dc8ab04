// Distillation from a teacher's top logits: loss and its gradient.
//
// Two kernels over slices of rows.  `distill_sums` leaves, per slice, the largest logit, the
// sum of exp2((x - largest) * c) (c = log2(e) / temperature) and the slice's
// part of sum_k p_k x[id_k]; `distill_grad` joins a row's parts in order and
// writes the slice's gradient.  The teacher's softmax is small: every block makes it again.
#include "head.hpp"

namespace embbag {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr int kSlice = 8192;  // logits per block

struct Part {
  float top, sum, cross;
};

struct DistillDev {
  embbag_distill_t a;
  uint32_t slices;
  Part* parts;
};

__device__ __forceinline__ float wave_max(float v) {
  for (int j = 1; j < kWave; j *= 2) v = fmaxf(v, __shfl_xor(v, j, kWave));
  return v;
}
__device__ __forceinline__ float wave_sum(float v) {
  for (int j = 1; j < kWave; j *= 2) v += __shfl_xor(v, j, kWave);
  return v;
}
// Over the block, to every thread; `s` has a float per wavefront.
__device__ __forceinline__ float block_max(float v, float* s) {
  v = wave_max(v);
  __syncthreads();
  if (lane_id() == 0) s[wave_id()] = v;
  __syncthreads();
  v = s[0];
  for (int w = 1; w < int(blockDim.x) / kWave; ++w) v = fmaxf(v, s[w]);
  return v;
}
__device__ __forceinline__ float block_sum(float v, float* s) {
  v = wave_sum(v);
  __syncthreads();
  if (lane_id() == 0) s[wave_id()] = v;
  __syncthreads();
  v = s[0];
  for (int w = 1; w < int(blockDim.x) / kWave; ++w) v += s[w];
  return v;
}

// The teacher's softmax of row r: ids and probabilities to LDS; returns whether the row
// counts (weight, entries), and sum p log p in *plogp.
__device__ __forceinline__ bool teacher_row(const embbag_distill_t& a, int r, int* ids, float* p,
                                            float* red, float* plogp, int* err) {
  const float w = a.row_weights != nullptr ? a.row_weights[r] : 1.f;
  const float inv_t = 1.f / a.temperature;
  const int64_t row = int64_t(r) * a.top;
  const float low = -__builtin_inff();
  float top = low, some = 0.f;
  for (int k = threadIdx.x; k < a.top; k += blockDim.x) {
    int id = a.ids[row + k];
    if (id >= a.vocab) {
      *err = EMBBAG_ERR_INDEX_RANGE;
      id = -1;
    }
    const float t = a.teacher_type == EMBBAG_BF16
                        ? to_f32(static_cast<const __bf16*>(a.teacher)[row + k])
                        : static_cast<const float*>(a.teacher)[row + k];
    ids[k] = id;
    p[k] = id >= 0 ? t * inv_t : low;
    top = id >= 0 ? fmaxf(top, t * inv_t) : top;
    if (id >= 0 && t != low) some = 1.f;  // (a NaN as well)
  }
  top = block_max(top, red);
  const bool live = w != 0.f && block_max(some, red) != 0.f;
  const float ref = top == low ? 0.f : top;
  float sum = 0.f;
  for (int k = threadIdx.x; k < a.top; k += blockDim.x)
    sum += ids[k] >= 0 ? __builtin_exp2f((p[k] - ref) * kLog2e) : 0.f;
  sum = block_sum(sum, red);
  const float inv = 1.f / sum, log_sum = __builtin_logf(sum);
  float pl = 0.f;
  for (int k = threadIdx.x; k < a.top; k += blockDim.x) {
    const float z = p[k] - ref;
    const float q = ids[k] >= 0 ? __builtin_exp2f(z * kLog2e) * inv : 0.f;
    p[k] = q;
    if (q != 0.f) pl += q * (z - log_sum);
  }
  *plogp = block_sum(pl, red);
  return live;
}

template <class T>
__global__ __launch_bounds__(kBlock) void distill_sums(DistillDev dv, int32_t* __restrict__ status) {
  __shared__ int ids[kMaxTeacher];
  __shared__ float p[kMaxTeacher];
  __shared__ float red[kWavesPerBlock];
  const embbag_distill_t& a = dv.a;
  const int r = int(blockIdx.x / dv.slices);
  const uint32_t sl = blockIdx.x - uint32_t(r) * dv.slices;
  const int base = int(sl) * kSlice;
  const int len = min(kSlice, a.vocab - base);
  const T* x = static_cast<const T*>(a.logits) + int64_t(r) * a.logits_stride + base;
  int err = 0;
  float plogp;
  const bool live = teacher_row(a, r, ids, p, red, &plogp, &err);
  if (err != 0 && status != nullptr) atomicMin(status, err);
  if (!live) return;
  const float c = kLog2e / a.temperature;
  const float low = -__builtin_inff();
  float top = low;
  for (int i = threadIdx.x; i < len; i += kBlock) top = fmaxf(top, to_f32(x[i]));
  top = block_max(top, red);
  const float ref = top == low ? 0.f : top;
  float sum = 0.f;
  for (int i = threadIdx.x; i < len; i += kBlock)
    sum += __builtin_exp2f((to_f32(x[i]) - ref) * c);
  sum = block_sum(sum, red);
  float cross = 0.f;
  for (int k = threadIdx.x; k < a.top; k += kBlock) {
    const int at = ids[k] - base;
    if (ids[k] >= 0 && uint32_t(at) < uint32_t(len) && p[k] != 0.f) cross += p[k] * to_f32(x[at]);
  }
  cross = block_sum(cross, red);
  if (threadIdx.x == 0) dv.parts[int64_t(r) * dv.slices + sl] = {top, sum, cross};
}

template <class T>
__global__ __launch_bounds__(kBlock) void distill_grad(DistillDev dv) {
  __shared__ int ids[kMaxTeacher];
  __shared__ float p[kMaxTeacher];
  __shared__ float red[kWavesPerBlock];
  const embbag_distill_t& a = dv.a;
  const int r = int(blockIdx.x / dv.slices);
  const uint32_t sl = blockIdx.x - uint32_t(r) * dv.slices;
  const int base = int(sl) * kSlice;
  const int len = min(kSlice, a.vocab - base);
  const T* x = static_cast<const T*>(a.logits) + int64_t(r) * a.logits_stride + base;
  T* g = a.grad != nullptr ? static_cast<T*>(a.grad) + int64_t(r) * a.grad_stride + base : nullptr;
  int err = 0;
  float plogp;
  bool live = teacher_row(a, r, ids, p, red, &plogp, &err);
  float top = -__builtin_inff(), sum = 0.f, cross = 0.f;
  const float c = kLog2e / a.temperature;
  if (live) {
    const Part* q = dv.parts + int64_t(r) * dv.slices;
    for (uint32_t i = 0; i < dv.slices; ++i) top = fmaxf(top, q[i].top);
    const float ref = top == -__builtin_inff() ? 0.f : top;
    for (uint32_t i = 0; i < dv.slices; ++i) {
      const float m = q[i].top == -__builtin_inff() ? 0.f : q[i].top;
      sum += q[i].sum == 0.f ? 0.f : q[i].sum * __builtin_exp2f((m - ref) * c);
      cross += q[i].cross;
    }
    live = !(sum == 0.f);
    top = ref;
  }
  const float w = live ? (a.row_weights != nullptr ? a.row_weights[r] : 1.f) : 0.f;
  const float T1 = a.temperature;
  if (sl == 0 && threadIdx.x == 0) {
    const float lse = top / T1 + __builtin_logf(sum);
    a.loss[r] = live ? w * T1 * T1 * (plogp - cross / T1 + lse) : 0.f;
  }
  if (g == nullptr) return;
  if (!live) {
    for (int i = threadIdx.x; i < len; i += kBlock) g[i] = T(0.f);
    return;
  }
  const float f = w * T1, inv = 1.f / sum;
  // An entry's logit is read before the slice is written: g may be x.  The first
  // entry of an id subtracts the probabilities of all its entries, in order.
  float fix[kMaxTeacher / kBlock];
#pragma unroll
  for (int j = 0; j < kMaxTeacher / kBlock; ++j) {
    const int k = j * kBlock + int(threadIdx.x);
    fix[j] = 0.f;
    if (k < a.top && ids[k] >= 0 && uint32_t(ids[k] - base) < uint32_t(len)) {
      bool first = true;
      float pk = 0.f;
      for (int i = 0; i < a.top; ++i) {
        if (ids[i] != ids[k]) continue;
        first = first && i >= k;
        pk += p[i];
      }
      fix[j] = f * (__builtin_exp2f((to_f32(x[ids[k] - base]) - top) * c) * inv - pk);
      if (!first) fix[j] = __builtin_nanf("");
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < len; i += kBlock)
    g[i] = T(f * (__builtin_exp2f((to_f32(x[i]) - top) * c) * inv));
  __syncthreads();
#pragma unroll
  for (int j = 0; j < kMaxTeacher / kBlock; ++j) {
    const int k = j * kBlock + int(threadIdx.x);
    if (k < a.top && ids[k] >= 0 && uint32_t(ids[k] - base) < uint32_t(len)) {
      bool first = true;
      for (int i = 0; i < k; ++i) first = first && ids[i] != ids[k];
      if (first) g[ids[k] - base] = T(fix[j]);
    }
  }
}

uint32_t slices_of(int32_t vocab) { return uint32_t((int64_t(vocab) + kSlice - 1) / kSlice); }

}  // namespace

size_t distill_workspace(int32_t rows, int32_t vocab, int32_t top) {
  const size_t n = size_t(rows) * slices_of(vocab) * sizeof(Part);
  return (n + 255) / 256 * 256 + 256;
}

hipError_t launch_distill(const embbag_distill_t& a, char* ws, int32_t* status, hipStream_t st) {
  if (a.rows == 0) return hipSuccess;
  DistillDev dv;
  dv.a = a;
  dv.slices = slices_of(a.vocab);
  dv.parts = reinterpret_cast<Part*>(ws);
  const dim3 grid(dv.slices * uint32_t(a.rows));
  if (a.type == EMBBAG_BF16) {
    hipLaunchKernelGGL(distill_sums<__bf16>, grid, dim3(kBlock), 0, st, dv, status);
    hipLaunchKernelGGL(distill_grad<__bf16>, grid, dim3(kBlock), 0, st, dv);
  } else {
    hipLaunchKernelGGL(distill_sums<float>, grid, dim3(kBlock), 0, st, dv, status);
    hipLaunchKernelGGL(distill_grad<float>, grid, dim3(kBlock), 0, st, dv);
  }
  return hipGetLastError();
}

}  // namespace embbag
