// Distillation from a teacher's top logits: loss and its gradient.
//
// With many rows a block takes a whole one and keeps it in registers (up to 256 KB: 16 vectors
// of 16 bytes for each of 1024 threads): the row is read once for its largest logit, the
// sum of the exponentials and the gradient, which is written once.  What does not fit is read
// again, from the caches if they still hold it.  With few rows a row is split into slices, one block
// each: a first kernel leaves every slice's largest logit and sum, a second joins a row's parts
// in order and writes the gradient.
//
// Bound by memory: 4096 x 131072 BF16 458 us, 2.04 GB (a twentieth of the rows is left out), 4.5 TB/s;
// few rows by the chain of load, sum, store: 33 x 32001 FP32 9.3 us.
//
// exp(x) is taken as 2^((x - largest) * log2(e) / temperature), and the loss sums p (x - largest): an
// offset that a row's logits share costs no digits.  The teacher's entries are few: one
// wavefront makes their softmax while the row is on its way.  The entry that names an id
// first subtracts all its entries' probabilities, after the row has been written: no atomics on
// sums.  A table in LDS shows whether any id comes twice; only then are the entries compared with
// each other (64 x 50000 BF16 with 1000 entries: 73 us with, 21 without).
#include "head.hpp"

namespace embbag {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kRowThreads = 1024;
constexpr int kPer = kMaxTeacher / kBlock;  // entries per thread of the smallest block

__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }

// Of a slice: the largest logit, the sum of the exponentials and the teacher's probabilities times the
// logits, both relative to that logit, and those probabilities' sum.
struct Part {
  float top, sum, cross, mass;
};

struct DistillDev {
  embbag_distill_t a;
  int32_t slice;    // elements per slice
  uint32_t slices;  // per row
  Part* parts;
  uint32_t first;   // row that the launch begins with, where a block takes a whole one
};

__device__ __forceinline__ float wave_max(float v) {
  for (int j = 1; j < kWave; j *= 2) v = fmaxf(v, __shfl_xor(v, j, kWave));
  return v;
}
__device__ __forceinline__ float wave_sum(float v) {
  for (int j = 1; j < kWave; j *= 2) v += __shfl_xor(v, j, kWave);
  return v;
}

// A row's teacher, in LDS.
constexpr int kIdSlots = 2 * kMaxTeacher;
struct Teacher {
  int ids[kMaxTeacher];
  float p[kMaxTeacher];
  int slots[kIdSlots];  // ids, -1 where free
  int repeated;
  float plogp;
  int live;
  float red[4][kRowThreads / kWave];
};

// The softmax of row r's entries, by one wavefront: ids (-1: none), probabilities, the sum of
// p log p, and whether the row has any entry that is not -infinity.  The temperature divides the distances
// to the largest entry: divided first, entries of 20 at 1e-4 would be off by 0.008 in the exponent.
__device__ __forceinline__ void teacher_row(const embbag_distill_t& a, int r, Teacher& t,
                                            int32_t* status) {
  const float inv_t = 1.f / a.temperature;
  const int64_t row = int64_t(r) * a.top;
  float top = low();
  bool some = false, bad = false;
  for (int k = lane_id(); k < a.top; k += kWave) {
    int id = a.ids[row + k];
    bad = bad || id >= a.vocab;
    if (id >= a.vocab) id = -1;
    const float x = a.teacher_type == EMBBAG_BF16
                        ? to_f32(static_cast<const __bf16*>(a.teacher)[row + k])
                        : static_cast<const float*>(a.teacher)[row + k];
    t.ids[k] = id;
    t.p[k] = id >= 0 ? x : low();
    if (id >= 0) top = fmaxf(top, x);
    some = some || (id >= 0 && x != low());  // (a NaN as well)
  }
  if (bad && status != nullptr) atomicMin(status, EMBBAG_ERR_INDEX_RANGE);
  top = wave_max(top);
  const float ref = top == low() ? 0.f : top;
  float sum = 0.f;
  for (int k = lane_id(); k < a.top; k += kWave)
    sum += t.ids[k] >= 0 ? exp2_of((t.p[k] - ref) * inv_t * kLog2e) : 0.f;
  sum = wave_sum(sum);
  const float inv = 1.f / sum, log_sum = __builtin_logf(sum);
  float pl = 0.f;
  for (int k = lane_id(); k < a.top; k += kWave) {
    const float z = (t.p[k] - ref) * inv_t;
    const float q = t.ids[k] >= 0 ? exp2_of(z * kLog2e) * inv : 0.f;
    t.p[k] = q;
    if (q != 0.f) pl += q * (z - log_sum);
  }
  pl = wave_sum(pl);
  const bool any = __builtin_amdgcn_ballot_w64(some) != 0ull;
  if (lane_id() == 0) {
    t.plogp = pl;
    t.live = any;
  }
}

// Before the teacher's barrier, and after it: enters the ids into the slots.
__device__ __forceinline__ void clear_slots(Teacher& t) {
  for (int i = threadIdx.x; i < kIdSlots; i += blockDim.x) t.slots[i] = -1;
  if (threadIdx.x == 0) t.repeated = 0;
}
__device__ __forceinline__ void enter_ids(Teacher& t, int top) {
  for (int k = threadIdx.x; k < top; k += blockDim.x) {
    const int id = t.ids[k];
    if (id < 0) continue;
    uint32_t h = uint32_t(id) * 2654435769u >> 21;
    static_assert(kIdSlots == 1 << 11, "the hash gives a slot");
    for (;; h = (h + 1) % kIdSlots) {  // at most half of the slots are taken
      const int was = atomicCAS(&t.slots[h], -1, id);
      if (was == id) t.repeated = 1;
      if (was == -1 || was == id) break;
    }
  }
}

// Entry k of the row: whether it is its id's first, and the probabilities of all the id's
// entries, added in order.
__device__ __forceinline__ bool first_entry(const Teacher& t, int top, int k, float* p) {
  *p = t.p[k];
  if (t.repeated == 0) return true;
  const int id = t.ids[k];
  bool first = true;
  float s = 0.f;
  for (int i = 0; i < top; ++i) {
    if (t.ids[i] != id) continue;
    first = first && i >= k;
    s += t.p[i];
  }
  *p = s;
  return first;
}

// Zeros to a row (or slice) of n elements.
template <class T>
__device__ __forceinline__ void zero_row(T* g, int n) {
  constexpr int V = kVec<T>;
  const float z[V] = {};
  for (int64_t i = int64_t(threadIdx.x) * V; i < n; i += int64_t(blockDim.x) * V)
    store_vec(g + i, int(min(int64_t(n) - i, int64_t(V))), z);
}

// Adds the exponentials of a vector to a running (top, sum).
template <int V>
__device__ __forceinline__ void add_online(const float (&v)[V], float c, float* top, float* sum) {
  float t = *top;
#pragma unroll
  for (int e = 0; e < V; ++e) t = fmaxf(t, v[e]);
  const float ref = t == low() ? 0.f : t;
  float s = *sum == 0.f ? 0.f : *sum * exp2_of((*top - ref) * c);
#pragma unroll
  for (int e = 0; e < V; ++e) s += exp2_of((v[e] - ref) * c);
  *top = t;
  *sum = s;
}

// One block per row; its first NV * THREADS vectors stay in registers.
template <class T, int THREADS, int NV>
__global__ __launch_bounds__(THREADS) void distill_row(DistillDev dv, int32_t* __restrict__ status) {
  constexpr int V = kVec<T>;
  constexpr int WAVES = THREADS / kWave;
  constexpr int PER = kMaxTeacher / THREADS;
  __shared__ Teacher t;
  const embbag_distill_t& a = dv.a;
  const int r = int(dv.first + blockIdx.x);
  const T* x = static_cast<const T*>(a.logits) + int64_t(r) * a.logits_stride;
  T* g = a.grad != nullptr ? static_cast<T*>(a.grad) + int64_t(r) * a.grad_stride : nullptr;
  const float w = a.row_weights != nullptr ? a.row_weights[r] : 1.f;
  if (w == 0.f) {
    // (A bad id of a row that is left out is an error all the same, as it is in the slices.)
    bool bad = false;
    for (int k = threadIdx.x; k < a.top; k += THREADS)
      bad = bad || a.ids[int64_t(r) * a.top + k] >= a.vocab;
    if (bad && status != nullptr) atomicMin(status, EMBBAG_ERR_INDEX_RANGE);
    if (threadIdx.x == 0) a.loss[r] = 0.f;
    if (g != nullptr) zero_row(g, a.vocab);
    return;
  }
  const float c = kLog2e / a.temperature;
  const int tid = threadIdx.x;
  auto left = [&](int i) { return a.vocab - (i * THREADS + tid) * V; };

  u4 v[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i)
    if (left(i) > 0) v[i] = load_vec(x + (i * THREADS + tid) * V, left(i));
  clear_slots(t);
  if (wave_id() == 0) teacher_row(a, r, t, status);
  float top = low();
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    if (left(i) > 0) {
      float f[V];
      unpack16(v[i], f);
#pragma unroll
      for (int e = 0; e < V; ++e) top = fmaxf(top, f[e]);
    }
  }
  // What the registers do not hold, with its sum at the same time.
  float rest_top = low(), rest = 0.f;
  for (int64_t i = (int64_t(NV) * THREADS + tid) * V; i < a.vocab; i += THREADS * V) {
    float f[V];
    unpack16(load_vec(x + i, int(min(a.vocab - i, int64_t(V)))), f);
    add_online<V>(f, c, &rest_top, &rest);
  }
  top = wave_max(fmaxf(top, rest_top));
  if (lane_id() == 0) t.red[0][wave_id()] = top;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < WAVES; ++i) top = fmaxf(top, t.red[0][i]);
  const float ref = top == low() ? 0.f : top;

  float sum = rest == 0.f ? 0.f : rest * exp2_of(((rest_top == low() ? 0.f : rest_top) - ref) * c);
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    if (left(i) > 0) {
      float f[V];
      unpack16(v[i], f);
#pragma unroll
      for (int e = 0; e < V; ++e) sum += exp2_of((f[e] - ref) * c);
    }
  }
  enter_ids(t, a.top);
  // The entries' logits, before the row is written (g may be x).
  float cross = 0.f, xk[PER];
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const int k = j * THREADS + tid;
    xk[j] = k < a.top && t.ids[k] >= 0 ? to_f32(x[t.ids[k]]) : 0.f;
    if (k < a.top && t.p[k] != 0.f) cross += t.p[k] * (xk[j] - ref);
  }
  sum = wave_sum(sum);
  cross = wave_sum(cross);
  if (lane_id() == 0) t.red[1][wave_id()] = sum, t.red[2][wave_id()] = cross;
  __syncthreads();
  sum = cross = 0.f;
#pragma unroll
  for (int i = 0; i < WAVES; ++i) sum += t.red[1][i], cross += t.red[2][i];
  const bool live = t.live && !(sum == 0.f);
  if (tid == 0) {
    const float T1 = a.temperature;
    a.loss[r] = live ? w * T1 * T1 * (t.plogp - cross / T1 + __builtin_logf(sum)) : 0.f;
  }
  if (g == nullptr) return;
  if (!live) {
    zero_row(g, a.vocab);
    return;
  }
  const float f = w * a.temperature, scale = f / sum;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    if (left(i) > 0) {
      float q[V];
      unpack16(v[i], q);
#pragma unroll
      for (int e = 0; e < V; ++e) q[e] = scale * exp2_of((q[e] - ref) * c);
      store_vec(g + (i * THREADS + tid) * V, left(i), q);
    }
  }
  for (int64_t i = (int64_t(NV) * THREADS + tid) * V; i < a.vocab; i += THREADS * V) {
    const int n = int(min(a.vocab - i, int64_t(V)));
    float q[V];
    unpack16(load_vec(x + i, n), q);
#pragma unroll
    for (int e = 0; e < V; ++e) q[e] = scale * exp2_of((q[e] - ref) * c);
    store_vec(g + i, n, q);
  }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const int k = j * THREADS + tid;
    float p;
    if (k < a.top && t.ids[k] >= 0 && first_entry(t, a.top, k, &p))
      g[t.ids[k]] = T(scale * exp2_of((xk[j] - ref) * c) - f * p);
  }
}

// Sums over the block, to every thread.
__device__ __forceinline__ float block_sum(float v, float* red) {
  v = wave_sum(v);
  if (lane_id() == 0) red[wave_id()] = v;
  __syncthreads();
  v = red[0];
#pragma unroll
  for (int i = 1; i < kWavesPerBlock; ++i) v += red[i];
  return v;
}

// Few rows: the parts of a slice.
template <class T>
__global__ __launch_bounds__(kBlock) void distill_sums(DistillDev dv, int32_t* __restrict__ status) {
  constexpr int V = kVec<T>;
  __shared__ Teacher t;
  const embbag_distill_t& a = dv.a;
  const int r = int(blockIdx.x / dv.slices);
  const uint32_t sl = blockIdx.x - uint32_t(r) * dv.slices;
  const int64_t base = int64_t(sl) * dv.slice;
  const int len = int(min(int64_t(dv.slice), a.vocab - base));
  const T* x = static_cast<const T*>(a.logits) + int64_t(r) * a.logits_stride + base;
  if (wave_id() == 0) teacher_row(a, r, t, sl == 0 ? status : nullptr);
  const float c = kLog2e / a.temperature;
  float top = low(), sum = 0.f;
  for (int i = threadIdx.x * V; i < len; i += kBlock * V) {
    float f[V];
    unpack16(load_vec(x + i, len - i), f);
    add_online<V>(f, c, &top, &sum);
  }
  const float mine = top;
  top = wave_max(top);
  if (lane_id() == 0) t.red[0][wave_id()] = top;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kWavesPerBlock; ++i) top = fmaxf(top, t.red[0][i]);
  const float ref = top == low() ? 0.f : top;
  sum = sum == 0.f ? 0.f : sum * exp2_of(((mine == low() ? 0.f : mine) - ref) * c);
  float cross = 0.f, mass = 0.f;
  for (int k = threadIdx.x; k < a.top; k += kBlock) {
    const int64_t at = t.ids[k] - base;
    if (t.ids[k] >= 0 && at >= 0 && at < len && t.p[k] != 0.f) {
      cross += t.p[k] * (to_f32(x[at]) - ref);
      mass += t.p[k];
    }
  }
  sum = block_sum(sum, t.red[1]);
  cross = block_sum(cross, t.red[2]);
  mass = block_sum(mass, t.red[3]);
  if (threadIdx.x == 0) dv.parts[int64_t(r) * dv.slices + sl] = {top, sum, cross, mass};
}

// Few rows: joins a row's parts, and the gradient of a slice.
template <class T>
__global__ __launch_bounds__(kBlock) void distill_grad(DistillDev dv) {
  constexpr int V = kVec<T>;
  __shared__ Teacher t;
  const embbag_distill_t& a = dv.a;
  const int r = int(blockIdx.x / dv.slices);
  const uint32_t sl = blockIdx.x - uint32_t(r) * dv.slices;
  const int64_t base = int64_t(sl) * dv.slice;
  const int len = int(min(int64_t(dv.slice), a.vocab - base));
  const T* x = static_cast<const T*>(a.logits) + int64_t(r) * a.logits_stride + base;
  T* g = a.grad != nullptr ? static_cast<T*>(a.grad) + int64_t(r) * a.grad_stride + base : nullptr;
  clear_slots(t);
  if (wave_id() == 0) teacher_row(a, r, t, nullptr);
  const float w = a.row_weights != nullptr ? a.row_weights[r] : 1.f;
  const float c = kLog2e / a.temperature;
  const Part* q = dv.parts + int64_t(r) * dv.slices;
  float top = low(), sum = 0.f, cross = 0.f;
  for (uint32_t i = 0; i < dv.slices; ++i) top = fmaxf(top, q[i].top);
  const float ref = top == low() ? 0.f : top;
  for (uint32_t i = 0; i < dv.slices; ++i) {
    const float m = q[i].top == low() ? 0.f : q[i].top;
    sum += q[i].sum == 0.f ? 0.f : q[i].sum * exp2_of((m - ref) * c);
    // (A slice without entries adds nothing, however far its largest logit is.)
    if (q[i].mass != 0.f) cross += q[i].cross + (m - ref) * q[i].mass;
  }
  __syncthreads();
  const bool live = w != 0.f && t.live && !(sum == 0.f);
  if (sl == 0 && threadIdx.x == 0) {
    const float T1 = a.temperature;
    a.loss[r] = live ? w * T1 * T1 * (t.plogp - cross / T1 + __builtin_logf(sum)) : 0.f;
  }
  if (g == nullptr) return;
  if (!live) {
    zero_row(g, len);
    return;
  }
  const float f = w * a.temperature, scale = f / sum;
  enter_ids(t, a.top);
  float xk[kPer];
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    const int k = j * kBlock + int(threadIdx.x);
    const int64_t at = k < a.top ? t.ids[k] - base : -1;
    xk[j] = k < a.top && t.ids[k] >= 0 && at >= 0 && at < len ? to_f32(x[at]) : 0.f;
  }
  __syncthreads();
  for (int i = threadIdx.x * V; i < len; i += kBlock * V) {
    float v[V];
    unpack16(load_vec(x + i, len - i), v);
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = scale * exp2_of((v[e] - ref) * c);
    store_vec(g + i, len - i, v);
  }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    const int k = j * kBlock + int(threadIdx.x);
    if (k >= a.top) break;
    const int64_t at = t.ids[k] - base;
    float p;
    if (t.ids[k] >= 0 && at >= 0 && at < len && first_entry(t, a.top, k, &p))
      g[at] = T(scale * exp2_of((xk[j] - ref) * c) - f * p);
  }
}

// Calls of this many rows, and shorter rows (128 KB), get a block per row.  Measured, us, rows /
// slices: 33 x 32001 FP32 10.8 / 13.2, 1 x 32001 10.8 / 12.9; of 131072 BF16 one row 23.2 / 16.1,
// 64 25.9 / 20.7, 128 29.1 / 27.6, 256 34.9 / 42.3; of 200003 FP32 64 51.2 / 35.0, 128 56.6 /
// 56.0, 512 239 / 266.  Slices of 16384 instead of 4096 at the least: one row of 131072 17.1.
constexpr int kWholeRows = 128;
constexpr int kWholeVecs = kRowThreads * 8;
constexpr int kLeastSlice = 4096;

// Slices of the rows of a call with few of them: about four blocks per compute unit.
int32_t slice_of(int32_t rows, int32_t vocab) {
  const int64_t want = (int64_t(kNumCu) * 4 + rows - 1) / (rows > 0 ? rows : 1);
  int64_t s = (int64_t(vocab) + want - 1) / want;
  s = (s + 7) / 8 * 8;
  return int32_t(s < kLeastSlice ? kLeastSlice : s);
}

template <class T, int THREADS, int NV>
void launch_row(DistillDev& dv, int32_t* status, hipStream_t st) {
  for_launches(dv.a.rows, THREADS, [&](uint32_t first, dim3 grid) {
    dv.first = first;
    hipLaunchKernelGGL((distill_row<T, THREADS, NV>), grid, dim3(THREADS), 0, st, dv, status);
  });
}

template <class T>
void launch_type(DistillDev& dv, int32_t* status, hipStream_t st) {
  const embbag_distill_t& a = dv.a;
  const int64_t vecs = (int64_t(a.vocab) + kVec<T> - 1) / kVec<T>;
  if (a.rows >= kWholeRows || vecs <= kWholeVecs) {
    if (vecs <= kBlock * 4)
      launch_row<T, kBlock, 4>(dv, status, st);
    else if (vecs <= kRowThreads * 4)
      launch_row<T, kRowThreads, 4>(dv, status, st);
    else if (vecs <= kRowThreads * 8)
      launch_row<T, kRowThreads, 8>(dv, status, st);
    else
      launch_row<T, kRowThreads, 16>(dv, status, st);
    return;
  }
  const dim3 grid(dv.slices * uint32_t(a.rows));
  hipLaunchKernelGGL(distill_sums<T>, grid, dim3(kBlock), 0, st, dv, status);
  hipLaunchKernelGGL(distill_grad<T>, grid, dim3(kBlock), 0, st, dv);
}

uint32_t slices_of(int32_t vocab, int32_t slice) {
  return uint32_t((int64_t(vocab) + slice - 1) / slice);
}

}  // namespace

size_t distill_workspace(int32_t rows, int32_t vocab, int32_t top) {
  if (rows >= kWholeRows) return 0;
  const size_t n = size_t(rows) * slices_of(vocab, slice_of(rows, vocab)) * sizeof(Part);
  return (n + 255) / 256 * 256;
}

hipError_t launch_distill(const embbag_distill_t& a, char* ws, int32_t* status, hipStream_t st) {
  if (a.rows == 0) return hipSuccess;
  DistillDev dv;
  dv.a = a;
  dv.slice = slice_of(a.rows, a.vocab);
  dv.slices = slices_of(a.vocab, dv.slice);
  dv.parts = reinterpret_cast<Part*>(ws);
  dv.first = 0;
  if (a.type == EMBBAG_BF16)
    launch_type<__bf16>(dv, status, st);
  else
    launch_type<float>(dv, status, st);
  return hipGetLastError();
}

}  // namespace embbag
