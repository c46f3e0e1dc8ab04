// What may be answered: penalties for seen tokens, biases and masks on rows of
// logits.
//
// A block takes one slice of one row.  It walks the row's lists and keeps in LDS,
// for every token of its slice, a word of occurrences (bit 31: in the prompt; the
// rest: how often after it) and the place of its last bias: integer additions and
// maxima, whose order does not matter.  The slice itself is on its way meanwhile, 16 bytes per
// load, and is read and written once.  A block is a chain of a few memory latencies
// (offsets, lists, stores), so the lists come in batches of 16 entries per thread and
// several blocks share a compute unit.  Every element is read and written by one thread, so
// that `out` may be `logits`.
#include "head.hpp"

namespace embbag {
namespace {

constexpr uint32_t kPrompt = 0x80000000u;
constexpr int kSliceTokens = 4096;

struct LogitsDev {
  embbag_logits_t a;
  uint32_t slices;  // per row
};

// [o[r], o[r+1]) of a list of n entries, empty (and an error) where it is none.
__device__ __forceinline__ void list_of(const int32_t* o, int r, int rows, int64_t n, int* from,
                                        int* to, int* err) {
  const int a = o[r], b = o[r + 1];
  const bool bad = a < 0 || b < a || b > n || (r == 0 && a != 0) || (r == rows - 1 && b != n);
  if (bad) *err = EMBBAG_ERR_OFFSETS;
  *from = bad ? 0 : a;
  *to = bad ? 0 : b;
}

// Calls fn(place in the list, entry) for entries [from, to) of `list`, four loads of four
// entries in flight per thread.
template <class Fn>
__device__ __forceinline__ void walk(const int32_t* list, int from, int to, Fn fn) {
  constexpr int U = 4;
  const uint32_t n = uint32_t(to) - uint32_t(from);
  list += from;
  uint32_t j0 = 0;
  for (; j0 < n; j0 += U * 4 * kBlock) {
    u4 v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint32_t j = j0 + (u * kBlock + threadIdx.x) * 4;
      v[u] = u4{0xFFFFFFFFu, 0xFFFFFFFFu, 0xFFFFFFFFu, 0xFFFFFFFFu};
      if (j + 4 <= n) {
        v[u] = load16(list + j);
      } else if (j < n) {
        v[u].x = uint32_t(list[j]);
        if (j + 1 < n) v[u].y = uint32_t(list[j + 1]);
        if (j + 2 < n) v[u].z = uint32_t(list[j + 2]);
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint32_t j = j0 + (u * kBlock + threadIdx.x) * 4;
      if (j < n) fn(j, v[u].x);
      if (j + 1 < n) fn(j + 1, v[u].y);
      if (j + 2 < n) fn(j + 2, v[u].z);
      if (j + 3 < n) fn(j + 3, v[u].w);
    }
  }
}

template <class T, bool SEEN, bool BIAS>
__global__ __launch_bounds__(kBlock) void logits_kernel(LogitsDev dv,
                                                        int32_t* __restrict__ status) {
  constexpr int V = kVec<T>;
  constexpr int NV = kSliceTokens / (kBlock * V);  // vectors per thread
  constexpr int LISTS = int(SEEN) + int(BIAS);
  __shared__ __align__(16) uint32_t lds[LISTS * kSliceTokens + 4];
  const embbag_logits_t& a = dv.a;
  const int r = int(blockIdx.x / dv.slices);
  const int base = int(blockIdx.x - uint32_t(r) * dv.slices) * kSliceTokens;
  const int len = min(kSliceTokens, a.vocab - base);
  const T* x = static_cast<const T*>(a.logits) + int64_t(r) * a.logits_stride + base;
  T* y = static_cast<T*>(a.out) + int64_t(r) * a.out_stride + base;
  int err = 0;
  uint32_t* occ = lds;
  uint32_t* bia = lds + (SEEN ? kSliceTokens : 0);

  u4 raw[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int v = (i * kBlock + int(threadIdx.x)) * V;
    if (v < len) raw[i] = load_vec(x + v, len - v);
  }
  int s0 = 0, s1 = 0, b0 = 0, b1 = 0;
  if constexpr (SEEN) list_of(a.seen_offsets, r, a.rows, a.num_seen, &s0, &s1, &err);
  if constexpr (BIAS) list_of(a.bias_offsets, r, a.rows, a.num_biases, &b0, &b1, &err);
  if constexpr (LISTS > 0) {
#pragma unroll
    for (int i = 0; i < LISTS * kSliceTokens / (kBlock * 4); ++i)
      *reinterpret_cast<u4*>(lds + (i * kBlock + threadIdx.x) * 4) = u4{0u, 0u, 0u, 0u};
    __syncthreads();
  }
  if constexpr (SEEN) {
    const int plen = a.prompt_lens != nullptr ? a.prompt_lens[r] : 0;
    walk(a.seen, s0, s1, [&](uint32_t j, uint32_t v) {
      if (v >= uint32_t(a.vocab)) {
        err = min(err, EMBBAG_ERR_INDEX_RANGE);
        return;
      }
      const uint32_t at = v - uint32_t(base);
      if (at < uint32_t(len)) {
        if (int64_t(j) < plen)
          atomicOr(&occ[at], kPrompt);
        else
          atomicAdd(&occ[at], 1u);
      }
    });
  }
  if constexpr (BIAS) {
    walk(a.bias_ids, b0, b1, [&](uint32_t j, uint32_t v) {
      if (v >= uint32_t(a.vocab)) {
        err = min(err, EMBBAG_ERR_INDEX_RANGE);
        return;
      }
      const uint32_t at = v - uint32_t(base);
      if (at < uint32_t(len)) atomicMax(&bia[at], j + 1u);
    });
  }
  const uint32_t* mask = nullptr;
  if (a.masks != nullptr) {
    const int id = a.mask_ids != nullptr ? a.mask_ids[r] : r;
    if (id >= a.num_masks)
      err = min(err, EMBBAG_ERR_INDEX_RANGE);
    else if (id >= 0)
      mask = a.masks + int64_t(id) * a.mask_stride;
  }
  const float rho = SEEN && a.repetition != nullptr ? a.repetition[r] : 1.f;
  const float freq = SEEN && a.frequency != nullptr ? a.frequency[r] : 0.f;
  const float pres = SEEN && a.presence != nullptr ? a.presence[r] : 0.f;
  if constexpr (LISTS > 0) __syncthreads();

#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int v = (i * kBlock + int(threadIdx.x)) * V;
    if (v >= len) continue;
    float l[V];
    unpack16(raw[i], l);
    if constexpr (SEEN) {
      uint32_t o[V], any = 0u;
#pragma unroll
      for (int e = 0; e < V; e += 4) {
        const u4 w = *reinterpret_cast<const u4*>(occ + v + e);
        o[e] = w.x, o[e + 1] = w.y, o[e + 2] = w.z, o[e + 3] = w.w;
        any |= w.x | w.y | w.z | w.w;
      }
      if (any != 0u) {
#pragma unroll
        for (int e = 0; e < V; ++e) {
          if (o[e] == 0u) continue;
          l[e] = l[e] > 0.f ? l[e] / rho : l[e] * rho;
          const uint32_t c = o[e] & ~kPrompt;
          if (c != 0u) l[e] -= freq * float(c) + pres;
        }
      }
    }
    if constexpr (BIAS) {
      uint32_t o[V], any = 0u;
#pragma unroll
      for (int e = 0; e < V; e += 4) {
        const u4 w = *reinterpret_cast<const u4*>(bia + v + e);
        o[e] = w.x, o[e + 1] = w.y, o[e + 2] = w.z, o[e + 3] = w.w;
        any |= w.x | w.y | w.z | w.w;
      }
      if (any != 0u) {
#pragma unroll
        for (int e = 0; e < V; ++e)
          if (o[e] != 0u) l[e] += a.biases[int64_t(b0) + o[e] - 1];
      }
    }
    if (mask != nullptr) {
      // V tokens from a multiple of V: their bits lie in one word.
      const uint32_t bits = mask[(base + v) >> 5] >> ((base + v) & 31);
#pragma unroll
      for (int e = 0; e < V; ++e)
        if (((bits >> e) & 1u) == 0u) l[e] = low();
    }
    store_vec(y + v, len - v, l);
  }
  if (err != 0 && status != nullptr) atomicMin(status, err);
}

template <class T>
void launch_type(const LogitsDev& dv, dim3 grid, int32_t* status, hipStream_t st) {
  const bool seen = dv.a.seen_offsets != nullptr, bias = dv.a.bias_offsets != nullptr;
  if (seen && bias)
    hipLaunchKernelGGL((logits_kernel<T, true, true>), grid, dim3(kBlock), 0, st, dv, status);
  else if (seen)
    hipLaunchKernelGGL((logits_kernel<T, true, false>), grid, dim3(kBlock), 0, st, dv, status);
  else if (bias)
    hipLaunchKernelGGL((logits_kernel<T, false, true>), grid, dim3(kBlock), 0, st, dv, status);
  else
    hipLaunchKernelGGL((logits_kernel<T, false, false>), grid, dim3(kBlock), 0, st, dv, status);
}

}  // namespace

hipError_t launch_logits(const embbag_logits_t& a, int32_t* status, hipStream_t st) {
  if (a.rows == 0) return hipSuccess;
  LogitsDev dv;
  dv.a = a;
  dv.slices = uint32_t((int64_t(a.vocab) + kSliceTokens - 1) / kSliceTokens);
  const dim3 grid(dv.slices * uint32_t(a.rows));
  if (a.type == EMBBAG_BF16)
    launch_type<__bf16>(dv, grid, status, st);
  else
    launch_type<float>(dv, grid, status, st);
  return hipGetLastError();
}

}  // namespace embbag
