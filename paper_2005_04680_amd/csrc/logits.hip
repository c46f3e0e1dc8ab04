// What may be answered: penalties for seen tokens, biases and masks on rows of
// logits.
//
// A block takes one slice of one row.  It walks the row's lists and keeps in LDS,
// for every token of its slice, a word of occurrences (bit 31: in the prompt; the
// rest: how often after it) and the place of its last bias: integer additions and
// maxima, whose order does not matter.  Then it streams the slice once, 16 bytes per
// lane where the row's alignment allows.  Every element is read and written by one
// thread, so that `out` may be `logits`.
#include "head.hpp"

namespace embbag {
namespace {

constexpr uint32_t kPrompt = 0x80000000u;

struct LogitsDev {
  embbag_logits_t a;
  int32_t slice;    // tokens per block, a multiple of 8
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

template <class T, bool SEEN, bool BIAS>
__global__ __launch_bounds__(kBlock) void logits_kernel(LogitsDev dv,
                                                        int32_t* __restrict__ status) {
  constexpr int V = kVec<T>;
  extern __shared__ uint32_t lds[];
  const embbag_logits_t& a = dv.a;
  const int r = int(blockIdx.x / dv.slices);
  const int base = int(blockIdx.x - uint32_t(r) * dv.slices) * dv.slice;
  const int len = min(dv.slice, a.vocab - base);
  const T* x = static_cast<const T*>(a.logits) + int64_t(r) * a.logits_stride + base;
  T* y = static_cast<T*>(a.out) + int64_t(r) * a.out_stride + base;
  int err = 0;

  // Vectors start at the first 16-byte boundary of x if y has one there too;
  // token v of the slice is at LDS place v + pad, so that vectors are aligned there.
  const int head0 = head_of(x);
  const int head = head0 == head_of(y) ? min(head0, len) : len;
  const int pad = (V - head % V) % V;
  const int places = dv.slice + V;
  uint32_t* occ = lds;
  uint32_t* bia = lds + (SEEN ? places : 0);
  int b0 = 0, b1 = 0;

  if constexpr (SEEN || BIAS) {
    const int words = places * (int(SEEN) + int(BIAS));
    for (int i = threadIdx.x * 4; i < words; i += kBlock * 4)
      *reinterpret_cast<u4*>(lds + i) = u4{0u, 0u, 0u, 0u};
    __syncthreads();
  }
  if constexpr (SEEN) {
    int s0, s1;
    list_of(a.seen_offsets, r, a.rows, a.num_seen, &s0, &s1, &err);
    const int plen = a.prompt_lens != nullptr ? a.prompt_lens[r] : 0;
    for (int64_t j = s0 + int(threadIdx.x); j < s1; j += kBlock) {
      const int v = a.seen[j];
      if (uint32_t(v) >= uint32_t(a.vocab)) {
        err = min(err, EMBBAG_ERR_INDEX_RANGE);
        continue;
      }
      const int at = v - base;
      if (uint32_t(at) < uint32_t(len)) {
        if (j - s0 < plen)
          atomicOr(&occ[at + pad], kPrompt);
        else
          atomicAdd(&occ[at + pad], 1u);
      }
    }
  }
  if constexpr (BIAS) {
    list_of(a.bias_offsets, r, a.rows, a.num_biases, &b0, &b1, &err);
    for (int64_t j = b0 + int(threadIdx.x); j < b1; j += kBlock) {
      const int v = a.bias_ids[j];
      if (uint32_t(v) >= uint32_t(a.vocab)) {
        err = min(err, EMBBAG_ERR_INDEX_RANGE);
        continue;
      }
      const int at = v - base;
      if (uint32_t(at) < uint32_t(len)) atomicMax(&bia[at + pad], uint32_t(j - b0) + 1u);
    }
  }
  if constexpr (SEEN || BIAS) __syncthreads();

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

  auto change = [&](float l, uint32_t o, uint32_t b) {
    if constexpr (SEEN) {
      if (o != 0u) {
        l = l > 0.f ? l / rho : l * rho;
        const uint32_t c = o & ~kPrompt;
        if (c != 0u) l -= freq * float(c) + pres;
      }
    }
    if constexpr (BIAS) {
      if (b != 0u) l += a.biases[int64_t(b0) + b - 1];
    }
    return l;
  };
  const float none = -__builtin_inff();

  // Elements before and after the vectors (all of them where x and y are not
  // aligned alike).
  const int vecs = (len - head) / V;
  const int scalars = len - vecs * V;
  for (int i = threadIdx.x; i < scalars; i += kBlock) {
    const int v = i < head ? i : i + vecs * V;
    float l = change(to_f32(x[v]), SEEN ? occ[v + pad] : 0u, BIAS ? bia[v + pad] : 0u);
    if (mask != nullptr && ((mask[(base + v) >> 5] >> ((base + v) & 31)) & 1u) == 0u) l = none;
    y[v] = T(l);
  }
  for (int i = threadIdx.x; i < vecs; i += kBlock) {
    const int v = head + i * V;
    float l[V];
    unpack16(*reinterpret_cast<const u4*>(x + v), l);
    if constexpr (SEEN || BIAS) {
      uint32_t o[V] = {}, b[V] = {};
#pragma unroll
      for (int e = 0; e < V; e += 4) {
        if constexpr (SEEN) {
          const u4 w = *reinterpret_cast<const u4*>(occ + v + pad + e);
          o[e] = w.x, o[e + 1] = w.y, o[e + 2] = w.z, o[e + 3] = w.w;
        }
        if constexpr (BIAS) {
          const u4 w = *reinterpret_cast<const u4*>(bia + v + pad + e);
          b[e] = w.x, b[e + 1] = w.y, b[e + 2] = w.z, b[e + 3] = w.w;
        }
      }
#pragma unroll
      for (int e = 0; e < V; ++e) l[e] = change(l[e], o[e], b[e]);
    }
    if (mask != nullptr) {
      // A vector's bits lie in one or two words.
      const int t = base + v, w0 = t >> 5, w1 = (t + V - 1) >> 5;
      const uint64_t bits = (uint64_t(mask[w1]) << 32 | mask[w0]) >> (t & 31);
#pragma unroll
      for (int e = 0; e < V; ++e)
        if (((bits >> e) & 1u) == 0u) l[e] = none;
    }
    *reinterpret_cast<u4*>(y + v) = pack16(l);
  }
  if (err != 0 && status != nullptr) atomicMin(status, err);
}

template <class T>
void launch_type(const LogitsDev& dv, dim3 grid, size_t lds, int32_t* status, hipStream_t st) {
  const bool seen = dv.a.seen_offsets != nullptr, bias = dv.a.bias_offsets != nullptr;
  if (seen && bias)
    hipLaunchKernelGGL((logits_kernel<T, true, true>), grid, dim3(kBlock), lds, st, dv, status);
  else if (seen)
    hipLaunchKernelGGL((logits_kernel<T, true, false>), grid, dim3(kBlock), lds, st, dv, status);
  else if (bias)
    hipLaunchKernelGGL((logits_kernel<T, false, true>), grid, dim3(kBlock), lds, st, dv, status);
  else
    hipLaunchKernelGGL((logits_kernel<T, false, false>), grid, dim3(kBlock), lds, st, dv, status);
}

}  // namespace

hipError_t launch_logits(const embbag_logits_t& a, int32_t* status, hipStream_t st) {
  if (a.rows == 0) return hipSuccess;
  LogitsDev dv;
  dv.a = a;
  dv.slice = 4096;
  dv.slices = uint32_t((int64_t(a.vocab) + dv.slice - 1) / dv.slice);
  const int lists = int(a.seen_offsets != nullptr) + int(a.bias_offsets != nullptr);
  const size_t lds = size_t(lists) * size_t(dv.slice + 8) * 4;
  const dim3 grid(dv.slices * uint32_t(a.rows));
  if (a.type == EMBBAG_BF16)
    launch_type<__bf16>(dv, grid, lds, status, st);
  else
    launch_type<float>(dv, grid, lds, status, st);
  return hipGetLastError();
}

}  // namespace embbag
