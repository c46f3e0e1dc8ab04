// What may be answered: penalties for seen tokens, biases and masks on rows of
// logits.
//
// A block takes one slice of one row.  It walks the row's lists and keeps in LDS a word
// for every token of its slice: bit 31, seen in the prompt; bit 30, has a bias; the rest, how
// often seen after the prompt (integer additions, whose order does not matter).  The biases of
// the slice are few: they go to a list, and a token's last one is found among them.  Its
// thread gets the token's value through the word and writes it again after the stream.  The
// slice itself is on its way meanwhile, 16 bytes per load, and is read and written once.  A
// block is a chain of a few memory latencies (offsets, lists, stores), so the lists
// come in batches of 16 entries per thread and many blocks share a compute unit.  Every
// element is read by one thread, so that `out` may be `logits`.
//
// 256 x 131072 BF16 with up to 4096 seen tokens, 300 biases and masks: 45 us (20 us without
// lists and masks, 6.6 TB/s; 33 us with the seen tokens alone): bound by the vector instructions of the
// lists' walk, which every slice repeats, and of the touched tokens (69% of the cycles), and by the
// chain.  Blocks that keep the lists in registers over several slices were slower (64 us: fewer of
// them share a unit), and so were biases added in the stream (47 us; 5000 of them 77 us, 57 here).
//
// Rows with more than kListed biases take them in a pass of their own first, with the words as the
// places of the tokens' last biases.
#include "head.hpp"

namespace embbag {
namespace {

constexpr uint32_t kPrompt = 0x80000000u;
constexpr uint32_t kBiased = 0x40000000u;
constexpr int kSliceTokens = 4096;
constexpr int kListed = 4 * kBlock;  // biases of a row that go to the list (16 bits hold their places)

struct LogitsDev {
  embbag_logits_t a;
  uint32_t slices;  // per row
  uint32_t first;   // block that the launch begins with
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

// Calls fn(place in the list, entry) for entries [from, to) of `list`, up to four loads of four
// entries in flight per thread.  Returns the largest entry, unsigned.
template <class Fn>
__device__ __forceinline__ uint32_t walk(const int32_t* list, int from, int to, Fn fn) {
  constexpr uint32_t U = 4, kStep = 4 * kBlock;
  const uint32_t n = uint32_t(to) - uint32_t(from);
  uint32_t largest = 0u;
  list += from;
  for (uint32_t j0 = 0; j0 < n; j0 += U * kStep) {
    u4 v[U];
#pragma unroll
    for (uint32_t u = 0; u < U; ++u) {
      const uint32_t j = j0 + u * kStep + threadIdx.x * 4;
      if (j0 + u * kStep < n && j + 4 <= n) v[u] = load16(list + j);
    }
#pragma unroll
    for (uint32_t u = 0; u < U; ++u) {
      if (j0 + u * kStep >= n) break;
      const uint32_t j = j0 + u * kStep + threadIdx.x * 4;
      if (j + 4 <= n) {
        largest = max(max(largest, max(v[u].x, v[u].y)), max(v[u].z, v[u].w));
        fn(j, v[u].x);
        fn(j + 1, v[u].y);
        fn(j + 2, v[u].z);
        fn(j + 3, v[u].w);
      } else {
        for (uint32_t i = j; i < n; ++i) {
          const uint32_t e = uint32_t(list[i]);
          largest = max(largest, e);
          fn(i, e);
        }
      }
    }
  }
  return largest;
}

// l / rho from the reciprocal: the product's remainder, which is exact, corrects it to the
// division's rounding.  (Overflow and infinities stay what the product gave.)
__device__ __forceinline__ float divide(float l, float rho, float inv) {
  const float q = l * inv;
  const float c = fmaf(fmaf(-q, rho, l), inv, q);
  return fabsf(q) < __builtin_inff() ? c : q;
}

template <class T, bool SEEN, bool BIAS>
__global__ __launch_bounds__(kBlock) void logits_kernel(LogitsDev dv,
                                                        int32_t* __restrict__ status) {
  constexpr int V = kVec<T>;
  constexpr int NV = kSliceTokens / (kBlock * V);  // vectors per thread
  constexpr int PER = kListed / kBlock;            // listed biases per thread
  constexpr bool ANY = SEEN || BIAS;
  __shared__ __align__(16) uint32_t words[ANY ? kSliceTokens : 4];
  // Token of the slice << 16 | place in the row's list.
  __shared__ __align__(16) uint32_t listed[BIAS ? kListed : 4];
  __shared__ uint32_t num_listed;
  const embbag_logits_t& a = dv.a;
  const uint32_t block = dv.first + blockIdx.x;
  const int r = int(block / dv.slices);
  const int base = int(block - uint32_t(r) * dv.slices) * kSliceTokens;
  const int len = min(kSliceTokens, a.vocab - base);
  const T* x = static_cast<const T*>(a.logits) + int64_t(r) * a.logits_stride + base;
  T* y = static_cast<T*>(a.out) + int64_t(r) * a.out_stride + base;
  int err = 0;

  u4 raw[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int v = (i * kBlock + int(threadIdx.x)) * V;
    if (v < len) raw[i] = load_vec(x + v, len - v);
  }
  int s0 = 0, s1 = 0, b0 = 0, b1 = 0;
  if constexpr (SEEN) list_of(a.seen_offsets, r, a.rows, a.num_seen, &s0, &s1, &err);
  if constexpr (BIAS) list_of(a.bias_offsets, r, a.rows, a.num_biases, &b0, &b1, &err);
  const uint32_t* mask = nullptr;
  if (a.masks != nullptr) {
    const int id = a.mask_ids != nullptr ? a.mask_ids[r] : r;
    if (id >= a.num_masks)
      err = min(err, EMBBAG_ERR_INDEX_RANGE);
    else if (id >= 0)
      mask = a.masks + int64_t(id) * a.mask_stride;
  }
  // V tokens from a multiple of V: their bits lie in one word.
  uint32_t bits[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int v = (i * kBlock + int(threadIdx.x)) * V;
    bits[i] = 0xFFFFFFFFu;
    if (mask != nullptr && v < len) bits[i] = mask[(base + v) >> 5] >> ((base + v) & 31);
  }
  const int plen = SEEN && a.prompt_lens != nullptr ? a.prompt_lens[r] : 0;
  const float rho = SEEN && a.repetition != nullptr ? a.repetition[r] : 1.f;
  const float inv = 1.f / rho;
  const bool plain = rho > 0x1p-60f && rho < 0x1p60f;
  const float freq = SEEN && a.frequency != nullptr ? a.frequency[r] : 0.f;
  const float pres = SEEN && a.presence != nullptr ? a.presence[r] : 0.f;
  auto clear = [&]() {
#pragma unroll
    for (int i = 0; i < kSliceTokens / (kBlock * 4); ++i)
      *reinterpret_cast<u4*>(words + (i * kBlock + threadIdx.x) * 4) = u4{0u, 0u, 0u, 0u};
  };

  // A long list of biases: their sum with 0 for this thread's tokens (-0.0 where there is none, which
  // adds nothing).
  const bool longer = BIAS && b1 - b0 > kListed;
  float add[NV * V];
  if (longer) {
    clear();
    __syncthreads();
    const uint32_t worst = walk(a.bias_ids, b0, b1, [&](uint32_t j, uint32_t v) {
      const uint32_t at = v - uint32_t(base);
      if (at < uint32_t(len)) atomicMax(&words[at], j + 1u);
    });
    if (worst >= uint32_t(a.vocab)) err = min(err, EMBBAG_ERR_INDEX_RANGE);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NV * V; ++i) {
      const int v = (i / V * kBlock + int(threadIdx.x)) * V + i % V;
      const uint32_t b = v < len ? words[v] : 0u;
      add[i] = b != 0u ? a.biases[int64_t(b0) + b - 1] : -0.f;
    }
    __syncthreads();
  }

  if constexpr (ANY) {
    clear();
    if constexpr (BIAS) *reinterpret_cast<u4*>(listed + threadIdx.x * 4) = u4{0u, 0u, 0u, 0u};
    if (threadIdx.x == 0) num_listed = 0u;
    __syncthreads();
  }
  if constexpr (BIAS) {
    if (!longer) {
      const uint32_t worst = walk(a.bias_ids, b0, b1, [&](uint32_t j, uint32_t v) {
        const uint32_t at = v - uint32_t(base);
        if (at < uint32_t(len)) {
          listed[atomicAdd(&num_listed, 1u)] = at << 16 | j;
          atomicOr(&words[at], kBiased);
        }
      });
      if (worst >= uint32_t(a.vocab)) err = min(err, EMBBAG_ERR_INDEX_RANGE);
    }
  }
  if constexpr (SEEN) {
    const uint32_t worst = walk(a.seen, s0, s1, [&](uint32_t j, uint32_t v) {
      const uint32_t at = v - uint32_t(base);
      if (at < uint32_t(len)) {
        if (int64_t(j) < plen)
          atomicOr(&words[at], kPrompt);
        else
          atomicAdd(&words[at], 1u);
      }
    });
    if (worst >= uint32_t(a.vocab)) err = min(err, EMBBAG_ERR_INDEX_RANGE);
  }
  if constexpr (ANY) __syncthreads();

  // The last listed bias of a token finds itself: no entry of the token has a later place.  (Four at
  // a time; the list's unused entries are 0, which is later than none.)
  const int n = BIAS ? int(num_listed) : 0;
  float bias[PER];
  int token[PER];
#pragma unroll
  for (int q = 0; q < PER; ++q) {
    const int e = q * kBlock + int(threadIdx.x);
    token[q] = -1;
    if (!BIAS || q * kBlock >= n || e >= n) continue;
    const uint32_t mine = listed[e];
    bool lastly = true;
    for (int i = 0; i < n; i += 4) {
      const u4 o = *reinterpret_cast<const u4*>(listed + i);
      auto before = [&](uint32_t other) { return other <= mine || (other >> 16) != (mine >> 16); };
      lastly = lastly && before(o.x) && before(o.y) && before(o.z) && before(o.w);
    }
    if (lastly) {
      token[q] = int(mine >> 16);
      bias[q] = a.biases[int64_t(b0) + (mine & 0xFFFFu)];
    }
  }

#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int v = (i * kBlock + int(threadIdx.x)) * V;
    if (v >= len) continue;
    float l[V];
    unpack16(raw[i], l);
    if constexpr (ANY) {
      uint32_t o[V], any = 0u;
#pragma unroll
      for (int e = 0; e < V; e += 4) {
        const u4 w = *reinterpret_cast<const u4*>(words + v + e);
        o[e] = w.x, o[e + 1] = w.y, o[e + 2] = w.z, o[e + 3] = w.w;
        any |= w.x | w.y | w.z | w.w;
      }
      if (any != 0u) {
#pragma unroll
        for (int e = 0; e < V; ++e) {
          if (SEEN && (o[e] & ~kBiased) != 0u) {
            l[e] = l[e] > 0.f ? (plain ? divide(l[e], rho, inv) : l[e] / rho) : l[e] * rho;
            const uint32_t c = o[e] & (kBiased - 1u);
            l[e] -= c != 0u ? freq * float(c) + pres : 0.f;
          }
          if (BIAS && (o[e] & kBiased) != 0u) words[v + e] = __float_as_uint(l[e]);
        }
      }
      if (longer) {
#pragma unroll
        for (int e = 0; e < V; ++e) l[e] += add[i * V + e];
      }
    }
    if (mask != nullptr) {
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const uint32_t keep = uint32_t(__builtin_amdgcn_sbfe(int(bits[i]), uint32_t(e), 1u));
        l[e] = __uint_as_float((__float_as_uint(l[e]) & keep) | (__float_as_uint(low()) & ~keep));
      }
    }
    store_vec(y + v, len - v, l);
  }
  if constexpr (BIAS) {
    if (n > 0) {
      __syncthreads();
#pragma unroll
      for (int q = 0; q < PER; ++q) {
        const int v = token[q];
        if (v < 0) continue;
        const bool out = mask != nullptr && ((mask[(base + v) >> 5] >> ((base + v) & 31)) & 1u) == 0u;
        y[v] = T(out ? low() : __uint_as_float(words[v]) + bias[q]);
      }
    }
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
  for_launches(int64_t(dv.slices) * a.rows, kBlock, [&](uint32_t first, dim3 grid) {
    dv.first = first;
    if (a.type == EMBBAG_BF16)
      launch_type<__bf16>(dv, grid, status, st);
    else
      launch_type<float>(dv, grid, status, st);
  });
  return hipGetLastError();
}

}  // namespace embbag
