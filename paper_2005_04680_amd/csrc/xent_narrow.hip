// Cross entropy over a narrow table (dim <= 128): the scores' gradient D is made where it is used and
// never leaves the registers.
//
// The products of a narrow table are short beside what D would cost in memory (at dim 64 a score takes
// 128 operations, D's element 2 to 6 bytes written and read several times), so each gradient computes the
// scores again for itself: 10 instead of 8 products' worth of operations, none of the traffic.
//   - Rows of x stand (in registers) and the table streams through LDS: scores' sums, and dx.
//   - Rows of the table stand and the rows that count stream: dW.
// A wavefront's 32 x 32 scores come out of the matrix instructions with a standing row per lane and the
// streaming rows 8 q + 4 (lane / 32) + e in registers 4 q + e.  As the second product's operand, a lane's
// 8 elements of k may be any, as long as the other side has the same: registers 8 t .. 8 t + 7 are the
// streaming rows 16 t + 4 (lane / 32) + {0..3, 8..11}, which two transposing reads of the streaming tile
// in LDS give in that order.  So D goes from one product to the next with no exchange between lanes.
//
// Streaming tiles are double-buffered: the next one's elements are on their way in registers while this
// one's products run, and are split into their BF16 terms on the way to LDS.
//
// Bound by matrix and vector instructions, each about half of the cycles (exponentials, D's terms and their
// packing beside the products).  Measured, us: FP32 2048 x 100003 x 64 671, 33 x 32001 x 128 56, BF16 4000 x 50000 x
// 128 332, its loss alone over 100000 158.  The FP32 gradients of dim > 64 have all 256 registers of two wavefronts per SIMD
// (96 for the standing rows' terms, 64 for their sums) and spill 108 to 168 bytes a lane.
#include <type_traits>

#include "xent.hpp"

namespace embbag {
namespace {

typedef float f16v __attribute__((ext_vector_type(16)));
typedef short s4v __attribute__((ext_vector_type(4)));

// The place of 16-byte chunk c of row r in LDS, rows of EP elements: rows r = 0..15 at one chunk, and four
// rows at four neighbouring ones, meet all banks.
template <int EP>
__device__ __forceinline__ int chunk_at(int r, int c) {
  const int f = EP == 64 ? (r >> 1 & 1) << 2 | (r >> 2 & 1) << 1 | (r >> 3 & 1)
                         : (r & 3) << 2 | (r >> 2 & 3);
  return c ^ f;
}

// Pair i of planes (smallest products first): of a side with P planes and one with PD.
template <int P, int PD>
constexpr int kPairs = P == 3 ? 6 : PD;
template <int P, int PD>
__device__ constexpr int first_of(int i) {
  constexpr int a[6] = {2, 1, 0, 1, 0, 0};
  return P == 3 ? a[i] : 0;
}
template <int P, int PD>
__device__ constexpr int second_of(int i) {
  constexpr int b[6] = {0, 1, 2, 0, 1, 0};
  return P == 3 ? b[i] : PD - 1 - i;
}

__device__ __forceinline__ f16v mfma(const u4& a, const u4& b, const f16v& c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf8, a), __builtin_bit_cast(bf8, b), c, 0,
                                                 0, 0);
}

// As P planes of BF16 terms.
template <int P, class T>
__device__ __forceinline__ void terms_of(const Eight<T>& x, u4 (&t)[P]) {
  if constexpr (P == 1) {
    t[0] = x.w;
  } else {
    float v[8];
    x.values(v);
    nearest_terms(v, t);
  }
}

// Fragments of a tile in LDS: rows of EP elements, plane after plane.
template <int EP>
struct Tile {
  static constexpr int ROW = EP * 2;
  // Row r, elements 16 s + 8 half on.
  static __device__ __forceinline__ u4 rows(const uint8_t* t, int r, int s, int half) {
    return *reinterpret_cast<const u4*>(t + r * ROW + chunk_at<EP>(r, 2 * s + half) * 16);
  }
  // Element e0 + lane % 32 of rows r0 + 4 half + {0..3, 8..11}.
  static __device__ __forceinline__ u4 turned(const uint8_t* t, int r0, int e0, int lane) {
    const int half = lane / 32, c = e0 / 8 + lane / 16 % 2 * 2 + lane % 4 / 2;
    const int r = r0 + half * 4 + lane % 16 / 4;
    typedef __attribute__((address_space(3))) s4v* lds4;
    const s4v lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
        (lds4)(t + r * ROW + chunk_at<EP>(r, c) * 16 + lane % 2 * 8));
    const s4v hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
        (lds4)(t + (r + 8) * ROW + chunk_at<EP>(r + 8, c) * 16 + lane % 2 * 8));
    const u2 l2 = __builtin_bit_cast(u2, lo), h2 = __builtin_bit_cast(u2, hi);
    return u4{l2.x, l2.y, h2.x, h2.y};
  }
};

// Registers 8 t .. 8 t + 7 of d as PD planes of BF16 terms.
template <int PD>
__device__ __forceinline__ void d_terms(const f16v& d, int t, u4 (&out)[PD]) {
  float v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = d[t * 8 + i];
#pragma unroll
  for (int k = 0; k < PD; ++k) {
    out[k] = pack16(v);
    if (k + 1 == PD) break;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] -= (i % 2 ? bf16_hi : bf16_lo)(out[k][i / 2]);
  }
}

// What the first term leaves of them, as BF16.
__device__ __forceinline__ u4 second_term(const f16v& d, int t, const u4& term) {
  float v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = d[t * 8 + i] - (i % 2 ? bf16_hi : bf16_lo)(term[i / 2]);
  return pack16(v);
}

struct TokenArgs {
  const void* table;
  int64_t stride;
  int64_t vocab;
  int32_t dim;
  const __bf16* x;
  int64_t x_plane;
  const Head* head;
  const Token* tokens;
  float* target;
  float unit;
  float2* sums;
  float* dx;
  int32_t rows;
  int32_t splits, per;
};

// Groups of 32 standing rows per wavefront: two meet every fragment of the streaming tile where their
// registers leave room for a second wavefront on the SIMD, whose products run while the first one makes D.
template <int EP, int P>
constexpr int kStanding = P == 1 && EP == 64 ? 2 : 1;
constexpr int standing(int dim, bool f32) { return !f32 && dim <= 64 ? 2 : 1; }
// Groups of 32 rows that a wavefront takes from a streaming tile of the table, and of x.
template <int P, int WV>
constexpr int kGroups = WV == 1 && P == 1 ? 2 : 1;
constexpr int groups(int wv, bool f32) { return wv == 1 && !f32 ? 2 : 1; }

// WM wavefronts side by side over rows of x (32 TM each), the others over the rows of the table's tile,
// SUB groups of 32 of them each.  GRAD: dx, else the sums.
template <int EP, int P, int PD, int WM, bool GRAD, class TW>
__device__ __forceinline__ void narrow_tokens(const TokenArgs& a, uint32_t block, uint8_t* lds) {
  constexpr int TM = kStanding<EP, P>, WV = 4 / WM, SUB = kGroups<P, WV>;
  constexpr int BM = 32 * TM * WM, VB = 32 * WV * SUB, S = EP / 16;
  constexpr int TILE = VB * EP * 2, STAGE = TILE * P;
  constexpr int CHUNKS = VB * EP / 8 / kBlock;
  static_assert(CHUNKS >= 1, "a chunk per thread");
  typedef Tile<EP> L;
  const int lane = lane_id(), wave = wave_id(), half = lane / 32, row = lane % 32;
  const int wm = wave % WM, wv = wave / WM;
  const int live = __builtin_amdgcn_readfirstlane(a.head->live);
  const uint32_t z = block % uint32_t(a.splits), tb = block / uint32_t(a.splits);
  if (int64_t(tb) * BM >= live) return;
  const int64_t v0 = int64_t(z) * a.per, v1 = min(v0 + a.per, a.vocab);

  // The standing rows, and what the gradient needs of them.
  u4 x[TM][P][S];
  int at[TM], label[TM];
  float top[TM], inv[TM], ratio[TM], sum[TM];
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    at[i] = int(tb) * BM + (wm * TM + i) * 32 + row;
    const int r = min(at[i], live - 1);
#pragma unroll
    for (int p = 0; p < P; ++p)
#pragma unroll
      for (int s = 0; s < S; ++s)
        x[i][p][s] = *reinterpret_cast<const u4*>(a.x + p * a.x_plane + int64_t(r) * EP + s * 16 + half * 8);
    const Token t = a.tokens[r];
    label[i] = t.label;
    top[i] = GRAD ? t.top : low(), inv[i] = t.inv, ratio[i] = t.ratio, sum[i] = 0.f;
  }

  Eight<TW> next[CHUNKS];
  const TW* w = static_cast<const TW*>(a.table);
  auto fetch = [&](int64_t v) {
#pragma unroll
    for (int i = 0; i < CHUNKS; ++i) {
      const int c = i * kBlock + threadIdx.x, r = c / (EP / 8), e = c % (EP / 8) * 8;
      next[i].load(w + min(v + r, a.vocab - 1) * a.stride + e, a.dim - e);
    }
  };
  auto put = [&](uint8_t* st) {
#pragma unroll
    for (int i = 0; i < CHUNKS; ++i) {
      const int c = i * kBlock + threadIdx.x, r = c / (EP / 8), k = c % (EP / 8);
      u4 t[P];
      terms_of<P>(next[i], t);
#pragma unroll
      for (int p = 0; p < P; ++p)
        *reinterpret_cast<u4*>(st + p * TILE + r * (EP * 2) + chunk_at<EP>(r, k) * 16) = t[p];
    }
  };
  f16v dx[GRAD ? TM : 1][EP / 32];
  if constexpr (GRAD) {
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int e = 0; e < EP / 32; ++e) dx[i][e] = f16v{};
  }

  fetch(v0);
  put(lds);
  int cur = 0;
  for (int64_t v = v0; v < v1; v += VB) {
    __syncthreads();  // this tile is in LDS, and the other one has been read
    const bool more = v + VB < v1;
    if (more) fetch(v + VB);
    const uint8_t* st = lds + cur * STAGE;
#pragma unroll
    for (int g = 0; g < SUB; ++g) {
      const int r0 = (wv * SUB + g) * 32;
      f16v z2[TM];
#pragma unroll
      for (int i = 0; i < TM; ++i) z2[i] = f16v{};
#pragma unroll
      for (int s = 0; s < S; ++s) {
        u4 f[P];
#pragma unroll
        for (int p = 0; p < P; ++p) f[p] = L::rows(st + p * TILE, r0 + row, s, half);
#pragma unroll
        for (int k = 0; k < kPairs<P, 1>; ++k)
#pragma unroll
          for (int i = 0; i < TM; ++i)
            z2[i] = mfma(f[first_of<P, 1>(k)], x[i][second_of<P, 1>(k)][s], z2[i]);
      }
      // The lane's columns: v + r0 + 8 q + 4 half + e.
      const int64_t first = v + r0 + half * 4;
      const bool whole = v + r0 + 32 <= v1;
      bool labels = false;  // whether any of the wavefront's elements here is a label's
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        const int64_t place = label[i] - first;
        const bool mine = place >= 0 && place < 32 && place / 4 % 2 == 0 && label[i] < v1;
        const bool some = __builtin_amdgcn_ballot_w64(mine) != 0ull;
        labels = labels || some;
        if constexpr (GRAD) {
          const float c = inv[i] * ratio[i];
#pragma unroll
          for (int r = 0; r < 16; ++r)
            z2[i][r] = exp2_of(__builtin_fmaf(z2[i][r], a.unit, -top[i])) * c;
          if (some) {
            asm volatile("");  // (a branch: few tiles hold a label)
            const float less = mine ? ratio[i] : 0.f;
#pragma unroll
            for (int r = 0; r < 16; ++r) z2[i][r] -= int(place) == r / 4 * 8 + r % 4 ? less : 0.f;
          }
          if (!whole) {
            asm volatile("");
#pragma unroll
            for (int r = 0; r < 16; ++r)
              if (first + r / 4 * 8 + r % 4 >= v1) z2[i][r] = 0.f;
          }
        } else {
          if (some) {
            asm volatile("");
            float t = 0.f;
#pragma unroll
            for (int r = 0; r < 16; ++r)
              if (int(place) == r / 4 * 8 + r % 4) t = z2[i][r];
            if (mine && at[i] < live) a.target[at[i]] = t;
          }
          if (!whole) {
            asm volatile("");
#pragma unroll
            for (int r = 0; r < 16; ++r)
              if (first + r / 4 * 8 + r % 4 >= v1) z2[i][r] = low();
          }
          // `top` is an exponent, the sum stands beside exactly that.
          float m = z2[i][0];
#pragma unroll
          for (int r = 1; r < 16; ++r) m = fmaxf(m, z2[i][r]);
          m = fmaxf(m * a.unit, top[i]);
          const float ref = m == low() ? 0.f : m;
          float more_sum = 0.f;
#pragma unroll
          for (int r = 0; r < 16; ++r) more_sum += exp2_of(__builtin_fmaf(z2[i][r], a.unit, -ref));
          sum[i] = sum[i] * exp2_of(top[i] - ref) + more_sum;
          top[i] = m;
        }
      }
      if constexpr (GRAD) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          u4 d[TM][PD];
#pragma unroll
          for (int i = 0; i < TM; ++i) d_terms<PD>(z2[i], t, d[i]);
#pragma unroll
          for (int e = 0; e < EP / 32; ++e) {
            u4 f[P];
#pragma unroll
            for (int p = 0; p < P; ++p) f[p] = L::turned(st + p * TILE, r0 + t * 16, e * 32, lane);
#pragma unroll
            for (int k = 0; k < kPairs<P, PD>; ++k)
#pragma unroll
              for (int i = 0; i < TM; ++i)
                dx[i][e] = mfma(f[first_of<P, PD>(k)], d[i][second_of<P, PD>(k)], dx[i][e]);
          }
          if (PD == 1 && labels) {  // a label's element is most of its row's gradient: its second term too
#pragma unroll
            for (int i = 0; i < TM; ++i) d[i][0] = second_term(z2[i], t, d[i][0]);
#pragma unroll
            for (int e = 0; e < EP / 32; ++e) {
              const u4 f = L::turned(st, r0 + t * 16, e * 32, lane);
#pragma unroll
              for (int i = 0; i < TM; ++i) dx[i][e] = mfma(f, d[i][0], dx[i][e]);
            }
          }
        }
      }
    }
    cur ^= 1;
    if (more) put(lds + cur * STAGE);
  }
  const int64_t part = int64_t(z) * WV + wv;
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    if constexpr (GRAD) {
      if (at[i] < live) {
        float* p = a.dx + (part * a.rows + at[i]) * a.dim;
#pragma unroll
        for (int e = 0; e < EP / 32; ++e)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const int c = e * 32 + q * 8 + half * 4;
            if (c < a.dim)
              store4(p + c, f4{dx[i][e][q * 4], dx[i][e][q * 4 + 1], dx[i][e][q * 4 + 2], dx[i][e][q * 4 + 3]});
          }
      }
    } else {
      const float ot = __shfl_xor(top[i], 32, kWave), os = __shfl_xor(sum[i], 32, kWave);
      const float m = fmaxf(top[i], ot), ref = m == low() ? 0.f : m;
      const float s = sum[i] * exp2_of(top[i] - ref) + os * exp2_of(ot - ref);
      if (half == 0 && at[i] < live) a.sums[part * a.rows + at[i]] = float2{m, s};
    }
  }
}

struct VocabArgs {
  const void* table;
  int64_t stride;
  int64_t vocab;
  int32_t dim;
  const __bf16* x;
  int64_t x_plane;
  const Head* head;
  const Token* tokens;
  float unit;
  void* dw;
  int64_t dw_stride;
  int64_t dw_part;
  const float* factor;
  int32_t splits, per;
};

// A wavefront's 32 TV rows of the table stand, rows that count stream.
template <int MB>
struct Streamed {
  float tops[2][MB], scales[2][MB], ratios[2][MB];
  int labels[2][MB];
};
template <int EP, int P, int PD, class TW, class TO>
__device__ __forceinline__ void narrow_vocab(const VocabArgs& a, uint32_t block, uint8_t* lds) {
  constexpr int TV = kStanding<EP, P>, SUB = kGroups<P, 1>, MB = 32 * SUB, S = EP / 16;
  constexpr int BV = 32 * TV * 4;
  constexpr int TILE = MB * EP * 2, STAGE = TILE * P;
  constexpr int ALL = MB * EP / 8 * P, CHUNKS = (ALL + kBlock - 1) / kBlock;
  static_assert(ALL % kBlock == 0, "whole chunks");
  typedef Tile<EP> L;
  Streamed<MB>& rows = *reinterpret_cast<Streamed<MB>*>(lds + 2 * STAGE);
  const int lane = lane_id(), wave = wave_id(), half = lane / 32, row = lane % 32;
  const uint32_t z = block % uint32_t(a.splits);
  const int64_t v0 = int64_t(block / uint32_t(a.splits)) * BV + wave * 32 * TV;
  const int live = __builtin_amdgcn_readfirstlane(a.head->live);
  const int m0 = int(z) * a.per, m1 = min(m0 + a.per, live);

  u4 w[TV][P][S];
#pragma unroll
  for (int i = 0; i < TV; ++i) {
    const TW* p = static_cast<const TW*>(a.table) + min(v0 + i * 32 + row, a.vocab - 1) * a.stride;
#pragma unroll
    for (int s = 0; s < S; ++s) {
      const int e = s * 16 + half * 8;
      Eight<TW> q;
      q.load(p + e, a.dim - e);
      u4 t[P];
      terms_of<P>(q, t);
#pragma unroll
      for (int k = 0; k < P; ++k) w[i][k][s] = t[k];
    }
  }
  f16v dw[TV][EP / 32];
#pragma unroll
  for (int i = 0; i < TV; ++i)
#pragma unroll
    for (int e = 0; e < EP / 32; ++e) dw[i][e] = f16v{};

  u4 next[CHUNKS];
  Token token = {0.f, 0.f, 0.f, -1};
  auto fetch = [&](int m) {
#pragma unroll
    for (int i = 0; i < CHUNKS; ++i) {
      const int c = i * kBlock + threadIdx.x, p = c / (MB * EP / 8), q = c % (MB * EP / 8);
      const int r = m + q / (EP / 8);
      next[i] = r < m1 ? *reinterpret_cast<const u4*>(a.x + p * a.x_plane + int64_t(r) * EP + q % (EP / 8) * 8)
                       : u4{0u, 0u, 0u, 0u};
    }
    token = Token{0.f, 0.f, 0.f, -1};
    if (threadIdx.x < MB && m + int(threadIdx.x) < m1) token = a.tokens[m + threadIdx.x];
  };
  auto put = [&](int stage) {
#pragma unroll
    for (int i = 0; i < CHUNKS; ++i) {
      const int c = i * kBlock + threadIdx.x, p = c / (MB * EP / 8), q = c % (MB * EP / 8);
      const int r = q / (EP / 8), k = q % (EP / 8);
      *reinterpret_cast<u4*>(lds + stage * STAGE + p * TILE + r * (EP * 2) + chunk_at<EP>(r, k) * 16) = next[i];
    }
    if (threadIdx.x < MB) {
      rows.tops[stage][threadIdx.x] = -token.top;
      rows.scales[stage][threadIdx.x] = token.inv * token.ratio;
      rows.ratios[stage][threadIdx.x] = token.ratio;
      rows.labels[stage][threadIdx.x] = token.label;
    }
  };
  if (m0 < m1) {
    fetch(m0);
    put(0);
  }
  int cur = 0;
  for (int m = m0; m < m1; m += MB) {
    __syncthreads();
    const bool more = m + MB < m1;
    if (more) fetch(m + MB);
    const uint8_t* st = lds + cur * STAGE;
#pragma unroll
    for (int g = 0; g < SUB; ++g) {
      const int r0 = g * 32;
      f16v d[TV];
#pragma unroll
      for (int i = 0; i < TV; ++i) d[i] = f16v{};
#pragma unroll
      for (int s = 0; s < S; ++s) {
        u4 f[P];
#pragma unroll
        for (int p = 0; p < P; ++p) f[p] = L::rows(st + p * TILE, r0 + row, s, half);
#pragma unroll
        for (int k = 0; k < kPairs<P, 1>; ++k)  // (in narrow_tokens' order: the same scores bit by bit)
#pragma unroll
          for (int i = 0; i < TV; ++i)
            d[i] = mfma(f[second_of<P, 1>(k)], w[i][first_of<P, 1>(k)][s], d[i]);
      }
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const f4 t = *reinterpret_cast<const f4*>(&rows.tops[cur][r0 + q * 8 + half * 4]);
        const f4 c = *reinterpret_cast<const f4*>(&rows.scales[cur][r0 + q * 8 + half * 4]);
#pragma unroll
        for (int i = 0; i < TV; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            d[i][q * 4 + e] = exp2_of(__builtin_fmaf(d[i][q * 4 + e], a.unit, t[e])) * c[e];
      }
      // The labels among the wavefront's rows of the table, one after the other.
      const int64_t off = rows.labels[cur][r0 + row] - v0;
      uint64_t some = __builtin_amdgcn_ballot_w64(half == 0 && off >= 0 && off < 32 * TV);
      const bool labels = some != 0ull;
      while (some != 0ull) {
        const int k = __builtin_ctzll(some);
        some &= some - 1;
        const int at = __builtin_amdgcn_readlane(int(off), k);  // of the table's rows
        const float ratio = rows.ratios[cur][r0 + k];
        const bool mine = row == at % 32 && half == k / 4 % 2;
        const int reg = k / 8 * 4 + k % 4;
#pragma unroll
        for (int i = 0; i < TV; ++i)
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if (mine && i == at / 32 && r == reg) d[i][r] -= ratio;
      }
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        u4 q[TV][PD];
#pragma unroll
        for (int i = 0; i < TV; ++i) d_terms<PD>(d[i], t, q[i]);
#pragma unroll
        for (int e = 0; e < EP / 32; ++e) {
          u4 f[P];
#pragma unroll
          for (int p = 0; p < P; ++p) f[p] = L::turned(st + p * TILE, r0 + t * 16, e * 32, lane);
#pragma unroll
          for (int k = 0; k < kPairs<P, PD>; ++k)
#pragma unroll
            for (int i = 0; i < TV; ++i)
              dw[i][e] = mfma(f[first_of<P, PD>(k)], q[i][second_of<P, PD>(k)], dw[i][e]);
        }
        if (PD == 1 && labels) {  // (as in narrow_tokens)
#pragma unroll
          for (int i = 0; i < TV; ++i) q[i][0] = second_term(d[i], t, q[i][0]);
#pragma unroll
          for (int e = 0; e < EP / 32; ++e) {
            const u4 f = L::turned(st, r0 + t * 16, e * 32, lane);
#pragma unroll
            for (int i = 0; i < TV; ++i) dw[i][e] = mfma(f, q[i][0], dw[i][e]);
          }
        }
      }
    }
    cur ^= 1;
    if (more) put(cur);
  }
  const float f = a.factor != nullptr ? *a.factor : 1.f;
#pragma unroll
  for (int i = 0; i < TV; ++i) {
    const int64_t v = v0 + i * 32 + row;
    if (v >= a.vocab) continue;
    TO* p = static_cast<TO*>(a.dw) + z * a.dw_part + v * a.dw_stride;
#pragma unroll
    for (int e = 0; e < EP / 32; ++e)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int c = e * 32 + q * 8 + half * 4;
        if (c < a.dim)
          store4(p + c, f4{dw[i][e][q * 4] * f, dw[i][e][q * 4 + 1] * f, dw[i][e][q * 4 + 2] * f,
                           dw[i][e][q * 4 + 3] * f});
      }
  }
}

template <int EP, int P, int WM>
constexpr int kTokenLds = 2 * 32 * (4 / WM) * kGroups<P, 4 / WM> * EP * 2 * P;
template <int EP, int P>
constexpr int kVocabLds = 2 * 32 * kGroups<P, 1> * EP * 2 * P + int(sizeof(Streamed<32 * kGroups<P, 1>>));

template <int EP, int P, int WM, class TW>
__global__ __launch_bounds__(kBlock, 2) void narrow_scores(TokenArgs a) {
  extern __shared__ __align__(16) uint8_t lds[];
  narrow_tokens<EP, P, 1, WM, false, TW>(a, blockIdx.x, lds);
}

// Both gradients, of which either may have no blocks: neither needs the other, and one launch leaves no
// compute unit idle between them.  Blocks from `turn` on are of the second kind; dx is the first kind if
// `dx_first`.  With PD == 1 D has two terms where at most `few` rows count.
template <int EP, int P, int PD, int WM, class TW, class TO>
__global__ __launch_bounds__(kBlock, 2) void narrow_gradients(TokenArgs t, VocabArgs v, uint32_t first,
                                                              uint64_t turn, bool dx_first, int32_t few) {
  extern __shared__ __align__(16) uint8_t lds[];
  const uint64_t block = uint64_t(first) + blockIdx.x;
  const bool second = block >= turn;
  const uint32_t at = uint32_t(second ? block - turn : block);
  auto run = [&](auto terms) {
    if (second != dx_first)
      narrow_tokens<EP, P, terms.value, WM, true, TW>(t, at, lds);
    else
      narrow_vocab<EP, P, terms.value, TW, TO>(v, at, lds);
  };
  if constexpr (PD == 1) {
    if (__builtin_amdgcn_readfirstlane(t.head->live) <= few) return run(std::integral_constant<int, 2>());
  }
  run(std::integral_constant<int, PD>());
}

int64_t up(int64_t a, int64_t b) { return (a + b - 1) / b; }

TokenArgs token_args(const NarrowArgs& n) {
  return {n.table, n.table_stride, n.n.vocab, n.n.dim, static_cast<const __bf16*>(n.x), n.x_plane,
          static_cast<const Head*>(n.head), static_cast<const Token*>(n.tokens), n.target, n.unit,
          static_cast<float2*>(n.sums), n.dx_parts, n.n.rows, n.n.splits, n.n.per};
}
VocabArgs vocab_args(const NarrowArgs& n) {
  return {n.table, n.table_stride, n.n.vocab, n.n.dim, static_cast<const __bf16*>(n.x), n.x_plane,
          static_cast<const Head*>(n.head), static_cast<const Token*>(n.tokens), n.unit, n.dw, n.dw_stride,
          n.n.vocab * n.n.dim, n.dw_factor, n.n.dw_splits, n.n.dw_per};
}

template <class K>
void allow_lds(K kernel, int lds) {
  if (lds > 65536)
    (void)hipFuncSetAttribute(reinterpret_cast<const void*>(kernel),
                              hipFuncAttributeMaxDynamicSharedMemorySize, lds);
}

template <int EP, int P, int WM, class TW>
void launch_sums(const NarrowArgs& n, hipStream_t st) {
  auto kernel = narrow_scores<EP, P, WM, TW>;
  constexpr int lds = kTokenLds<EP, P, WM>;
  allow_lds(kernel, lds);
  hipLaunchKernelGGL(kernel, dim3(unsigned(up(n.n.rows, n.n.bm) * n.n.splits)), dim3(kBlock), lds, st,
                     token_args(n));
}

template <int EP, int P, int PD, int WM, class TW, class TO>
void launch_both(const NarrowArgs& n, hipStream_t st) {
  auto kernel = narrow_gradients<EP, P, PD, WM, TW, TO>;
  constexpr int lds = kTokenLds<EP, P, WM> > kVocabLds<EP, P> ? kTokenLds<EP, P, WM> : kVocabLds<EP, P>;
  static_assert(lds <= 160 * 1024, "LDS");
  allow_lds(kernel, lds);
  constexpr int BV = 32 * kStanding<EP, P> * 4;
  const int64_t nx = n.dx_parts != nullptr ? up(n.n.rows, n.n.bm) * n.n.splits : 0;
  const int64_t nw = n.dw != nullptr ? up(n.n.vocab, BV) * n.n.dw_splits : 0;
  // The longer blocks first.
  const bool dx_first = int64_t(n.n.per) * n.n.bm > int64_t(n.n.dw_per) * BV;
  for_launches(nx + nw, kBlock, [&](uint32_t first, dim3 grid) {
    hipLaunchKernelGGL(kernel, grid, dim3(kBlock), lds, st, token_args(n), vocab_args(n), first,
                       uint64_t(dx_first ? nx : nw), dx_first, n.few);
  });
}

// Calls fn(WM).
template <int EP, int P, class Fn>
void for_rows(const NarrowArgs& n, Fn fn) {
  constexpr int TM = kStanding<EP, P>;
  if constexpr (P == 1) {
    if (n.n.bm == 32 * TM) return fn(std::integral_constant<int, 1>());
  }
  if (n.n.bm == 64 * TM)
    fn(std::integral_constant<int, 2>());
  else
    fn(std::integral_constant<int, 4>());
}

// Calls fn(EP, P, PD, the table's type).
template <class Fn>
void for_kind(const NarrowArgs& a, Fn fn) {
  auto width = [&](auto P, auto PD, auto w) {
    if (a.n.dim <= 64)
      fn(std::integral_constant<int, 64>(), P, PD, w);
    else
      fn(std::integral_constant<int, 128>(), P, PD, w);
  };
  const std::integral_constant<int, 1> one;
  const std::integral_constant<int, 2> two;
  const std::integral_constant<int, 3> three;
  if (a.terms == 3) {
    if (a.table_bf16)
      width(three, three, __bf16());
    else
      width(three, three, float());
  } else if (a.terms == 2) {
    width(one, two, __bf16());
  } else {
    width(one, one, __bf16());
  }
}

}  // namespace

Narrow narrow_plan(int32_t rows, int64_t vocab, int32_t dim, bool f32) {
  Narrow n = {};
  n.rows = rows, n.dim = dim, n.vocab = vocab;
  // Few rows: wavefronts share them and take different rows of the table.
  const int each = 32 * standing(dim, f32);
  int wm = f32 ? 2 : 1;
  while (wm < 4 && wm * each < rows) wm *= 2;
  n.bm = wm * each;
  const int wv = 4 / wm, vb = 32 * wv * groups(wv, f32);
  n.parts = wv;
  // Two blocks per compute unit, of at least 2 tiles of the table.
  const int64_t blocks = up(rows > 0 ? rows : 1, n.bm), tiles = up(vocab, vb);
  int64_t splits = 2 * kNumCu / blocks;
  if (splits > tiles / 2) splits = tiles / 2;
  if (splits < 1) splits = 1;
  while (up(tiles, splits) * vb > (int64_t(1) << 30)) ++splits;  // (ranges fit 31 bits)
  n.per = int32_t(up(tiles, splits) * vb);
  n.splits = int32_t(up(vocab, n.per));
  const int mb = 32 * groups(1, f32), bv = 4 * each;
  const int64_t vblocks = up(vocab, bv), steps = up(rows > 0 ? rows : 1, mb);
  int64_t ds = 2 * kNumCu / vblocks;
  if (ds > steps / 2) ds = steps / 2;
  if (ds < 1) ds = 1;
  n.dw_per = int32_t(up(steps, ds) * mb);
  n.dw_splits = int32_t(up(rows > 0 ? rows : 1, n.dw_per));
  return n;
}

hipError_t launch_narrow_scores(const NarrowArgs& n, hipStream_t st) {
  if (n.n.rows > 0)
    for_kind(n, [&](auto EP, auto P, auto, auto w) {
      for_rows<EP.value, P.value>(n, [&](auto WM) {
        launch_sums<EP.value, P.value, WM.value, decltype(w)>(n, st);
      });
    });
  return hipGetLastError();
}

hipError_t launch_narrow_gradients(const NarrowArgs& n, hipStream_t st) {
  for_kind(n, [&](auto EP, auto P, auto PD, auto w) {
    for_rows<EP.value, P.value>(n, [&](auto WM) {
      using TW = decltype(w);
      if constexpr (sizeof(TW) == 2) {
        if (n.dw_bf16) return launch_both<EP.value, P.value, PD.value, WM.value, TW, __bf16>(n, st);
      }
      launch_both<EP.value, P.value, PD.value, WM.value, TW, float>(n, st);
    });
  });
  return hipGetLastError();
}

}  // namespace embbag
