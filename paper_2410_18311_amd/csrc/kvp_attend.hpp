// Attention of packed rows over a cache in pages (ci_kvp in coreinfer.h): out = softmax(scale q k^T) v over the slots t <= p, with a window
// those of t > p - window or t < sinks, in one pass with a running maximum and sum.
//
// Logits come out of the matrix cores with slots down and rows across, so that a lane holds one row's: its maximum and sum need two exchanges,
// its sums of values one factor, and its probabilities enter the product with the values as they lie.
#pragma once

#include <math.h>

#include "kvp.hpp"

namespace ci {

constexpr int kMaxPieces = 64;   // of a sentence's slots: the lanes of the join keep a factor of each

struct KvpAttend {
  Kvp c;
  const void* q;
  int64_t q_t, q_h;   // strides in elements
  void* out;
  float* lse;
  const int32_t *first, *lens;
  int T, G, max_rows, max_len, window, sinks;   // window 0: none
  float scale;                                  // of the logits, with log2(e)
  int q_vectors;
  // Few rows: `row_tiles` tiles of 16 rows a head (what more rows a sentence has, others do); the slots of all sentences in `wanted` pieces
  // and one more a head, none below `least` steps; wanted 0: one piece a head.
  int few, row_tiles, blocks, wanted, least, join_rows;   // join_rows: packed rows of such a sentence at most
  int2* place;        // [B]: a sentence's first piece and how many a head has
  float *m, *l, *o;   // [blocks, row_tiles 16] twice and [.., D]
  // Prompts: `tiles` tiles of tile_rows rows at most, the steps of each in `pieces`.
  int tiles, tile_rows, pieces;
  float *tile_m, *tile_l, *tile_exact, *tile_o;   // [tiles H, pieces, tile_rows] three times (the third for lse) and [.., D]
};

// rows, tiles: which of the kernels
template <class E> int launch_kvp_attend_type(const KvpAttend& a, int D, bool rows, bool tiles, hipStream_t s);

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

template <class E>
__device__ __forceinline__ f32x4 product16(const uint4& a, const uint4& b, const f32x4& c) {
  if constexpr (E::BYTES == 4) return c;
  else if constexpr (__is_same(E, F16))
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 product16_f32(float a, float b, const f32x4& c) {
  return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
}

// Two numbers rounded to E (one instruction), and what that leaves of them.
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
template <class E>
__device__ __forceinline__ uint32_t pair_of(float x, float y) {
  const f32x2 v = {x, y};
  if constexpr (__is_same(E, F16))
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, half2_t));
  else
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
}
template <class E>
__device__ __forceinline__ f32x2 both_of(uint32_t u) {
  if constexpr (__is_same(E, F16)) return __builtin_convertvector(__builtin_bit_cast(half2_t, u), f32x2);
  else return f32x2{u2f(u << 16), u2f(u & 0xffff0000u)};
}
template <class E>
__device__ __forceinline__ void two_pieces(float x, float y, uint32_t* high, uint32_t* low) {
  *high = pair_of<E>(x, y);
  const f32x2 t = both_of<E>(*high);
  *low = pair_of<E>(x - t[0], y - t[1]);
}

// A row's running reference m is below the largest logit so far by this to begin with, and follows it when one passes m by kRaise: weights of up to
// 2^15 are numbers of every type, and in fp16, whose smallest step is 2^-24, those of 2^-31 of the largest still count when there are very many.
template <class E> constexpr float kBelow = __is_same(E, F16) ? 7.0f : 0.0f;
template <class E> constexpr float kRaise = kBelow<E> + 8.0f;

__device__ __forceinline__ bool finite(float x) { return fabsf(x) < INFINITY; }   // false for NaN
// The factor of a sum of weighted values that brings it to another maximum.  Weights are above 0, however small next to others: where fp32 has 0 for
// the factor, an infinite sum stays infinite.
__device__ __forceinline__ float factor_of(float sum, float factor) { return factor == 0.0f && !finite(sum) ? 1.0f : factor; }

// A sentence's rows: they begin at packed row `first`, `rows` of them are this call's, the first in slot `slot` (negative: ahead of the
// first slot, where it sees nothing).
struct Sentence {
  int first, rows, len, slot;
};
__device__ __forceinline__ Sentence sentence(const KvpAttend& a, int b) {
  const int from = clamp_row(a.first[b], a.T), n = max(clamp_row(a.first[b + 1], a.T) - from, 0);
  const int len = min(max(a.lens[b], 0), a.max_len);
  return Sentence{from, min(n, a.max_rows), len, len - n};
}

// The same in scalar registers, for a sentence that all lanes share.
__device__ __forceinline__ Sentence uniform(const Sentence& s) {
  return Sentence{__builtin_amdgcn_readfirstlane(s.first), __builtin_amdgcn_readfirstlane(s.rows), __builtin_amdgcn_readfirstlane(s.len),
                  __builtin_amdgcn_readfirstlane(s.slot)};
}

// Steps of STEP slots that rows in slots p0 .. p1 see something of: `sinks` of them from the first slot on, then those from `window` on.
template <int STEP>
struct Steps {
  int sinks, window, total;
  __device__ Steps(const KvpAttend& a, int p0, int p1, int len) {
    const int high = min(len, p1 + 1), low = a.window ? max(0, p0 - a.window + 1) : 0;
    window = low / STEP;
    sinks = min((min(a.sinks, low) + STEP - 1) / STEP, window);
    total = high <= 0 ? 0 : sinks + max(0, (high + STEP - 1) / STEP - window);
  }
  __device__ int slot(int step) const { return (step < sinks ? step : window + step - sinks) * STEP; }
};

// Without a branch for each of a lane's logits.
__device__ __forceinline__ bool sees(const KvpAttend& a, int p, int t) {
  return (t <= p) & ((a.window == 0) | (t > p - a.window) | (t < a.sinks));
}

// A sentence's pages.  Slots from the last one in use on read that one, which is as finite as the rest.
struct Pages {
  const __attribute__((address_space(4))) int32_t* table;   // constant: a uniform slot's entry comes by a scalar load
  int last;
  __device__ Pages(const KvpAttend& a, int b, int len)
      : table((const __attribute__((address_space(4))) int32_t*)(uintptr_t)(a.c.table + (int64_t)b * a.c.most)), last(max(len - 1, 0)) {}
  // Page of a slot; -1: none.
  __device__ int of(const KvpAttend& a, int slot) const {
    const int n = table[min(slot, last) >> a.c.shift];
    return (uint32_t)n < a.c.pages ? n : -1;   // pages below 2^31
  }
};
// What a row in slot p gives that has no weights: 0 if it sees no slot, as none of its pages is one, else NaN, its logits being all -infinity.
__device__ __forceinline__ float without_weights(const KvpAttend& a, const Pages& pages, int p) {
  const int low = a.window ? max(0, p - a.window + 1) : 0;
  bool any = false;
  auto look = [&](int from, int to) {   // pages from .. to, eight requests at once
    for (int n = from; n <= to && !any; n += 8)
#pragma unroll
      for (int j = 0; j < 8; ++j) any |= (uint32_t)pages.table[min(n + j, to)] < a.c.pages;
  };
  if (p >= 0) {
    look(low >> a.c.shift, p >> a.c.shift);
    look(0, (min(a.sinks, low) - 1) >> a.c.shift);
  }
  return any ? NAN : 0.0f;
}

__device__ __forceinline__ bool rarely(bool x) { return __builtin_expect(x, false); }

// Elements from the pages' start to the first slot of a head in a page; page -1: of page 0, whatever lies there.
template <int D>
__device__ __forceinline__ int64_t page_start(const KvpAttend& a, int page, int h) {
  return (((int64_t)max(page, 0) * a.c.H + h) << a.c.shift) * D;
}

template <class E>
__device__ __forceinline__ void store_row4(const KvpAttend& a, int D, int64_t at, int d, const float (&v)[4]) {
  typename E::T* dst = reinterpret_cast<typename E::T*>(a.out) + at * D + d;
  if constexpr (E::VEC == 4)
    *reinterpret_cast<float4*>(dst) = make_float4(v[0], v[1], v[2], v[3]);
  else
    *reinterpret_cast<uint2*>(dst) = make_uint2(pair_of<E>(v[0], v[1]), pair_of<E>(v[2], v[3]));
}
__device__ __forceinline__ void store_lse(const KvpAttend& a, int64_t at, float m, float l) {
  // a maximum of infinity beside no weights is a logit beyond fp32
  if (a.lse) a.lse[at] = l == 0.0f && m != INFINITY ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * 0.69314718055994531f;
}
// Workgroups for that many pieces of work; beyond, one takes several.
inline unsigned join_blocks(int64_t n) { return (unsigned)(n < 262144 ? n : 262144); }

// Packed row and head of row r of head h of the cache, as a row of out.
__device__ __forceinline__ int64_t out_row(const KvpAttend& a, const Sentence& s, int h, int r) {
  const int i = r / a.G;
  return ((int64_t)s.first + i) * a.c.H * a.G + h * a.G + (r - i * a.G);
}

}  // namespace
}  // namespace ci
