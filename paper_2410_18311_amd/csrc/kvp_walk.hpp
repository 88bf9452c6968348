// Sixteen rows of a head over a cache in pages (kvp_attend.hpp) by a workgroup of four waves: the whole work of few rows, and in prompts that of rows
// whose values were not all finite.
//
// A wave takes every fourth step of 32 slots with a running maximum of its own.  It reads keys and values as they lie, 16 bytes a lane, a step
// ahead, without the LDS, which would only add a wait: nobody else of the workgroup reads them.  A lane's channels of eight slots are
// turned into operands of one channel by one permutation a word.
//
// AGAIN: for rows whose sums came out infinite or NaN.  The products multiply what a row does not see by 0, and 0 times infinity is NaN, so this
// time infinite values and NaN count as 0 in them; where 32 slots hold some, three products more, of zeros and ones, say which rows see which:
// +infinity, -infinity, NaN, which is both, and any of them behind a logit of -infinity, which is NaN too.  4096 tokens of 32 heads, 128 channels, with an
// infinite value among the first: 1.0 ms, where finite values take 0.17; row by row and slot by slot, without products, it had been 179 ms.
#pragma once

#include "kvp_attend.hpp"

namespace ci {
namespace {

// What a lane holds of 32 slots: of keys the row n of both halves, a quarter (g) of each 64 bytes; of values the channels CH n .. of the slots
// 4 g .. + 3 of both halves.
template <class E, int D>
struct Step32 {
  static constexpr int K = D * E::BYTES / 64, CH = D / 16, V = CH * E::BYTES / 4;   // vectors of keys; channels and words of values
  uint4 k[2][K];
  uint32_t v[8][V];
  int page[2];   // of the halves
};

template <int WORDS>
__device__ __forceinline__ void ld_words(const void* p, uint32_t (&to)[WORDS]) {
  if constexpr (WORDS == 2) {
    const uint2 u = *reinterpret_cast<const uint2*>(p);
    to[0] = u.x, to[1] = u.y;
  } else {
#pragma unroll
    for (int i = 0; i < WORDS; i += 4) {
      const uint4 u = ld16(reinterpret_cast<const uint32_t*>(p) + i);
      to[i] = u.x, to[i + 1] = u.y, to[i + 2] = u.z, to[i + 3] = u.w;
    }
  }
}

// A row of q as the operand that goes with the keys' vectors.
template <class E, int D>
__device__ __forceinline__ void load_query(const KvpAttend& a, const Sentence& s, int h, int r, uint4 (&q)[Step32<E, D>::K]) {
  const int g = (threadIdx.x & 63) >> 4, i = r / a.G;
  const typename E::T* src = reinterpret_cast<const typename E::T*>(a.q) + (int64_t)(s.first + i) * a.q_t +
                             (int64_t)(h * a.G + r - i * a.G) * a.q_h + g * E::VEC;
#pragma unroll
  for (int j = 0; j < Step32<E, D>::K; ++j) {
    if (a.q_vectors) {
      q[j] = ld16(src + 4 * j * E::VEC);
    } else {
      typename E::T x[E::VEC];
#pragma unroll
      for (int e = 0; e < E::VEC; ++e) x[e] = src[4 * j * E::VEC + e];
      __builtin_memcpy(&q[j], x, sizeof(x));
    }
  }
}

template <int D>
struct RowsLds {
  float ml[2][4][16];
  __attribute__((aligned(16))) float sums[4][16][D + 4];
  unsigned broken;   // rows, a bit each
};

// Channels of a lane's sums that are not finite, a bit each: c * 4 + r.
struct Marks {
  uint32_t up, down, nan;
};

// Where infinities and NaN are among a word's one or two values: a 1 in the lowest bit of each.
template <class E>
struct NotFinite {
  static constexpr uint32_t kOnes = E::BYTES == 2 ? 0x00010001u : 1u, kSign = 8 * E::BYTES - 1, kMantissa = __is_same(E, F16) ? 10 : __is_same(E, BF16) ? 7 : 23;
  static constexpr uint32_t kLow = kOnes << kMantissa, kFraction = kLow - kOnes, kExponent = (kOnes << kSign) - kLow;
  uint32_t any, nan, negative;
  __device__ explicit NotFinite(uint32_t w)
      : any(((w & kExponent) + kLow) >> kSign & kOnes),   // an exponent of ones only is carried into the sign's place
        nan(((w & kFraction) + kFraction) >> kMantissa & any), negative(w >> kSign & kOnes) {}
  // 0: towards -infinity, ~0: towards +infinity
  __device__ uint32_t towards(uint32_t up) const { return any & (nan | (negative ^ up)); }
};

// 32 slots' values whose infinities and NaN are taken out, and marked for the rows that see them.  seen, below: which of the lane's eight slots its row n
// sees, and which of those at a logit of -infinity, a bit each.
template <class E, int D>
__device__ __forceinline__ void take_out(Step32<E, D>& x, unsigned seen, unsigned below, Marks& marks) {
  constexpr int CH = Step32<E, D>::CH, W = Step32<E, D>::V;
  constexpr uint32_t one = __is_same(E, F16) ? 0x3c00u : __is_same(E, BF16) ? 0x3f80u : 0x3f800000u;
  uint32_t any = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int w = 0; w < W; ++w) any |= NotFinite<E>(x.v[i][w]).any;
  if (!__any(any != 0)) return;
#pragma unroll 1
  for (int kind = 0; kind < 3; ++kind) {   // +infinity, -infinity, either behind a logit of -infinity
    const uint32_t rows = kind == 2 ? below : seen, up = kind == 0 ? ~0u : 0u, either = kind == 2 ? ~0u : 0u;
    auto counts = [&](uint32_t w) {
      const NotFinite<E> x(w);
      return x.towards(up) | (x.any & either);
    };
    uint32_t mark = 0;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      f32x4 hits = {0.0f, 0.0f, 0.0f, 0.0f};
      __builtin_amdgcn_sched_barrier(0);   // channel by channel, anew for each kind, so that no registers hold what is made of the words
#pragma unroll
      for (int i = 0; i < 8; ++i) asm("" : "+v"(x.v[i][c * E::BYTES / 4]));
      if constexpr (E::BYTES == 2) {
        uint32_t v[4], r[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t first = counts(x.v[2 * i][c / 2]), second = counts(x.v[2 * i + 1][c / 2]);
          v[i] = ((first >> (16 * (c % 2)) & 1) | (second >> (16 * (c % 2)) & 1) << 16) * one;
          r[i] = ((rows >> (2 * i) & 1) | (rows >> (2 * i + 1) & 1) << 16) * one;
        }
        hits = product16<E>(make_uint4(v[0], v[1], v[2], v[3]), make_uint4(r[0], r[1], r[2], r[3]), hits);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) hits = product16_f32(u2f(counts(x.v[i][c]) * one), u2f((rows >> i & 1) * one), hits);
      }
#pragma unroll
      for (int r = 0; r < 4; ++r) mark |= (0u - f2u(hits[r])) >> 31 << (4 * c + r);   // hits above 0
      asm("" : "+v"(mark));
    }
    marks.up |= kind == 0 ? mark : 0u;
    marks.down |= kind == 1 ? mark : 0u;
    marks.nan |= kind == 2 ? mark : 0u;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int w = 0; w < W; ++w) {
      __builtin_amdgcn_sched_barrier(0);
      asm("" : "+v"(x.v[i][w]));
      x.v[i][w] &= ~(NotFinite<E>(x.v[i][w]).any * (E::BYTES == 2 ? 0xffffu : ~0u));
      asm("" : "+v"(x.v[i][w]));
    }
}

// The 16 rows from row0 on (past the last, R, repeated) of a head over the steps begin .. end - 1, whose slots `slot` says.
// store(r, d, m, l, v): four channels of row r, sums of weights 2^(logit - m) with values and alone; called for AGAIN for the rows in `only`.  Without
// AGAIN the rows are returned (a bit each) whose sums are not finite while their weights' is.
template <class E, int D, bool AGAIN, class Slot, class Store>
__device__ __forceinline__ unsigned sixteen_rows(const KvpAttend& a, const Sentence& s, const Pages& pages, int h, int row0, int R, Slot slot, int begin,
                                                 int end, unsigned only, RowsLds<D>& lds, Store store) {
  using S32 = Step32<E, D>;
  constexpr int K = S32::K, CH = S32::CH, VW = S32::V;
  auto& ml = lds.ml;
  auto& sums = lds.sums;
  if constexpr (AGAIN) asm volatile("" : "+s"(row0));   // nothing of the first time is kept in registers for this one
  const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int inside = (1 << a.c.shift) - 1;
  const int row = min(row0 + n, R - 1);
  const int p = s.slot + row / a.G;
  const int p_low = s.slot + row0 / a.G, p_high = s.slot + min(row0 + 15, R - 1) / a.G;   // of all

  uint4 q[K];
  load_query<E, D>(a, s, h, row, q);
  [[maybe_unused]] Marks marks = {0, 0, 0};

  S32 x;
  auto find_pages = [&](int step) {
    const int t = slot(min(step, end - 1));
#pragma unroll
    for (int i = 0; i < 2; ++i) x.page[i] = pages.of(a, t + 16 * i);
  };
  auto load_keys = [&](int step, const int (&page)[2]) {
    const int t = slot(step);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int at = min(t + 16 * i + n, pages.last) & inside;
      const typename E::T* src = reinterpret_cast<const typename E::T*>(a.c.k) + page_start<D>(a, page[i], h) + at * D + g * E::VEC;
#pragma unroll
      for (int j = 0; j < K; ++j) x.k[i][j] = ld16(src + 4 * j * E::VEC);
    }
  };
  auto load_values = [&](int step, const int (&page)[2]) {
    const int t = slot(step);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const typename E::T* src = reinterpret_cast<const typename E::T*>(a.c.v) + page_start<D>(a, page[i], h) + n * CH;
#pragma unroll
      for (int r = 0; r < 4; ++r) ld_words<VW>(src + (min(t + 16 * i + 4 * g + r, pages.last) & inside) * D, x.v[4 * i + r]);
    }
  };

  float m = -INFINITY, l = 0.0f;   // l: of the lane's own slots
  f32x4 acc[CH];
#pragma unroll
  for (int c = 0; c < CH; ++c) acc[c] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

  int step = begin + wave;
  if (step < end) {
    find_pages(step);
    int page[2] = {x.page[0], x.page[1]};
    if constexpr (!AGAIN) {
      load_keys(step, page);
      load_values(step, page);
      find_pages(step + 4);
    }
    for (; step < end; step += 4) {
      if constexpr (AGAIN) {   // nothing ahead: registers that the first time does without are not asked for
        find_pages(step);
        page[0] = x.page[0];
        page[1] = x.page[1];
        load_keys(step, page);
      }
      const int t = slot(step);
      const int next[2] = {x.page[0], x.page[1]};
      const bool more = !AGAIN && step + 4 < end;
      f32x4 z[2] = {{0.0f, 0.0f, 0.0f, 0.0f}, {0.0f, 0.0f, 0.0f, 0.0f}};
#pragma unroll
      for (int j = 0; j < K; ++j)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          if constexpr (E::BYTES == 2) {
            z[i] = product16<E>(x.k[i][j], q[j], z[i]);
          } else {
            float kf[4], qf[4];
            unpack<F32>(x.k[i][j], kf);
            unpack<F32>(q[j], qf);
#pragma unroll
            for (int c = 0; c < 4; ++c) z[i] = product16_f32(kf[c], qf[c], z[i]);
          }
        }
      if (more) load_keys(step + 4, next);
      [[maybe_unused]] unsigned seen_slots = 0, below = 0;
      const bool masked = AGAIN || page[0] < 0 || page[1] < 0 || t + 31 > p_low || (a.window && t <= p_high - a.window && t + 31 >= a.sinks);
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          z[i][r] *= a.scale;
          if (masked) {
            const bool seen = (page[i] >= 0) & sees(a, p, t + 16 * i + 4 * g + r);
            z[i][r] = seen ? z[i][r] : -INFINITY;
            if constexpr (AGAIN) {
              seen_slots |= seen ? 1u << (4 * i + r) : 0u;
              below |= z[i][r] == -INFINITY ? 1u << (4 * i + r) : 0u;
            }
          }
        }
      if constexpr (AGAIN) {
        load_values(step, page);
        take_out<E, D>(x, seen_slots, below & seen_slots, marks);
      }
      float top = fmaxf(fmaxf(fmaxf(z[0][0], z[0][1]), fmaxf(z[0][2], z[0][3])), fmaxf(fmaxf(z[1][0], z[1][1]), fmaxf(z[1][2], z[1][3])));
      // m is raised only when a logit passes it by kRaise; the sums hold that range in fp32, unless the values are next to its largest.
      if (__any(top > m + (AGAIN ? kBelow<E> : kRaise<E>))) {
        top = fmaxf(top, __shfl_xor(top, 16, kWave));
        top = fmaxf(top, __shfl_xor(top, 32, kWave));
        const float raised = fmaxf(m, top - kBelow<E>), was = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m - raised);
        m = raised;
        l *= was;
#pragma unroll
        for (int c = 0; c < CH; ++c) acc[c] *= was;
      }
      const float ref = m == -INFINITY ? 0.0f : m;
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          z[i][r] = __builtin_amdgcn_exp2f(z[i][r] - ref);
          l += z[i][r];
        }
      if constexpr (E::BYTES == 2) {
        uint4 high, low;
        two_pieces<E>(z[0][0], z[0][1], &high.x, &low.x);
        two_pieces<E>(z[0][2], z[0][3], &high.y, &low.y);
        two_pieces<E>(z[1][0], z[1][1], &high.z, &low.z);
        two_pieces<E>(z[1][2], z[1][3], &high.w, &low.w);
#pragma unroll
        for (int c = 0; c < CH; ++c) {
          const uint32_t half = c % 2 ? 0x07060302u : 0x05040100u;
          const uint4 e = make_uint4(__builtin_amdgcn_perm(x.v[1][c / 2], x.v[0][c / 2], half), __builtin_amdgcn_perm(x.v[3][c / 2], x.v[2][c / 2], half),
                                     __builtin_amdgcn_perm(x.v[5][c / 2], x.v[4][c / 2], half), __builtin_amdgcn_perm(x.v[7][c / 2], x.v[6][c / 2], half));
          acc[c] = product16<E>(e, high, acc[c]);
          acc[c] = product16<E>(e, low, acc[c]);
        }
      } else {
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
          for (int i = 0; i < 8; ++i) acc[c] = product16_f32(u2f(x.v[i][c]), z[i / 4][i % 4], acc[c]);
      }
      if (more) {
        load_values(step + 4, next);
        page[0] = next[0];
        page[1] = next[1];
        find_pages(step + 8);
        // else the compiler puts these requests and the first step's together at the loop's head, where the first products wait for the keys
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  }

  // the four waves' sums against their common maximum; a lane's slots are a quarter of its row's
  l += __shfl_xor(l, 16, kWave);
  l += __shfl_xor(l, 32, kWave);
  if (g == 0) {
    ml[0][wave][n] = m;
    ml[1][wave][n] = l;
  }
  __syncthreads();
  if (!AGAIN && threadIdx.x == 0) lds.broken = 0;   // everybody has read the last call's
  float top = ml[0][0][n];
#pragma unroll
  for (int w = 1; w < 4; ++w) top = fmaxf(top, ml[0][w][n]);
  const float own = m == -INFINITY ? (l != 0.0f ? NAN : 0.0f) : __builtin_amdgcn_exp2f(m - top);
#pragma unroll
  for (int c = 0; c < CH; ++c)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      acc[c][r] *= own;
      if constexpr (AGAIN) {
        const uint32_t bit = 1u << (4 * c + r);
        if (marks.up & bit) acc[c][r] = INFINITY;
        if (marks.down & bit) acc[c][r] = marks.up & bit ? NAN : -INFINITY;
        if (marks.nan & bit) acc[c][r] = NAN;
      }
    }
  if (row0 + n < R) {
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int c = 0; c < CH; c += 4)
        *reinterpret_cast<float4*>(&sums[wave][n][CH * (4 * g + r) + c]) = make_float4(acc[c][r], acc[c + 1][r], acc[c + 2][r], acc[c + 3][r]);
  }
  __syncthreads();

  const int live = min(16, R - row0);
  for (int e = threadIdx.x; e < live * (D / 4); e += 256) {
    const int r = e / (D / 4), d = e % (D / 4) * 4;
    float t = -INFINITY, total = 0.0f, v[4];
#pragma unroll
    for (int w = 0; w < 4; ++w) t = fmaxf(t, ml[0][w][r]);
#pragma unroll
    for (int w = 0; w < 4; ++w)
      total += ml[0][w][r] == -INFINITY ? ml[1][w][r] : ml[1][w][r] * __builtin_amdgcn_exp2f(ml[0][w][r] - t);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = (sums[0][r][d + i] + sums[1][r][d + i]) + (sums[2][r][d + i] + sums[3][r][d + i]);
    if constexpr (!AGAIN) {
      // a logit of +infinity or NaN makes the row's sum NaN, and with it the row: nothing of it is to be done again
      if (total == total && !(finite(v[0]) && finite(v[1]) && finite(v[2]) && finite(v[3]))) atomicOr(&lds.broken, 1u << r);
    }
    if (!AGAIN || (only >> r & 1)) store(r, d, t, total, v);
  }
  __syncthreads();
  return AGAIN ? 0 : __builtin_amdgcn_readfirstlane(lds.broken);
}

}  // namespace
}  // namespace ci
