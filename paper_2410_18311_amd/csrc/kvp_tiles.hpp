// Attention of prompts over a cache in pages (kvp_attend.hpp), 16-bit types: bound by the matrix cores and the vector instructions between products.
//
// A workgroup takes a tile of 128 rows of a head, 32 to a wave, and steps of 64 slots, which go from the pages straight into the LDS, a step ahead.  Products
// of 32 x 32: the logits of 32 rows come out with a row's 32 slots in two lanes, and the values are read from the LDS transposed, four slots of a
// channel to a lane, in the order in which the probabilities lie, so that nothing is exchanged between lanes but a new maximum.  Two workgroups
// of 128 channels, three of 64, share a compute unit: one's softmax runs beside the other's products.
//
// Weights are rounded to the cache's type, as the matrix cores take it: half a unit of a weight, averaged over the slots.  Their sum is that
// of the rounded ones, so that a row's weights add up to 1; the log-sum, when asked for, is of the exact ones.
//
// 4096 tokens of 32 heads of 128, fp16, causal: 152 to 160 us (the first forty calls of a run up to 203, as the clock is regulated), 0.86 to 0.9 PFLOP/s of the visible half,
// where a large product of the library reaches 1.17 to 1.2.  The LDS's reads are as high a bound as the products: 32 KB a wave and step, 2048 cycles for a
// compute unit's eight waves, whose products take as many.  The matrix
// cores are busy for 44 % of the cycles and vector instructions (4.5 a logit, one of them an exponential) take most of the others; the two
// overlap little: of 32 products in 1030 cycles, reading their operands from the LDS makes 1290 and the next step's loads 1540.
// Also measured, the same case: 256 rows in eight waves, whose halves take turns at products and softmax, 161 us; 64 rows a wave, one wave a SIMD,
// 225; steps of 32 slots in a pipeline, 180; operands 6 or 12 products ahead instead of 8, the same; without the waves' raised priority in
// products 154 where it was 149.  64 channels, 777 rows over 8192 slots, 32 heads: 90 us, where products are a third of the time.
#pragma once

#include "gemm_tile.hpp"
#include "kvp_walk.hpp"

namespace ci {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));

template <class E>
__device__ __forceinline__ f32x16 mfma32(const uint4& a, const uint4& b, const f32x16& c) {
  if constexpr (__is_same(E, F16))
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

constexpr int kSchedProduct = 0x8, kSchedLds = 0x100;   // kinds of instructions for the compiler's scheduler: matrix products, reads of the LDS
constexpr int kTileStep = 64;   // slots of a step

// Rows of D channels in the LDS, 16-byte chunk c of row r in the place c ^ swizzle(r), so that what 16 lanes read at once lies in
// different banks.  Keys: the same chunk of 16 rows; values: 64 bytes of four rows.
template <int D>
__device__ __forceinline__ int key_swizzle(int r) { return D == 128 ? r & 15 : r >> 1 & 7; }
template <int D>
__device__ __forceinline__ int value_swizzle(int r) { return (D == 128 ? r & 3 : r >> 1 & 1) << 2; }

// load_to_lds that is no access of memory to the compiler: it writes a buffer that nobody reads before the next meeting of the waves.
__device__ __forceinline__ void load_ahead(uint32_t lds, uint32_t off, i32x4 rsrc) {
  uint32_t m0;
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tbuffer_load_dwordx4 %2, %3, 0 offen lds" : "={m0}"(m0) : "s"(lds), "v"(off), "s"(rsrc));
}
// Two numbers added to a sum.
template <class E>
__device__ __forceinline__ float add_pair(uint32_t u, float sum) {
  if constexpr (__is_same(E, F16))
    return __builtin_amdgcn_fdot2(__builtin_bit_cast(half2_t, u), half2_t{(_Float16)1.0f, (_Float16)1.0f}, sum, false);
  else
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, u), bf16x2{(__bf16)1.0f, (__bf16)1.0f}, sum, false);
}

// Where the tiles of a sentence begin among all: each has at least as many as its rows fill, whatever `rows` of a tile.
__device__ __forceinline__ int64_t tile_start(const KvpAttend& a, int b, int rows) {
  return (int64_t)clamp_row(a.first[b], a.T) * a.G / rows + b;
}
__device__ __forceinline__ int sentence_of_tile(const KvpAttend& a, int tile, int rows) {
  const int lane = threadIdx.x & 63;
  int lo = 0, n = a.c.B;
  while (n > 1) {
    const int step = (n + 63) / 64, at = lane * step;
    const bool before = lane == 0 || (at < n && tile_start(a, lo + at, rows) <= tile);
    const int last = __popcll(__ballot(before)) - 1;
    lo += last * step;
    n = min(step, n - last * step);
  }
  return __builtin_amdgcn_readfirstlane(lo);
}

// Piece `piece` of the steps of a tile of a head.
template <class E, int D, int WAVES, bool LSE>
__device__ __forceinline__ void tile_block(const KvpAttend& a, int block, int piece) {
  constexpr int BM = 32 * WAVES, ROW = 2 * D, HALF = kTileStep * ROW, KK = D / 16, CB = D / 32;
  constexpr int LOADS = HALF / 1024 / WAVES, ROWS = 1024 / ROW;   // loads of a wave and tensor, rows of a load
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];   // two steps' keys and two steps' values, 64 rows each
  __shared__ unsigned broken[WAVES];
  __shared__ int missing[WAVES];   // whether a wave has met slots without a page
  const int lane = threadIdx.x & 63, n = lane & 31, g = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int h = block % a.c.H, tile = a.tiles - 1 - block / a.c.H;   // the last tiles of a prompt see most
  const int b = sentence_of_tile(a, tile, BM);
  const Sentence s = uniform(sentence(a, b));
  const int R = s.rows * a.G;
  const int64_t local = tile - tile_start(a, b, BM);
  if (R <= a.few || local < 0 || local * BM >= R) return;
  const int row0 = __builtin_amdgcn_readfirstlane((int)local) * BM, mine0 = row0 + 32 * wave;   // of the tile, of the wave
  const bool live = mine0 < R;
  const int row = min(mine0 + n, R - 1), p = s.slot + row / a.G;
  const int p_low = s.slot + min(mine0, R - 1) / a.G, p_high = s.slot + min(mine0 + 31, R - 1) / a.G;
  const Steps<kTileStep> steps(a, max(s.slot + row0 / a.G, 0), s.slot + min(row0 + BM - 1, R - 1) / a.G, s.len);
  const int begin = (int)((int64_t)steps.total * piece / a.pieces), end = (int)((int64_t)steps.total * (piece + 1) / a.pieces);
  const Pages pages(a, b, s.len);
  const int inside = (1 << a.c.shift) - 1;

  uint4 q[KK];
  {
    const int i = row / a.G;
    const typename E::T* src = reinterpret_cast<const typename E::T*>(a.q) + (int64_t)(s.first + i) * a.q_t +
                               (int64_t)(h * a.G + row - i * a.G) * a.q_h + 8 * g;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
      if (a.q_vectors) {
        q[kk] = ld16(src + 16 * kk);
      } else {
        typename E::T x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = src[16 * kk + e];
        __builtin_memcpy(&q[kk], x, sizeof(x));
      }
    }
  }

  // A wave fetches LOADS * ROWS neighbouring rows of a step's keys and values, which are of one page; what lies behind the last slot in use comes as
  // zeros.  off: the lane's 16 bytes of a load.
  const int fetch_row = lane / (ROW / 16), fetch_chunk = lane % (ROW / 16), fetch_from = wave * LOADS * ROWS;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) unsigned char*)smem + fetch_from * ROW;
  int key_off[LOADS], value_off[LOADS];
#pragma unroll
  for (int i = 0; i < LOADS; ++i) {
    const int r = i * ROWS + fetch_row;
    key_off[i] = r * ROW + 16 * (fetch_chunk ^ key_swizzle<D>(fetch_from + r));
    value_off[i] = r * ROW + 16 * (fetch_chunk ^ value_swizzle<D>(fetch_from + r));
  }
  auto rows_at = [&](int step, int page, const void* tensor) {
    const int t = steps.slot(step) + fetch_from;
    const int64_t at = page_start<D>(a, page, h) * 2 + (t & inside) * ROW;
    i32x4 r = rsrc_at(reinterpret_cast<const char*>(tensor) + at);
    int rows = max(s.len - t, 0);
    asm("" : "+s"(rows));   // else the two become one vector instruction
    r[2] = min(rows, kTileStep) * ROW;
    return r;
  };
  auto fetch = [&](int step, int page, const void* tensor, int place, bool keys) {
    const i32x4 rsrc = rows_at(step, page, tensor);
#pragma unroll
    for (int i = 0; i < LOADS; ++i) load_ahead(lds0 + place * HALF + i * 1024, keys ? key_off[i] : value_off[i], rsrc);
  };
  auto page_of = [&](int step) { return pages.of(a, steps.slot(min(step, end - 1)) + fetch_from); };
  int page1 = 0, page2 = 0;   // of the step whose values are fetched next, of the one behind it, whose keys are
  if (begin < end) {
    const int page0 = page_of(begin);
    page1 = page_of(begin + 1);
    page2 = page_of(begin + 2);
    fetch(begin, page0, a.c.k, 0, true);
    fetch(begin, page0, a.c.v, 2, false);
    fetch(min(begin + 1, end - 1), page1, a.c.k, 1, true);
    if (lane == 0) missing[wave] = (page0 | page1 | page2) < 0;
  }
  // here, not at their first use in the loop, where the wait would be for the loads of the next step as well
#pragma unroll
  for (int kk = 0; kk < KK; ++kk) asm volatile("" : "+v"(q[kk].x), "+v"(q[kk].y), "+v"(q[kk].z), "+v"(q[kk].w));

  float m = -INFINITY, l = 0.0f, exact = 0.0f;   // m: scaled; sums of the lane's own slots, of the weights as they are multiplied and before
  f32x16 acc[CB], z[2];
  uint4 w[4];   // probabilities of 16 slots each, as operands
#pragma unroll
  for (int c = 0; c < CB; ++c) acc[c] = f32x16{};

  // the lane's places in a step's rows: keys of row n, 16 bytes of the first 16 channels; values of slots 4 g + .., 8 bytes of the first 32 channels.
  // Those of the channels 16 kk or 32 c on differ in bits of their own.
  const int key_at = n * ROW + 16 * (g ^ key_swizzle<D>(n));
  const int value_row = 4 * g + (lane & 15) / 4;
  const int value_at = value_row * ROW + 32 * (lane >> 4 & 1) + 8 * (lane & 3) + 16 * value_swizzle<D>(value_row);
  // 32 slots' keys or 32 channels' values as operands; at: the lane's place in the step's buffer
  auto key_operand = [&](int at, int kk, int i) { return *reinterpret_cast<const uint4*>(smem + (at ^ (32 * kk)) + i * 32 * ROW); };
  auto value_operand = [&](int at, int kb, int c) {
    const unsigned char* from = smem + (at ^ (64 * c)) + 16 * kb * ROW;
    const s16x4 first = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)from);
    const s16x4 second = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(from + 8 * ROW));
    const uint2 x = __builtin_bit_cast(uint2, first), y = __builtin_bit_cast(uint2, second);
    return make_uint4(x.x, x.y, y.x, y.y);
  };
  // the products of 64 slots' keys with the rows, slots down
  auto logits = [&](int buffer) {
    z[0] = z[1] = f32x16{};
#pragma unroll
    for (int kk = 0; kk < KK; ++kk)
#pragma unroll
      for (int i = 0; i < 2; ++i) z[i] = mfma32<E>(key_operand(key_at + buffer * HALF, kk, i), q[kk], z[i]);
  };
  // The logits as weights of the products with the values.  any: some slot has no page.
  // load(i), i = 0 .. 3: what else is to be done on the way.
  auto weights = [&](int step, bool any, auto load) {
    const int t = steps.slot(step);
    if (any || step >= end || t + kTileStep - 1 > p_low || (a.window && t <= p_high - a.window && t + kTileStep - 1 >= a.sinks)) {
      // of the lane's first slot: how far it is behind the row, its window and the sinks' end, against constants
      const int behind = step < end ? p - t - 4 * g : -1, outside = a.window ? behind - a.window : -1, sinks = a.sinks - t - 4 * g;
      int page[4] = {0, 0, 0, 0};
      if (any) {
#pragma unroll
        for (int i = 0; i < 4; ++i) page[i] = pages.of(a, t + 16 * i);
      }
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int c = 32 * i + 8 * (e / 4) + e % 4;
          z[i][e] = ((page[2 * i + e / 8] >= 0) & (c <= behind) & ((c > outside) | (c < sinks))) ? z[i][e] : -INFINITY;
        }
    }
    float tops[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      tops[j] = z[j / 2][8 * (j % 2)];
#pragma unroll
      for (int e = 1; e < 8; ++e) tops[j] = fmaxf(tops[j], z[j / 2][8 * (j % 2) + e]);
    }
    float top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3])) * a.scale;
    // m is raised only when a logit passes it by kRaise; the sums hold that range in fp32, and so do weights of 16 bits.
    if (__any(top > m + kRaise<E>)) {
      top = fmaxf(top, __shfl_xor(top, 32, kWave));
      const float raised = fmaxf(m, top - kBelow<E>), was = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m - raised);
      m = raised;
      l *= was;
      exact *= was;
#pragma unroll
      for (int c = 0; c < CB; ++c)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[c][e] *= was;
    }
    const float ref = m == -INFINITY ? 0.0f : m;
    float add[4] = {};
#pragma unroll
    for (int kb = 0; kb < 4; ++kb) {
      const int i = kb / 2, e = 8 * (kb % 2);
      float x[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        x[j] = __builtin_amdgcn_exp2f(__builtin_fmaf(z[i][e + j], a.scale, -ref));
        if constexpr (LSE) exact += x[j];
      }
      // what is added up is what enters the products, so that a row's weights have the sum 1 however they are rounded
      w[kb] = make_uint4(pair_of<E>(x[0], x[1]), pair_of<E>(x[2], x[3]), pair_of<E>(x[4], x[5]), pair_of<E>(x[6], x[7]));
      add[0] = add_pair<E>(w[kb].x, add[0]);
      add[1] = add_pair<E>(w[kb].y, add[1]);
      add[2] = add_pair<E>(w[kb].z, add[2]);
      add[3] = add_pair<E>(w[kb].w, add[3]);
      load(kb);
    }
    l += (add[0] + add[1]) + (add[2] + add[3]);
  };
  // nothing is moved over these by the compiler
  auto meet = [&]() {
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  };
  auto arrived = [&]() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory"); };

  if (begin < end) {
    arrived();
    meet();
    int buffer = 0;   // of this step
    auto no_page = [&]() { return __any(missing[lane % WAVES]); };
    logits(0);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    meet();
    for (int step = begin; step < end; ++step) {
      // The next step's values and the keys of the one behind it (past the last step: its rows again, to places that nobody reads) go to
      // where this step's keys and the values of the one before were.
      const i32x4 k = rows_at(min(step + 2, end - 1), page2, a.c.k), v = rows_at(min(step + 1, end - 1), page1, a.c.v);
      const uint32_t k_to = lds0 + buffer * HALF, v_to = lds0 + (2 + (buffer ^ 1)) * HALF;
      weights(step, no_page(), [&](int i) {
#pragma unroll
        for (int j = i * LOADS / 4; j < (i + 1) * LOADS / 4; ++j) {
          load_ahead(k_to + j * 1024, key_off[j], k);
          load_ahead(v_to + j * 1024, value_off[j], v);
        }
      });
      page1 = page2;
      page2 = page_of(step + 3);
      if (page2 < 0 && lane == 0) missing[wave] = 1;   // two steps before it matters
      // Logits of the next step (where there is none, nobody looks at them) and products of this one.  Operands are asked for eight
      // products ahead: the LDS takes 150 to 200 cycles, a product 32.
      __builtin_amdgcn_s_setprio(1);
      const int keys = key_at + (buffer ^ 1) * HALF, values = value_at + (2 + buffer) * HALF;
      constexpr int P = 2 * KK + 4 * CB, AHEAD = 8;
      uint4 x[P];
      auto operand = [&](int i) {
        return i < 2 * KK ? key_operand(keys, i / 2, i % 2) : value_operand(values, (i - 2 * KK) / CB, (i - 2 * KK) % CB);
      };
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) x[i] = operand(i);
      __builtin_amdgcn_sched_group_barrier(kSchedLds, AHEAD, 0);
      z[0] = z[1] = f32x16{};
#pragma unroll
      for (int i = 0; i < P; ++i) {
        if (i < 2 * KK) {
          z[i % 2] = mfma32<E>(x[i], q[i / 2], z[i % 2]);
        } else {
          const int kb = (i - 2 * KK) / CB, c = (i - 2 * KK) % CB;
          acc[c] = mfma32<E>(x[i], w[kb], acc[c]);
        }
        __builtin_amdgcn_sched_group_barrier(kSchedProduct, 1, 0);
        if (i + AHEAD < P) {
          x[i + AHEAD] = operand(i + AHEAD);
          if (i + AHEAD < 2 * KK) __builtin_amdgcn_sched_group_barrier(kSchedLds, 1, 0);
          else __builtin_amdgcn_sched_group_barrier(kSchedLds, 2, 0);
        }
      }
      __builtin_amdgcn_s_setprio(0);
      arrived();
      meet();
      buffer ^= 1;
    }
  }

  arrived();   // loads that nobody reads
  l += __shfl_xor(l, 32, kWave);
  exact += __shfl_xor(exact, 32, kWave);
  bool whole = true;
#pragma unroll
  for (int c = 0; c < CB; ++c)
#pragma unroll
    for (int e = 0; e < 16; ++e) whole = whole && finite(acc[c][e]);
  const uint64_t bad = __ballot(!whole && l == l);   // a logit of +infinity or NaN makes l NaN, and with it the row
  const bool valid = live && mine0 + n < R;
  const size_t part = ((size_t)block * a.pieces + piece) * BM + 32 * wave;
  if (valid && g == 0) {
    if (a.pieces > 1) {
      a.tile_m[part + n] = m;
      a.tile_l[part + n] = l;
      if (LSE) a.tile_exact[part + n] = exact;
    } else if (LSE) {
      store_lse(a, out_row(a, s, h, row), m, exact);
    }
  }
  // Through the wave's part of the LDS, so that 16 neighbouring bytes of a row go to a lane and whole rows to neighbouring lanes: 32 channels at a
  // time, in fp32 where the sums are to be joined.
  meet();
  constexpr int PITCH = 32 * 4 + 16;   // of a row; 32 rows of four waves are below the buffers' size
  unsigned char* mine = smem + wave * 32 * PITCH;
  const float inverse = a.pieces > 1 ? 1.0f : rarely(l == 0.0f) ? without_weights(a, pages, p) : 1.0f / l;
  if (a.pieces > 1) {
#pragma unroll
    for (int c = 0; c < CB; ++c) {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        *reinterpret_cast<float4*>(mine + n * PITCH + 16 * (2 * j + g)) = make_float4(acc[c][4 * j], acc[c][4 * j + 1], acc[c][4 * j + 2], acc[c][4 * j + 3]);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int r = 8 * i + lane / 8;
        const float4 v = *reinterpret_cast<const float4*>(mine + r * PITCH + 16 * (lane % 8));
        if (mine0 + r < R) *reinterpret_cast<float4*>(a.tile_o + (part + r) * D + 32 * c + 4 * (lane % 8)) = v;
      }
    }
  } else {
#pragma unroll
    for (int c = 0; c < CB; c += 2) {
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          *reinterpret_cast<uint2*>(mine + n * PITCH + 64 * k + 8 * (2 * j + g)) =
              make_uint2(pair_of<E>(acc[c + k][4 * j] * inverse, acc[c + k][4 * j + 1] * inverse),
                         pair_of<E>(acc[c + k][4 * j + 2] * inverse, acc[c + k][4 * j + 3] * inverse));
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int r = 8 * i + lane / 8;
        const uint4 v = *reinterpret_cast<const uint4*>(mine + r * PITCH + 16 * (lane % 8));
        if (mine0 + r < R)
          *reinterpret_cast<uint4*>(reinterpret_cast<typename E::T*>(a.out) + out_row(a, s, h, mine0 + r) * D + 32 * c + 8 * (lane % 8)) = v;
      }
    }
  }
  if (lane == 0) broken[wave] = (unsigned)bad | (unsigned)(bad >> 32);
  __syncthreads();
  // an infinity or a NaN among the values, seen or not
  static_assert(WAVES == 4 && sizeof(RowsLds<D>) <= 4 * HALF);
  for (int w = 0; w < 2 * WAVES; ++w) {
    const int first = row0 + 16 * w;
    const unsigned only = __builtin_amdgcn_readfirstlane(broken[w / 2] >> (16 * (w % 2))) & 0xffffu;
    if (!rarely(only != 0) || first >= R) continue;
    sixteen_rows<E, D, true>(
        a, s, pages, h, first, R, [&](int step) { return steps.slot(step / 2) + 32 * (step % 2); }, 2 * begin, 2 * end, only,
        *reinterpret_cast<RowsLds<D>*>(smem), [&](int r, int d, float mr, float lr, float (&v)[4]) {
          if (a.pieces > 1) {
            const size_t to = ((size_t)block * a.pieces + piece) * BM + 16 * w + r;
            *reinterpret_cast<float4*>(a.tile_o + to * D + d) = make_float4(v[0], v[1], v[2], v[3]);
            if (d == 0) {
              a.tile_m[to] = mr;
              a.tile_l[to] = lr;
              if (LSE) a.tile_exact[to] = lr;
            }
          } else {
            const float inverse = lr == 0.0f ? without_weights(a, pages, s.slot + (first + r) / a.G) : 1.0f / lr;
            const int64_t at = out_row(a, s, h, first + r);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] *= inverse;
            store_row4<E>(a, D, at, d, v);
            if (d == 0) store_lse(a, at, mr, lr);
          }
        });
  }
}

template <class E, int D, int WAVES, bool LSE>
__global__ __launch_bounds__(64 * WAVES, 2) void gemm_kvp_tiles_kernel(KvpAttend a) { tile_block<E, D, WAVES, LSE>(a, blockIdx.x, blockIdx.y); }

// The pieces of a tile's rows put together, eight channels of a row a thread, all pieces' requests at once, eight at a time.
template <class E, int D>
__device__ __forceinline__ void join_tiles(const KvpAttend& a, int64_t first, int64_t blocks) {
  constexpr int LANES = D / 8, ROWS = 256 / LANES, N = 8;   // lanes of a row, rows of a workgroup
  const int BM = a.tile_rows, parts = BM / ROWS, lane = threadIdx.x % LANES;
  for (int64_t each = first; each < (int64_t)a.tiles * a.c.H * parts; each += blocks) {
    const int block = (int)(each / parts), r0 = (int)(each - (int64_t)block * parts) * ROWS + threadIdx.x / LANES;
    const int h = block % a.c.H, tile = a.tiles - 1 - block / a.c.H;
    const int b = sentence_of_tile(a, tile, BM);
    const Sentence s = sentence(a, b);
    const int R = s.rows * a.G;
    const int64_t row = (tile - tile_start(a, b, BM)) * BM + r0;
    if (R <= a.few || row < r0 || row >= R) continue;
    const size_t from = (size_t)block * a.pieces * BM + r0;
    float top = -INFINITY, total = 0.0f, exact = 0.0f, sum[8] = {};
    for (int i0 = 0; i0 < a.pieces; i0 += N) {
      float m[N], l[N], x[N];
      float4 o[N][2];
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const size_t at = from + (size_t)min(i0 + i, a.pieces - 1) * BM;
        m[i] = i0 + i < a.pieces ? a.tile_m[at] : -INFINITY;
        l[i] = i0 + i < a.pieces ? a.tile_l[at] : 0.0f;
        x[i] = a.lse ? a.tile_exact[at] : 0.0f;
        const float4* src = reinterpret_cast<const float4*>(a.tile_o + at * D + 8 * lane);
        o[i][0] = src[0];
        o[i][1] = src[1];
      }
      float next = top;
#pragma unroll
      for (int i = 0; i < N; ++i) next = fmaxf(next, m[i]);
      const float was = top == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(top - next);
      top = next;
      total *= was;   // a NaN that came without a maximum stays
      exact *= was;
#pragma unroll
      for (int c = 0; c < 8; ++c) sum[c] *= factor_of(sum[c], was);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        // a piece without a maximum saw nothing, or nothing but NaN
        const float f = m[i] == -INFINITY ? (l[i] != 0.0f ? NAN : 0.0f) : __builtin_amdgcn_exp2f(m[i] - top);
        const float v[8] = {o[i][0].x, o[i][0].y, o[i][0].z, o[i][0].w, o[i][1].x, o[i][1].y, o[i][1].z, o[i][1].w};
        if (f == 0.0f) {   // only what is not finite counts
          if (i0 + i >= a.pieces) continue;
          total += l[i] * 0.0f;
#pragma unroll
          for (int c = 0; c < 8; ++c) sum[c] += finite(v[c]) ? 0.0f : v[c];
          continue;
        }
        total = __builtin_fmaf(l[i], f, total);
        exact = __builtin_fmaf(x[i], f, exact);
#pragma unroll
        for (int c = 0; c < 8; ++c) sum[c] = __builtin_fmaf(v[c], f, sum[c]);
      }
    }
    const float inverse = rarely(total == 0.0f) ? without_weights(a, Pages(a, b, s.len), s.slot + (int)row / a.G) : 1.0f / total;
    const int64_t at = out_row(a, s, h, (int)row);
    *reinterpret_cast<uint4*>(reinterpret_cast<typename E::T*>(a.out) + at * D + 8 * lane) =
        make_uint4(pair_of<E>(sum[0] * inverse, sum[1] * inverse), pair_of<E>(sum[2] * inverse, sum[3] * inverse),
                   pair_of<E>(sum[4] * inverse, sum[5] * inverse), pair_of<E>(sum[6] * inverse, sum[7] * inverse));
    if (lane == 0) store_lse(a, at, top, total != total ? total : exact);
  }
}

template <class E, int D>
__global__ __launch_bounds__(256) void kvp_join_tiles_kernel(KvpAttend a) { join_tiles<E, D>(a, blockIdx.x, gridDim.x); }
template <int D>
unsigned join_tiles_blocks(const KvpAttend& a) { return join_blocks((int64_t)a.tiles * a.c.H * (a.tile_rows / (256 / (D / 8)))); }

template <class E, int D, int WAVES>
int launch_tiles(const KvpAttend& a, hipStream_t s) {
  const size_t lds = 4 * kTileStep * 2 * D;
  auto launch = [&](auto kernel, std::atomic<uint64_t>& seen) -> int {
    const int rc = allow_dynamic_lds(seen, reinterpret_cast<const void*>(kernel), lds);
    if (rc != CI_OK) return rc;
    hipLaunchKernelGGL(kernel, dim3((unsigned)(a.tiles * a.c.H), (unsigned)a.pieces), dim3(64 * WAVES), lds, s, a);
    CI_HIP_CHECK_LAUNCH();
    return CI_OK;
  };
  static std::atomic<uint64_t> with{0}, without{0};
  const int rc = a.lse ? launch(gemm_kvp_tiles_kernel<E, D, WAVES, true>, with) : launch(gemm_kvp_tiles_kernel<E, D, WAVES, false>, without);
  if (rc != CI_OK) return rc;
  if (a.pieces > 1) {
    hipLaunchKernelGGL((kvp_join_tiles_kernel<E, D>), dim3(join_tiles_blocks<D>(a)), dim3(256), 0, s, a);
    CI_HIP_CHECK_LAUNCH();
  }
  return CI_OK;
}

}  // namespace
}  // namespace ci
