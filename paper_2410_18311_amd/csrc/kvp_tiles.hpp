// Attention of prompts over a cache in pages (kvp_attend.hpp), 16-bit types: bound by the matrix cores and what feeds them.
//
// A workgroup takes a tile of rows of a head, 32 to a wave, and steps of 64 slots, which go from the pages straight into the LDS, a step ahead.  Products
// of 32 x 32: the logits of 32 rows come out with a row's 32 slots in two lanes, and the values are read from the LDS transposed, four slots of a
// channel to a lane, in the order in which the probabilities lie.
#pragma once

#include "gemm_tile.hpp"
#include "kvp_attend.hpp"

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

constexpr int kTileStep = 64;   // slots of a step

// Rows of D channels in the LDS, 16-byte chunk c of row r in the place c ^ swizzle(r), so that what 16 lanes read at once lies in
// different banks.  Keys: the same chunk of 16 rows; values: 64 bytes of four rows.
template <int D>
__device__ __forceinline__ int key_swizzle(int r) { return D == 128 ? r & 15 : r >> 1 & 7; }
template <int D>
__device__ __forceinline__ int value_swizzle(int r) { return (D == 128 ? r & 3 : r >> 1 & 1) << 2; }

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

template <class E, int D, int WAVES>
__global__ __launch_bounds__(64 * WAVES, 2) void gemm_kvp_tiles_kernel(KvpAttend a) {
  constexpr int BM = 32 * WAVES, ROW = 2 * D, HALF = kTileStep * ROW, KK = D / 16, CB = D / 32;
  constexpr int LOADS = HALF / 1024 / WAVES, ROWS = 1024 / ROW;   // loads of a wave and tensor, rows of a load
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];   // [2][keys, values][64 rows]
  __shared__ unsigned broken[WAVES];
  const int lane = threadIdx.x & 63, n = lane & 31, g = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int h = blockIdx.x % a.c.H, tile = a.tiles - 1 - (int)(blockIdx.x / a.c.H);   // the last tiles of a prompt see most
  const int b = sentence_of_tile(a, tile, BM);
  const Sentence s = sentence(a, b);
  const int R = s.rows * a.G;
  const int64_t local = tile - tile_start(a, b, BM);
  if (R <= a.few || local < 0 || local * BM >= R) return;
  const int row0 = (int)local * BM, mine0 = row0 + 32 * wave;   // of the tile, of the wave
  const bool live = mine0 < R;
  const int row = min(mine0 + n, R - 1), p = s.slot + row / a.G;
  const int p_low = s.slot + min(mine0, R - 1) / a.G, p_high = s.slot + min(mine0 + 31, R - 1) / a.G;
  const Steps<kTileStep> steps(a, max(s.slot + row0 / a.G, 0), s.slot + min(row0 + BM - 1, R - 1) / a.G, s.len);
  const int begin = (int)((int64_t)steps.total * blockIdx.y / a.pieces), end = (int)((int64_t)steps.total * (blockIdx.y + 1) / a.pieces);
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

  // A wave fetches LOADS * ROWS neighbouring rows of a step, which are of one page.
  const int fetch_row = lane / (ROW / 16), fetch_chunk = lane % (ROW / 16);
  auto fetch = [&](int step, int buffer) {
    const int t = steps.slot(step) + wave * LOADS * ROWS;
    const int page = pages.of(a, t);
    const int64_t at = page_start<D>(a, page, h) * 2;
    const i32x4 k = rsrc_at(reinterpret_cast<const char*>(a.c.k) + at), v = rsrc_at(reinterpret_cast<const char*>(a.c.v) + at);
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int r = wave * LOADS * ROWS + i * ROWS + fetch_row;
      const int from = (min(t + i * ROWS + fetch_row, pages.last) & inside) * ROW;
      unsigned char* to = smem + buffer * 2 * HALF + (wave * LOADS + i) * 1024;
      load_to_lds(to, from + 16 * (fetch_chunk ^ key_swizzle<D>(r)), k);
      load_to_lds(to + HALF, from + 16 * (fetch_chunk ^ value_swizzle<D>(r)), v);
    }
  };

  float m = -INFINITY, l = 0.0f;   // m: scaled; l: of the lane's own slots
  f32x16 acc[CB];
#pragma unroll
  for (int c = 0; c < CB; ++c) acc[c] = f32x16{};

  // the lane's places in a buffer: keys of row n, by 16 channels; values of slots 4 g + .. by 32 channels
  const int value_row = 4 * g + (lane & 15) / 4;
  const int value_at = value_row * ROW + 32 * (lane >> 4 & 1) + 8 * (lane & 3);
  if (begin < end) fetch(begin, 0);
  for (int step = begin; step < end; ++step) {
    const int buffer = (step - begin) & 1;
    // this step's slots have come for all waves, and all have done with the other buffer
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    if (step + 1 < end) fetch(step + 1, buffer ^ 1);
    const int t = steps.slot(step);
    if (!live || t > p_high) continue;
    const unsigned char* keys = smem + buffer * 2 * HALF;
    const unsigned char* values = keys + HALF;
    f32x16 z[2] = {f32x16{}, f32x16{}};
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
      const int at = n * ROW + 16 * ((2 * kk + g) ^ key_swizzle<D>(n));
#pragma unroll
      for (int i = 0; i < 2; ++i) z[i] = mfma32<E>(*reinterpret_cast<const uint4*>(keys + at + i * 32 * ROW), q[kk], z[i]);
    }
    bool masked = t + kTileStep - 1 > p_low || (a.window && t <= p_high - a.window && t + kTileStep - 1 >= a.sinks);
    int page[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      page[i] = pages.of(a, t + 16 * i);
      masked = masked || page[i] < 0;
    }
    if (masked) {
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (page[2 * i + e / 8] < 0 || !sees(a, p, t + 32 * i + 8 * (e / 4) + 4 * g + e % 4)) z[i][e] = -INFINITY;
    }
    float top = z[0][0];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) top = fmaxf(top, z[i][e]);
    top *= a.scale;
    // The maximum is raised only when a logit passes it by 2^8; the sums hold that range in fp32, and so do probabilities of 16 bits.
    if (__any(top > m + 8.0f)) {
      top = fmaxf(top, __shfl_xor(top, 32, kWave));
      const float raised = fmaxf(m, top), was = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m - raised);
      m = raised;
      l *= was;
#pragma unroll
      for (int c = 0; c < CB; ++c)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[c][e] *= was;
    }
    const float ref = m == -INFINITY ? 0.0f : m;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        z[i][e] = __builtin_amdgcn_exp2f(__builtin_fmaf(z[i][e], a.scale, -ref));
        l += z[i][e];
      }
#pragma unroll
    for (int kb = 0; kb < 4; ++kb) {
      const int i = kb / 2, e = 8 * (kb % 2);
      const uint4 w = make_uint4(pair_of<E>(z[i][e], z[i][e + 1]), pair_of<E>(z[i][e + 2], z[i][e + 3]), pair_of<E>(z[i][e + 4], z[i][e + 5]),
                                 pair_of<E>(z[i][e + 6], z[i][e + 7]));
#pragma unroll
      for (int c = 0; c < CB; ++c) {
        const int at = value_at + ((64 * c) ^ (16 * value_swizzle<D>(value_row))) + 16 * kb * ROW;
        const s16x4 first = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(values + at));
        const s16x4 second = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(values + at + 8 * ROW));
        const uint2 x = __builtin_bit_cast(uint2, first), y = __builtin_bit_cast(uint2, second);
        acc[c] = mfma32<E>(make_uint4(x.x, x.y, y.x, y.y), w, acc[c]);
      }
    }
  }

  l += __shfl_xor(l, 32, kWave);
  bool whole = true;
#pragma unroll
  for (int c = 0; c < CB; ++c)
#pragma unroll
    for (int e = 0; e < 16; ++e) whole = whole && finite(acc[c][e]);
  const uint64_t bad = __ballot(!whole);
  const bool valid = live && mine0 + n < R;
  const size_t part = ((size_t)blockIdx.x * a.pieces + blockIdx.y) * BM + 32 * wave + n;
  if (valid && a.pieces > 1) {
    if (g == 0) {
      a.tile_m[part] = m;
      a.tile_l[part] = l;
    }
#pragma unroll
    for (int c = 0; c < CB; ++c)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        *reinterpret_cast<float4*>(a.tile_o + part * D + 32 * c + 8 * j + 4 * g) =
            make_float4(acc[c][4 * j], acc[c][4 * j + 1], acc[c][4 * j + 2], acc[c][4 * j + 3]);
  } else if (valid) {
    const int64_t at = out_row(a, s, h, row);
    const float inverse = l == 0.0f ? 0.0f : 1.0f / l;
    if (g == 0) store_lse(a, at, m, l);
#pragma unroll
    for (int c = 0; c < CB; ++c)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float v[4] = {acc[c][4 * j] * inverse, acc[c][4 * j + 1] * inverse, acc[c][4 * j + 2] * inverse, acc[c][4 * j + 3] * inverse};
        store_row4<E>(a, D, at, 32 * c + 8 * j + 4 * g, v);
      }
  }
  if (lane == 0) broken[wave] = (unsigned)bad | (unsigned)(bad >> 32);
  __syncthreads();
  for (int w = 0; w < WAVES; ++w) {
    // an infinity or a NaN among the values, seen or not
    for (unsigned left = broken[w]; left; left &= left - 1) {
      const int r = row0 + 32 * w + __builtin_ctz(left);
      if (r >= R) break;
      float mr, lr, o;
      careful_row<E, D, kTileStep>(a, s, pages, h, r, steps, begin, end, reinterpret_cast<float*>(smem), &mr, &lr, &o);
      if (a.pieces > 1) {
        const size_t to = ((size_t)blockIdx.x * a.pieces + blockIdx.y) * BM + r - row0;
        if (threadIdx.x < D) a.tile_o[to * D + threadIdx.x] = o;
        if (threadIdx.x == 0) {
          a.tile_m[to] = mr;
          a.tile_l[to] = lr;
        }
      } else {
        const int64_t at = out_row(a, s, h, r);
        if (threadIdx.x < D) reinterpret_cast<typename E::T*>(a.out)[at * D + threadIdx.x] = from_float<E>(lr == 0.0f ? 0.0f : o / lr);
        if (threadIdx.x == 0) store_lse(a, at, mr, lr);
      }
    }
  }
}

// The pieces of a tile's rows put together, a wave a row.
template <class E, int D>
__global__ __launch_bounds__(256) void kvp_join_tiles_kernel(KvpAttend a) {
  const int lane = threadIdx.x & 63, BM = a.tile_rows;
  for (int64_t each = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); each < (int64_t)a.tiles * a.c.H * BM;
       each += (int64_t)gridDim.x * 4) {   // row of a tile of a head
    const int block = (int)(each / BM), r0 = (int)(each - (int64_t)block * BM);
    const int h = block % a.c.H, tile = a.tiles - 1 - block / a.c.H;
    const int b = sentence_of_tile(a, tile, BM);
    const Sentence s = sentence(a, b);
    const int R = s.rows * a.G;
    const int64_t local = tile - tile_start(a, b, BM);
    if (R <= a.few || local < 0 || local * BM + r0 >= R) continue;
    const size_t from = (size_t)block * a.pieces * BM + r0, next = BM;
    const float m = lane < a.pieces ? a.tile_m[from + lane * next] : -INFINITY, l = lane < a.pieces ? a.tile_l[from + lane * next] : 0.0f;
    float top = m;
  #pragma unroll
    for (int off = 1; off < 64; off <<= 1) top = fmaxf(top, __shfl_xor(top, off, kWave));
    const float factor = m == -INFINITY ? (l != 0.0f ? NAN : 0.0f) : __builtin_amdgcn_exp2f(m - top);
    const float total = wave_sum(m == -INFINITY ? l : l * factor);
    float sum[D / 64] = {};
    for (int i = 0; i < a.pieces; ++i) {
      const float f = __shfl(factor, i, kWave);
      const float* o = a.tile_o + (from + i * next) * D + lane * (D / 64);
  #pragma unroll
      for (int c = 0; c < D / 64; ++c) sum[c] += f == 0.0f ? 0.0f : f * o[c];
    }
    const float inverse = total == 0.0f ? 0.0f : 1.0f / total;
    const int64_t at = out_row(a, s, h, (int)local * BM + r0);
    typename E::T* dst = reinterpret_cast<typename E::T*>(a.out) + at * D + lane * (D / 64);
  #pragma unroll
    for (int c = 0; c < D / 64; ++c) dst[c] = from_float<E>(sum[c] * inverse);
    if (lane == 0) store_lse(a, at, top, total);
  }
}

template <class E, int D, int WAVES>
int launch_tiles(const KvpAttend& a, hipStream_t s) {
  static std::atomic<uint64_t> seen{0};
  const size_t lds = 4 * kTileStep * 2 * D;
  const int rc = allow_dynamic_lds(seen, reinterpret_cast<const void*>(&gemm_kvp_tiles_kernel<E, D, WAVES>), lds);
  if (rc != CI_OK) return rc;
  hipLaunchKernelGGL((gemm_kvp_tiles_kernel<E, D, WAVES>), dim3((unsigned)(a.tiles * a.c.H), (unsigned)a.pieces), dim3(64 * WAVES), lds, s, a);
  CI_HIP_CHECK_LAUNCH();
  if (a.pieces > 1) {
    hipLaunchKernelGGL((kvp_join_tiles_kernel<E, D>), dim3(join_blocks((int64_t)a.tiles * a.c.H * a.tile_rows)), dim3(256), 0, s, a);
    CI_HIP_CHECK_LAUNCH();
  }
  return CI_OK;
}

}  // namespace
}  // namespace ci
