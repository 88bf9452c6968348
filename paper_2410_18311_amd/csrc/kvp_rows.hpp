// Attention of few rows of a head over a cache in pages (kvp_attend.hpp), one token a sentence above all: bound by the cache's bytes.
//
// The slots of all sentences are shared out by length over four workgroups a compute unit (or a head's stay together), whose waves take every fourth step of 32 slots, each with
// its own running maximum; a second launch joins the pieces.  A wave reads keys and values as they lie, 16 bytes a lane, a step
// ahead, without the LDS, which would only add a wait: nobody else of the workgroup reads them.  A lane's channels of eight slots are
// turned into operands of one channel by one permutation a word.  Logits and sums are fp32; probabilities enter the product as two 16-bit
// pieces (rounded to one they would cost fp16 results more than their own rounding; the second product is hidden behind the loads), and
// fp32 caches go through fp32 products as they are.
//
// Eight sentences to 65536 slots, 8 x 8 heads of 128, bf16: 178 us for 973 MB, 5.5 TB/s (a copy of 1 GiB: 5.2), of which the join takes 6.  4096 slots
// of 40 heads: 20.5 us for 84 MB, 4 of them the join.  Of the bf16 kernel's 173 registers the keys and values on their way are most: at
// three waves a SIMD it spilled, 193 and 25.5 us.  fp32 prompts take this way too, 16 rows a workgroup, at 68 TFLOP/s (4096 tokens of 32 heads of 128:
// 2031 us), where a library product reaches 153: each tile reads the cache from the L2 again.
#pragma once

#include "kvp_attend.hpp"

namespace ci {
namespace {

// How the slots are shared out: pieces of `chunk` steps, so that a long sentence among short ones has as many workgroups as its
// length asks for; or a head's slots in one piece where there are enough heads.  Everything follows from first and lens, in every
// wave for itself, a sentence a lane.
struct Piece {
  Sentence s;
  int b, before, pieces;   // the sentence, the pieces before its own, how many a head has; b = B: no such piece
  int chunk;
  __device__ Piece(const KvpAttend& a, int at) {
    if (!a.wanted) {
      // nothing to look for: one token of 4000 sentences of 64 slots, 8 heads, 297 us, and 1127 when their pieces were counted all the same
      b = at / a.c.H;
      before = b * a.c.H;
      pieces = 1;
      chunk = 1 << 30;
      s = uniform(sentence(a, b));
      if (s.rows == 0 || (int64_t)s.rows * a.G > a.few) b = a.c.B;
      return;
    }
    const int lane = threadIdx.x & 63;
    Sentence own{0, 0, 0, 0};
    int mine = -1;   // steps of the lane's sentence; -1: another's work, or none
    auto look = [&](int b0) {
      mine = -1;
      if (b0 + lane >= a.c.B) return;
      own = sentence(a, b0 + lane);
      if (own.rows > 0 && (int64_t)own.rows * a.G <= a.few)
        mine = Steps<32>(a, max(own.slot, 0), own.slot + own.rows - 1, own.len).total;
    };
    look(0);
    int64_t total = 0;
    int longest = 0;
    for (int b0 = 0;;) {
      const int v = max(mine, 0);
      if (a.c.B == 1) {
        total = longest = __builtin_amdgcn_readfirstlane(v);
      } else {
        total += __builtin_amdgcn_readlane(scan_add(v), 63);
        longest = max(longest, __builtin_amdgcn_readlane(scan_max(v), 63));
      }
      b0 += 64;
      if (b0 >= a.c.B) break;
      look(b0);
    }
    if (a.c.B > 64) look(0);
    // all pieces together are at most wanted + B H: a sentence's last one need not be full
    const int64_t even = (total * a.c.H + a.wanted - 1) / a.wanted, least = max(a.least, (longest + kMaxPieces - 1) / kMaxPieces);
    chunk = (int)((max(even, least) + 3) / 4 * 4);
    int base = 0;
    for (int b0 = 0;;) {
      // at least one piece: it writes the zeros of rows that see nothing
      const int count = mine < 0 ? 0 : max(1, (mine + chunk - 1) / chunk), upto = a.c.B == 1 ? count : scan_add(count);
      const uint64_t past = __ballot(base + upto * a.c.H > at);
      if (past) {
        const int hit = __builtin_ctzll(past);
        b = b0 + hit;
        pieces = __builtin_amdgcn_readlane(count, hit);
        before = base + (__builtin_amdgcn_readlane(upto, hit) - pieces) * a.c.H;
        s = Sentence{__builtin_amdgcn_readlane(own.first, hit), __builtin_amdgcn_readlane(own.rows, hit),
                     __builtin_amdgcn_readlane(own.len, hit), __builtin_amdgcn_readlane(own.slot, hit)};
        return;
      }
      base += __builtin_amdgcn_readlane(upto, 63) * a.c.H;
      b0 += 64;
      if (b0 >= a.c.B) break;
      look(b0);
    }
    b = a.c.B;
  }
};

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

// Piece `block` of all, the tiles from tile0 on that are `stride` apart.
template <class E, int D>
__device__ __forceinline__ void rows_block(const KvpAttend& a, int block, int tile0, int stride, RowsLds<D>& lds) {
  using S32 = Step32<E, D>;
  constexpr int K = S32::K, CH = S32::CH, VW = S32::V;
  auto& ml = lds.ml;
  auto& sums = lds.sums;
  const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Piece found(a, block);
  const int b = found.b;
  if (b >= a.c.B) return;
  const int piece = (block - found.before) / a.c.H, h = block - found.before - piece * a.c.H;
  const Sentence s = found.s;
  const int R = s.rows * a.G;
  const Steps<32> all(a, max(s.slot, 0), s.slot + s.rows - 1, s.len);
  if (a.wanted && block == found.before && tile0 == 0 && threadIdx.x == 0)
    a.place[b] = make_int2(found.before, found.pieces);   // for the join
  const Pages pages(a, b, s.len);
  const int inside = (1 << a.c.shift) - 1;
  for (int tile = tile0; tile * 16 < R; tile += stride) {
    const int row0 = tile * 16;
    const int row = min(row0 + n, R - 1);   // rows past the last repeat it
    const int p = s.slot + row / a.G;
    const int p_low = s.slot + row0 / a.G, p_high = s.slot + min(row0 + 15, R - 1) / a.G;   // of the tile's rows
    // a piece of the sentence's steps, or all of the tile's own
    const Steps<32> steps = found.pieces > 1 ? all : Steps<32>(a, max(p_low, 0), p_high, s.len);
    const int begin = min(steps.total, piece * found.chunk), end = min(steps.total, begin + min(found.chunk, steps.total));

    if (threadIdx.x == 0) lds.broken = 0;
    uint4 q[K];
    load_query<E, D>(a, s, h, row, q);

    S32 x;
    auto find_pages = [&](int step) {
      const int t = steps.slot(min(step, end - 1));
#pragma unroll
      for (int i = 0; i < 2; ++i) x.page[i] = pages.of(a, t + 16 * i);
    };
    auto load_keys = [&](int step, const int (&page)[2]) {
      const int t = steps.slot(step);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int slot = min(t + 16 * i + n, pages.last) & inside;
        const typename E::T* src = reinterpret_cast<const typename E::T*>(a.c.k) + page_start<D>(a, page[i], h) + slot * D + g * E::VEC;
#pragma unroll
        for (int j = 0; j < K; ++j) x.k[i][j] = ld16(src + 4 * j * E::VEC);
      }
    };
    auto load_values = [&](int step, const int (&page)[2]) {
      const int t = steps.slot(step);
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
      load_keys(step, page);
      load_values(step, page);
      find_pages(step + 4);
      for (; step < end; step += 4) {
        const int t = steps.slot(step);
        const int next[2] = {x.page[0], x.page[1]};
        const bool more = step + 4 < end;
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
        const bool masked = page[0] < 0 || page[1] < 0 || t + 31 > p_low || (a.window && t <= p_high - a.window && t + 31 >= a.sinks);
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            z[i][r] *= a.scale;
            if (masked) z[i][r] = ((page[i] >= 0) & sees(a, p, t + 16 * i + 4 * g + r)) ? z[i][r] : -INFINITY;
          }
        float top = fmaxf(fmaxf(fmaxf(z[0][0], z[0][1]), fmaxf(z[0][2], z[0][3])), fmaxf(fmaxf(z[1][0], z[1][1]), fmaxf(z[1][2], z[1][3])));
        // m is raised only when a logit passes it by kRaise; the sums hold that range in fp32.
        if (__any(top > m + kRaise<E>)) {
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
    float top = ml[0][0][n];
#pragma unroll
    for (int w = 1; w < 4; ++w) top = fmaxf(top, ml[0][w][n]);
    const float own = m == -INFINITY ? (l != 0.0f ? NAN : 0.0f) : __builtin_amdgcn_exp2f(m - top);
    if (row0 + n < R) {
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int c = 0; c < CH; c += 4)
          *reinterpret_cast<float4*>(&sums[wave][n][CH * (4 * g + r) + c]) =
              make_float4(acc[c][r] * own, acc[c + 1][r] * own, acc[c + 2][r] * own, acc[c + 3][r] * own);
    }
    __syncthreads();

    const int live = min(16, R - row0);
    const size_t part = a.wanted ? ((size_t)block * a.row_tiles + tile) * 16 : 0;
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
      // a logit of +infinity or NaN makes the row's sum NaN, and with it the row: nothing of it is to be done again
      if (total == total && !(finite(v[0]) && finite(v[1]) && finite(v[2]) && finite(v[3]))) atomicOr(&lds.broken, 1u << r);
      if (a.wanted) {
        *reinterpret_cast<float4*>(a.o + (part + r) * D + d) = make_float4(v[0], v[1], v[2], v[3]);
        if (d == 0) {
          a.m[part + r] = t;
          a.l[part + r] = total;
        }
      } else {
        const float inverse = total == 0.0f ? without_weights(a, pages, s.slot + (row0 + r) / a.G) : 1.0f / total;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] *= inverse;
        const int64_t at = out_row(a, s, h, row0 + r);
        store_row4<E>(a, D, at, d, v);
        if (d == 0) store_lse(a, at, t, total);
      }
    }
    __syncthreads();
    // an infinity or a NaN among the values, seen or not
    for (unsigned left = lds.broken; left; left &= left - 1) {
      const int r = __builtin_ctz(left);
      float mr, lr, o;
      careful_row<E, D, 32, 256>(a, s, pages, h, row0 + r, steps, begin, end, &sums[0][0][0], &mr, &lr, &o);
      if (a.wanted) {
        if (threadIdx.x < D) a.o[(part + r) * D + threadIdx.x] = o;
        if (threadIdx.x == 0) {
          a.m[part + r] = mr;
          a.l[part + r] = lr;
        }
      } else {
        const int64_t at = out_row(a, s, h, row0 + r);
        if (threadIdx.x < D) reinterpret_cast<typename E::T*>(a.out)[at * D + threadIdx.x] = from_float<E>(lr == 0.0f ? without_weights(a, pages, s.slot + (row0 + r) / a.G) : o / lr);
        if (threadIdx.x == 0) store_lse(a, at, mr, lr);
      }
    }
    __syncthreads();
  }
}

template <class E, int D>
__global__ __launch_bounds__(256, 2) void gemm_kvp_rows_kernel(KvpAttend a) {
  __shared__ RowsLds<D> lds;
  rows_block<E, D>(a, blockIdx.x, blockIdx.y, gridDim.y, lds);
}

// The pieces of a row put together, a workgroup a row: a wave takes every fourth, all of which it requests at once.
template <class E, int D>
__device__ __forceinline__ void join_rows(const KvpAttend& a, int64_t block, int64_t blocks) {
  constexpr int N = kMaxPieces / 4, C = D / 64;
  __shared__ float sums[4][D];
  const int Hq = a.c.H * a.G, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  for (int64_t each = block; each < (int64_t)a.c.B * a.join_rows * Hq; each += blocks) {
    const int b = (int)(each / (a.join_rows * Hq)), in = (int)(each - (int64_t)b * a.join_rows * Hq);
    const int i = in / Hq, head = in - i * Hq, h = head / a.G;
    const Sentence s = sentence(a, b);
    const int2 place = a.place[b];   // written for sentences that have few rows only
    if (i >= s.rows || (int64_t)s.rows * a.G > a.few) continue;
    const int r = i * a.G + head - h * a.G;
    const int64_t at = (int64_t)(s.first + i) * Hq + head;   // row of out
    const size_t from = ((size_t)(place.x + h) * a.row_tiles + r / 16) * 16 + r % 16, next = (size_t)a.c.H * a.row_tiles * 16;
    const float m = lane < place.y ? a.m[from + lane * next] : -INFINITY, l = lane < place.y ? a.l[from + lane * next] : 0.0f;
    float o[N][C];
#pragma unroll
    for (int n = 0; n < N; ++n)
      if (wave + 4 * n < place.y) __builtin_memcpy(o[n], a.o + (from + (wave + 4 * n) * next) * D + lane * C, sizeof(o[n]));
    float top = m;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) top = fmaxf(top, __shfl_xor(top, off, kWave));
    // a piece without a maximum saw nothing, or nothing but NaN
    const float factor = m == -INFINITY ? (l != 0.0f ? NAN : 0.0f) : __builtin_amdgcn_exp2f(m - top);
    const float total = wave_sum(m == -INFINITY ? l : l * factor);
    float sum[C] = {};
#pragma unroll
    for (int n = 0; n < N; ++n) {
      if (wave + 4 * n >= place.y) continue;
      const float f = __shfl(factor, wave + 4 * n, kWave);
#pragma unroll
      for (int c = 0; c < C; ++c) sum[c] = __builtin_fmaf(o[n][c], factor_of(o[n][c], f), sum[c]);
    }
#pragma unroll
    for (int c = 0; c < C; ++c) sums[wave][lane * C + c] = sum[c];
    __syncthreads();
    if (threadIdx.x < D) {
      const int d = threadIdx.x;
      const float v = (sums[0][d] + sums[1][d]) + (sums[2][d] + sums[3][d]);
      reinterpret_cast<typename E::T*>(a.out)[at * D + d] = from_float<E>(total == 0.0f ? without_weights(a, Pages(a, b, s.len), s.slot + i) : v * (1.0f / total));
      if (d == 0) store_lse(a, at, top, total);
    }
    __syncthreads();
  }
}

template <class E, int D>
__global__ __launch_bounds__(256) void kvp_join_kernel(KvpAttend a) { join_rows<E, D>(a, blockIdx.x, gridDim.x); }
inline unsigned join_rows_blocks(const KvpAttend& a) { return join_blocks((int64_t)a.c.B * a.join_rows * a.c.H * a.G); }

template <class E, int D>
int launch_rows(const KvpAttend& a, hipStream_t s) {
  hipLaunchKernelGGL((gemm_kvp_rows_kernel<E, D>), dim3((unsigned)a.blocks, (unsigned)a.row_tiles), dim3(256), 0, s, a);
  CI_HIP_CHECK_LAUNCH();
  if (a.wanted) {
    hipLaunchKernelGGL((kvp_join_kernel<E, D>), dim3(join_rows_blocks(a)), dim3(256), 0, s, a);
    CI_HIP_CHECK_LAUNCH();
  }
  return CI_OK;
}

}  // namespace
}  // namespace ci
