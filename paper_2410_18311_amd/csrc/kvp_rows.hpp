// Attention of few rows of a head over a cache in pages (kvp_attend.hpp), one token a sentence above all: bound by the cache's bytes.
//
// The slots of all sentences are shared out by length over four workgroups a compute unit (or a head's stay together), which take 16 rows at a time
// (kvp_walk.hpp); a second launch joins the pieces.  Logits and sums are fp32; probabilities enter the product as two 16-bit
// pieces (rounded to one they would cost fp16 results more than their own rounding; the second product is hidden behind the loads), and
// fp32 caches go through fp32 products as they are.
//
// Eight sentences to 65536 slots, 8 x 8 heads of 128, bf16: 178 us for 973 MB, 5.5 TB/s (a copy of 1 GiB: 5.2), of which the join takes 6.  4096 slots
// of 40 heads: 20.5 us for 84 MB, 4 of them the join.  fp32 prompts take this way too, 16 rows a workgroup, at 70 TFLOP/s (4096 tokens of 32 heads
// of 128: 1940 to 1990 us), where a library product reaches 153: each tile reads the cache from the L2 again.
#pragma once

#include "kvp_walk.hpp"

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

// Piece `block` of all, the tiles from tile0 on that are `stride` apart.
template <class E, int D>
__device__ __forceinline__ void rows_block(const KvpAttend& a, int block, int tile0, int stride, RowsLds<D>& lds) {
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
  for (int tile = tile0; tile * 16 < R; tile += stride) {
    const int row0 = tile * 16;
    // a piece of the sentence's steps, or all of the tile's own
    const Steps<32> steps =
        found.pieces > 1 ? all : Steps<32>(a, max(s.slot + row0 / a.G, 0), s.slot + min(row0 + 15, R - 1) / a.G, s.len);
    const int begin = min(steps.total, piece * found.chunk), end = min(steps.total, begin + min(found.chunk, steps.total));
    const size_t part = a.wanted ? ((size_t)block * a.row_tiles + tile) * 16 : 0;
    auto slot = [&](int step) { return steps.slot(step); };
    auto store = [&](int r, int d, float m, float l, float (&v)[4]) {
      if (a.wanted) {
        *reinterpret_cast<float4*>(a.o + (part + r) * D + d) = make_float4(v[0], v[1], v[2], v[3]);
        if (d == 0) {
          a.m[part + r] = m;
          a.l[part + r] = l;
        }
      } else {
        const float inverse = rarely(l == 0.0f) ? without_weights(a, pages, s.slot + (row0 + r) / a.G) : 1.0f / l;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] *= inverse;
        const int64_t at = out_row(a, s, h, row0 + r);
        store_row4<E>(a, D, at, d, v);
        if (d == 0) store_lse(a, at, m, l);
      }
    };
    const unsigned broken = sixteen_rows<E, D, false>(a, s, pages, h, row0, R, slot, begin, end, 0, lds, store);
    // an infinity or a NaN among the values, seen or not
    if (rarely(broken != 0)) sixteen_rows<E, D, true>(a, s, pages, h, row0, R, slot, begin, end, broken, lds, store);
  }
}

// With 128 channels two workgroups a compute unit and not three, for which 163 registers would do: of four, two and two take 178 us over eight sentences
// to 65536 slots, three and one 184.
template <class E, int D>
__global__ __attribute__((amdgpu_flat_work_group_size(256, 256), amdgpu_waves_per_eu(2, D == 128 ? 2 : 4))) void gemm_kvp_rows_kernel(
    KvpAttend a) {
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
      reinterpret_cast<typename E::T*>(a.out)[at * D + d] = from_float<E>(rarely(total == 0.0f) ? without_weights(a, Pages(a, b, s.len), s.slot + i) : v * (1.0f / total));
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
