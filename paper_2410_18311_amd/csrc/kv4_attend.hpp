// Attention over a cache in 4 bits (kv4.hpp): out = softmax(scale q k^T, causal) v for S rows of each query head, one token or a prompt's
// chunk, in one pass over the cache with a running maximum and sum.
//
// A wave takes a tile of 16 rows (of the S G rows that share a head of the cache, G query heads to each) and steps of 32 slots.  The logits come out
// of the matrix cores with slots down and rows across, four slots to a lane: just the layout in which the probabilities enter the product with
// the values, so nothing is exchanged between lanes.  Steps and lowest values enter in
// fp32: logit = step (q . codes) + low (sum q), and the probabilities are multiplied by the values' steps before they are split into
// bf16 pieces (16 bits of them for 16-bit results, 24 for fp32; one piece would cost fp16 results as much as their own rounding).  The
// running maximum is raised only when a logit passes it by 2^8, which a first look at the lane's own eight logits decides; the sums hold
// that range in fp32.  The results' sums and what has to leave them again, the codes' offset times the probabilities, and their lowest values, are large
// and nearly cancel, ever more so the more slots average out, so they are put together every few steps (kFold).
//
// Few rows: the waves of a workgroup take different steps and their sums are joined, and the slots of all sentences are shared out by length
// over three workgroups a compute unit, joined by a second launch.  Bound by the cache's bytes: eight sentences of up to 65536 slots,
// 259 MB, 57 us and 7 of the join (4.5 TB/s); where there are few of them by two launches' latency: 4096 slots of 40 heads 13 and 5 us.
// Many rows: the waves take different tiles and share a step's operands.  512 rows over 2048 slots of 32 heads 58 us, of which vector
// instructions, 28 a logit and row, are 27, operands from the LDS (16 KB a wave and step) up to 22 and matrix products 11: side by side only in part, and
// the waves, three a SIMD, wait in 29 % of their cycles.  27 us for the slots' weights, for which the logits are computed again.
#pragma once

#include "kv4.hpp"

namespace ci {
namespace {

// Steps of 32 slots after which a wave puts its sums together.  What stands between is 5 times (fp32: 2) what the slots' values come to at random
// and rounded at every step: 1e-5 of the results (fp32 2e-6) however many slots there are.
template <int OP> constexpr int kFold = OP == kOpExact ? 4 : 8;

template <class T> struct AttendType;
template <> struct AttendType<F32> { static constexpr int P = 3, OPV = kOpExact; };
template <> struct AttendType<F16> { static constexpr int P = 2, OPV = kOpBF16; };
template <> struct AttendType<BF16> { static constexpr int P = 2, OPV = kOpBF16; };

__device__ __forceinline__ uint32_t word_of(const uint4& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }

// A lane's 16 (D = 64: 8) bytes.
template <int D>
__device__ __forceinline__ uint4 ld_row(const uint32_t* p) {
  if constexpr (D == 128) return ld16(p);
  const uint2 u = *reinterpret_cast<const uint2*>(p);
  return make_uint4(u.x, u.y, 0, 0);
}

// The token of a row: row / G, rows and G being below 2^20 and 2^12.
__device__ __forceinline__ int row_token(const Kv4Attend& a, int row) { return a.G == 1 ? row : (int)__umulhi((uint32_t)row, a.inverse_G); }

// A lane's channels of a row of q as they are in memory: eight of each 32.
template <class T, int D>
struct RawRow {
  uint4 raw[D / 32][8 / T::VEC];
};
template <class T>
__device__ __forceinline__ void load_channels(const Kv4Attend& a, int b, int h, int row, int channel, uint4 (&to)[8 / T::VEC]) {
  const int s = row_token(a, row), i = row - s * a.G;
  const typename T::T* src = reinterpret_cast<const typename T::T*>(a.q) + b * a.q_b + s * a.q_s + (int64_t)(h * a.G + i) * a.q_h + channel;
  if (a.q_vectors) {
#pragma unroll
    for (int e = 0; e < 8 / T::VEC; ++e) to[e] = ld16(src + e * T::VEC);
  } else {
    typename T::T x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = src[e];
    __builtin_memcpy(to, x, sizeof(x));
  }
}
template <class T, int D>
__device__ __forceinline__ void load_raw(const Kv4Attend& a, int b, int h, int row, RawRow<T, D>& r) {
  const int g = (threadIdx.x & 63) >> 4;
#pragma unroll
  for (int j = 0; j < D / 32; ++j) load_channels<T>(a, b, h, row, 32 * j + 8 * g, r.raw[j]);
}
// The same as operands, and the sums of the row's channels by group.
template <class T, int D, int GR>
__device__ __forceinline__ void make_rows(const RawRow<T, D>& r, uint4 (&q)[D / 32][Q4Type<T>::PIECES], float (&sums)[D / GR]) {
  constexpr int OP = Q4Type<T>::OP, PIECES = Q4Type<T>::PIECES;
#pragma unroll
  for (int j = 0; j < D / 32; ++j) {
    if constexpr (T::VEC == 8) {
      q[j][0] = r.raw[j][0];
    } else {
      float x[8];
      __builtin_memcpy(x, r.raw[j], sizeof(x));
      uint32_t p[4][3];
#pragma unroll
      for (int e = 0; e < 4; ++e) split_bf16<3>(x[2 * e], x[2 * e + 1], p[e]);
#pragma unroll
      for (int c = 0; c < 3; ++c) q[j][c] = make_uint4(p[0][c], p[1][c], p[2][c], p[3][c]);
    }
  }
  const uint4 ones = make_uint4(kOnes<OP>, kOnes<OP>, kOnes<OP>, kOnes<OP>);
#pragma unroll
  for (int f = 0; f < D / GR; ++f) {
    f32x4q acc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int j = f * (GR / 32); j < (f + 1) * (GR / 32); ++j)
#pragma unroll
      for (int c = 0; c < PIECES; ++c) acc = mfma_q4<OP>(ones, q[j][c], acc);
    sums[f] = acc[0];
  }
}

// Channels 16 j + n of eight slots as an operand: bits 4 (j % 4) of the words of half j / 4 of each pair of slots.
template <int OP, int D>
__device__ __forceinline__ uint4 value_operand(const uint4 (&v)[2], int j, const Q4Magic& magic) {
  uint32_t e[4];
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    const uint32_t w = word_of(v[c / 2], (D / 64) * (c % 2) + j / 4);
    if constexpr (OP != kOpExact) {
      e[c] = q4_pair<OP>(w, j % 4, magic);
    } else {
      const uint32_t two = (w >> (4 * (j % 4))) & 0x000f000fu;
      e[c] = __builtin_amdgcn_perm(f2u((float)(two >> 16)), f2u((float)(two & 0xffffu)), 0x07060302u);
    }
  }
  return make_uint4(e[0], e[1], e[2], e[3]);
}

// Logits (without the scale) of 16 slots, four to a lane, and the rows of q.  rest: the lowest value less the codes' offset in steps.
template <class T, int D, int GR>
__device__ __forceinline__ void rests_of(const uint4 (&scale)[D / GR], float (&rest)[D / GR][4]) {
#pragma unroll
  for (int f = 0; f < D / GR; ++f)
#pragma unroll
    for (int r = 0; r < 4; ++r)
      rest[f][r] = __builtin_fmaf(half_lo(word_of(scale[f], r)), -kOffset<Q4Type<T>::OP>, half_hi(word_of(scale[f], r)));
}
template <class T, int D, int GR>
__device__ __forceinline__ f32x4q logits_of(const uint4 (&k)[D / 32], const uint4 (&scale)[D / GR], const float (&rest)[D / GR][4],
                                            const uint4 (&q)[D / 32][Q4Type<T>::PIECES], const float (&sums)[D / GR]) {
  constexpr int OP = Q4Type<T>::OP, PIECES = Q4Type<T>::PIECES;
  f32x4q x = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int f = 0; f < D / GR; ++f) {
    f32x4q acc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int j = f * (GR / 32); j < (f + 1) * (GR / 32); ++j)
#pragma unroll
      for (int c = 0; c < PIECES; ++c) acc = mfma_q4<OP>(k[j], q[j][c], acc);
#pragma unroll
    for (int r = 0; r < 4; ++r)
      x[r] = __builtin_fmaf(half_lo(word_of(scale[f], r)), acc[r], __builtin_fmaf(rest[f][r], sums[f], x[r]));
  }
  return x;
}

// Four results of neighbouring channels.
template <class T>
__device__ __forceinline__ void store_out(const Kv4Attend& a, int D, int b, int h, int row, int d, const f32x4q& v) {
  const int s = row_token(a, row), i = row - s * a.G;
  typename T::T* dst = reinterpret_cast<typename T::T*>(a.out) + (((int64_t)b * a.S + s) * a.c.H * a.G + h * a.G + i) * D + d;
  if constexpr (T::VEC == 4) {
    *reinterpret_cast<float4*>(dst) = make_float4(v[0], v[1], v[2], v[3]);
  } else {
    uint2 u;
    if constexpr (Q4Type<T>::OP == kOpF16) {
      half2_t x, y;
      x[0] = (_Float16)v[0]; x[1] = (_Float16)v[1]; y[0] = (_Float16)v[2]; y[1] = (_Float16)v[3];
      u = make_uint2(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, y));
    } else {
      u = make_uint2(pk_bf16(v[0], v[1]), pk_bf16(v[2], v[3]));
    }
    *reinterpret_cast<uint2*>(dst) = u;
  }
}

// Slots that a row sees: those before the limit.
__device__ __forceinline__ int row_limit(const Kv4Attend& a, int len, int row) { return min(len, len - a.S + row_token(a, row) + 1); }
// log2 of a row's sum over slots; +infinity where it sees none, so that every probability against it is 0.
__device__ __forceinline__ float log_sum(float m, float l) { return l == 0.0f ? INFINITY : m + __builtin_amdgcn_logf(l); }
__device__ __forceinline__ void store_lse(const Kv4Attend& a, int b, int h, int row, float z) {
  if (!a.lse) return;
  const int s = row_token(a, row), i = row - s * a.G;
  // natural logarithm; -infinity for a row that sees nothing
  a.lse[((int64_t)b * a.S + s) * a.c.H * a.G + h * a.G + i] = z == INFINITY ? -INFINITY : z * 0.69314718055994531f;
}

// How the slots of all sentences are shared out: pieces of `chunk` steps, so that a long sentence among short ones has as many workgroups
// as its length asks for.  Everything follows from lens, in every wave for itself.
struct Shares {
  int chunk;
  __device__ static int steps_of(const Kv4Attend& a, int b) { return (min(max(a.lens[b], 0), a.max_len) + 31) / 32; }
  __device__ int count(int steps) const { return max(1, (steps + chunk - 1) / chunk); }

  __device__ explicit Shares(const Kv4Attend& a) {
    if (a.wanted == 0) {
      chunk = 1 << 30;
      return;
    }
    int64_t total = 0;
    int longest = 0;
    if (a.c.B == 1) {
      total = longest = steps_of(a, 0);
    } else {
      for (int b = threadIdx.x & 63; b < a.c.B; b += 64) {
        const int n = steps_of(a, b);
        total += n;
        longest = max(longest, n);
      }
#pragma unroll
      for (int off = 1; off < 64; off <<= 1) {
        total += __shfl_xor(total, off, kWave);
        longest = max(longest, __shfl_xor(longest, off, kWave));
      }
    }
    // all pieces together are at most wanted + B H: a sentence's last one need not be full
    const int64_t even = (total * a.c.H + a.wanted - 1) / a.wanted, least = max(a.least, (longest + kMaxSplits - 1) / kMaxSplits);
    const int64_t steps = max(even, least);
    chunk = __builtin_amdgcn_readfirstlane((int)((steps + a.token_waves - 1) / a.token_waves * a.token_waves));
  }
  // The sentence of piece `at` and the pieces before that sentence's; b = B where there is no such piece.
  __device__ void find(const Kv4Attend& a, int at, int* b, int* first) const {
    if (a.wanted == 0) {
      *b = at / a.c.H;
      *first = *b * a.c.H;
      return;
    }
    if (a.c.B == 1) {
      *b = at < count(steps_of(a, 0)) * a.c.H ? 0 : 1;
      *first = 0;
      return;
    }
    const int lane = threadIdx.x & 63;
    int base = 0;
    for (int b0 = 0; b0 < a.c.B; b0 += 64) {
      const int mine = b0 + lane < a.c.B ? count(steps_of(a, b0 + lane)) * a.c.H : 0;
      int upto = mine;
#pragma unroll
      for (int off = 1; off < 64; off <<= 1) {
        const int n = __shfl_up(upto, off, kWave);
        if (lane >= off) upto += n;
      }
      const uint64_t past = __ballot(base + upto > at);
      if (past) {
        const int hit = __builtin_ctzll(past);
        *b = b0 + hit;
        *first = base + __shfl(upto - mine, hit, kWave);
        return;
      }
      base += __shfl(upto, 63, kWave);
    }
    *b = a.c.B;
    *first = base;
  }
};

// A row's maximum and sum over its pieces (their values `next` apart), which N neighbouring lanes share; factor[i]: of piece N i + the
// lane's number, against that maximum.
template <int N>
__device__ __forceinline__ void join_pieces(const float* m, const float* l, size_t next, int pieces, float* top, float* total,
                                            float (&factor)[kMaxSplits / N]) {
  const int lane = threadIdx.x % N;
  float mi[kMaxSplits / N], li[kMaxSplits / N], t = -INFINITY, sum = 0.0f;
#pragma unroll
  for (int i = 0; i < kMaxSplits / N; ++i) {
    const int s = lane + N * i;
    mi[i] = s < pieces ? m[s * next] : -INFINITY;
    li[i] = s < pieces ? l[s * next] : 0.0f;
  }
#pragma unroll
  for (int i = 0; i < kMaxSplits / N; ++i) t = fmaxf(t, mi[i]);
#pragma unroll
  for (int off = 1; off < N; off <<= 1) t = fmaxf(t, __shfl_xor(t, off, kWave));
#pragma unroll
  for (int i = 0; i < kMaxSplits / N; ++i) {
    // a piece without a maximum saw nothing, or nothing but NaN
    factor[i] = mi[i] == -INFINITY ? (li[i] != 0.0f ? NAN : 0.0f) : __builtin_amdgcn_exp2f(mi[i] - t);
    sum += mi[i] == -INFINITY ? li[i] : li[i] * factor[i];
  }
#pragma unroll
  for (int off = 1; off < N; off <<= 1) sum += __shfl_xor(sum, off, kWave);
  *top = t;
  *total = sum;
}

// Waves of a SIMD that the registers are to leave room for.
template <class T, int D, int GR> constexpr int kAttendWaves = D / GR == 4 || T::VEC == 4 ? 2 : 3;

// How the four waves of a workgroup share the work: one tile of rows and different slots, their sums joined at the end (storing the logits for
// the weights or not), or the same slots and different tiles; then the cache goes through the LDS as operands, each wave fetching and
// unpacking a quarter of a step for all four.
enum { kSlots, kSlotsAndLogits, kTiles };

template <class T, int D, int GR, int SHARE>
__global__ __launch_bounds__(256, (kAttendWaves<T, D, GR>)) void gemm_q4_attend_kernel(Kv4Attend a) {
  constexpr bool LOGITS = SHARE == kSlotsAndLogits, JOINED = SHARE != kTiles;
  constexpr int OP = Q4Type<T>::OP, OPV = AttendType<T>::OPV, PIECES = Q4Type<T>::PIECES, P = AttendType<T>::P;
  constexpr int NG = D / GR, JK = D / 32, JV = D / 16;
  __shared__ float ml[2][4][16];
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Shares shares(a);
  int b, first;
  shares.find(a, blockIdx.x, &b, &first);
  b = __builtin_amdgcn_readfirstlane(b);
  first = __builtin_amdgcn_readfirstlane(first);
  if (b >= a.c.B) return;
  const int h = ((int)blockIdx.x - first) % a.c.H, split = ((int)blockIdx.x - first) / a.c.H, bh = b * a.c.H + h;
  const int row0 = (JOINED ? (int)blockIdx.y : (int)blockIdx.y * 4 + wave) * 16, row = min(row0 + n, a.R - 1);   // rows past the last repeat it
  const int len = min(max(a.lens[b], 0), a.max_len);
  const int pieces = a.wanted == 0 ? 1 : shares.count((len + 31) / 32);
  if (a.wanted && (int)blockIdx.x == first && blockIdx.y == 0 && threadIdx.x == 0) a.place[b] = make_int2(first, pieces);   // for the join

  // slots that all rows of the wave see, and those that any row of the waves that go together sees
  const int low_limit = row_limit(a, len, min(row0, a.R - 1));
  const int high_limit = row_limit(a, len, min(JOINED ? row0 + 16 : ((int)blockIdx.y + 1) * 64, a.R) - 1);

  const Q4Magic mk = q4_magic<OP>(), mv = q4_magic<OPV>();
  // where the lane's share of a step lies
  const uint32_t* kp = a.c.k + ((size_t)bh * a.c.cap + n) * (D / 8) + g * (D / 32);
  const uint32_t* vp = a.c.v + ((size_t)bh * (a.c.cap / 4) + g) * (D / 2) + n * (D / 32);
  const uint32_t* ksp = a.c.ks + (size_t)bh * NG * a.c.cap + 4 * g;
  const uint32_t* vsp = a.c.vs + (size_t)bh * NG * a.c.cap + 4 * g;
  uint4 k[2], ks[2][NG], v[2], vs[2][NG];
  // Slots: keys and values are each requested again as soon as they have been used: the keys' way is behind the softmax and the values' product,
  // and the other way round, with one set of registers.  (A ring in LDS with twice as much on its way was no faster.)
  auto load_keys = [&](int step) {
    const int t = step * 32;   // t + 32 <= cap, which is whole steps
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      k[i] = ld_row<D>(kp + (size_t)(t + 16 * i) * (D / 8));
#pragma unroll
      for (int f = 0; f < NG; ++f) ks[i][f] = ld16(ksp + (size_t)f * a.c.cap + t + 16 * i);
    }
  };
  auto load_values = [&](int step) {
    const int t = step * 32;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      v[i] = ld_row<D>(vp + (size_t)(t / 4 + 4 * i) * (D / 2));
#pragma unroll
      for (int f = 0; f < NG; ++f) vs[i][f] = ld16(vsp + (size_t)f * a.c.cap + t + 16 * i);
    }
  };
  // Tiles: waves 0 and 1 fetch 16 slots' keys each, 2 and 3 half of the values' channels each, and 16 NG lanes of wave 0 all scales.
  uint4 raw_codes[2], scales;
  constexpr int OPERANDS = 2 * JK + JV;
  uint4 (*operands)[OPERANDS][64] = reinterpret_cast<uint4 (*)[OPERANDS][64]>(smem);   // [2 places][keys of two tiles, values]
  uint4 (*scales_of)[2][2][NG][4] = reinterpret_cast<uint4 (*)[2][2][NG][4]>(smem + 2 * OPERANDS * 1024);
  auto fetch = [&](int step) {
    const int t = step * 32;
    if (wave < 2) {
      raw_codes[0] = ld_row<D>(kp + (size_t)(t + 16 * wave) * (D / 8));
    } else {
#pragma unroll
      for (int i = 0; i < 2; ++i) raw_codes[i] = ld_row<D>(vp + (size_t)(t / 4 + 4 * i) * (D / 2));
    }
    if (threadIdx.x < 16 * NG) {
      const int which = threadIdx.x / (8 * NG), i = threadIdx.x / (4 * NG) % 2, f = threadIdx.x / 4 % NG, quad = threadIdx.x % 4;
      scales = ld16((which ? a.c.vs : a.c.ks) + ((size_t)bh * NG + f) * a.c.cap + t + 16 * i + 4 * quad);
    }
  };
  auto exchange = [&](int place) {
    if (wave < 2) {
#pragma unroll
      for (int j = 0; j < JK; ++j) operands[place][wave * JK + j][lane] = q4_operand<OP>(word_of(raw_codes[0], j), mk);
    } else {
#pragma unroll
      for (int j = 0; j < JV; ++j)
        if (j / (JV / 2) == wave - 2) operands[place][2 * JK + j][lane] = value_operand<OPV, D>(raw_codes, j, mv);
    }
    if (threadIdx.x < 16 * NG) (&scales_of[place][0][0][0][0])[threadIdx.x] = scales;
    __syncthreads();   // two places by turns: one barrier a step
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int f = 0; f < NG; ++f) ks[i][f] = scales_of[place][0][i][f][g], vs[i][f] = scales_of[place][1][i][f][g];
  };
  const int begin = split ? split * shares.chunk : 0;   // one piece: the chunk may be anything
  const int step0 = begin + (JOINED ? wave : 0), stride = JOINED ? 4 : 1;
  const int end = pieces == 1 ? 1 << 30 : begin + shares.chunk, steps = min(end, (max(high_limit, 0) + 31) / 32);
  const uint4 ones = make_uint4(kOnes<OPV>, kOnes<OPV>, kOnes<OPV>, kOnes<OPV>);

  if (step0 < steps) {
    if constexpr (JOINED) {
      load_keys(step0);
      load_values(step0);
    } else {
      fetch(step0);
    }
  }
  uint4 q[JK][PIECES];
  float sums[NG];
  {
    RawRow<T, D> raw;
    load_raw<T, D>(a, b, h, row, raw);
    make_rows<T, D, GR>(raw, q, sums);
  }
  const int limit = row_limit(a, len, row);

  f32x4q o[JV], one[NG];
  float m = -INFINITY, l = 0.0f, low[NG];
#pragma unroll
  for (int f = 0; f < NG; ++f) one[f] = f32x4q{0.0f, 0.0f, 0.0f, 0.0f}, low[f] = 0.0f;
#pragma unroll
  for (int j = 0; j < JV; ++j) o[j] = f32x4q{0.0f, 0.0f, 0.0f, 0.0f};

  auto fold = [&] {   // the constants that entered with the codes, and the lowest values, over the lanes of a row
#pragma unroll
    for (int f = 0; f < NG; ++f) {
      float c = low[f] + __shfl_xor(low[f], 16, kWave);
      c += __shfl_xor(c, 32, kWave);
      if constexpr (OPV != kOpExact) c = __builtin_fmaf(-kOffset<OPV>, one[f][0], c);
#pragma unroll
      for (int j = f * (GR / 16); j < (f + 1) * (GR / 16); ++j) o[j] += c;
      low[f] = 0.0f;
      one[f] = f32x4q{0.0f, 0.0f, 0.0f, 0.0f};
    }
  };
  int unfolded = 0;

  for (int step = step0; step < steps; step += stride) {
    const int t0 = step * 32, after = min(step + stride, steps - 1);
    const bool partial = t0 + 32 > low_limit;
    if constexpr (!JOINED) {
      exchange(step & 1);
      fetch(after);
    }
    float x[8];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      uint4 kop[JK];
#pragma unroll
      for (int j = 0; j < JK; ++j) kop[j] = JOINED ? q4_operand<OP>(word_of(k[i], j), mk) : operands[step & 1][i * JK + j][lane];
      float rest[NG][4];
      rests_of<T, D, GR>(ks[i], rest);
      const f32x4q y = logits_of<T, D, GR>(kop, ks[i], rest, q, sums);
#pragma unroll
      for (int r = 0; r < 4; ++r) x[4 * i + r] = y[r];
    }
    if constexpr (JOINED) load_keys(after);
    if (partial) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (t0 + 16 * (i / 4) + 4 * g + i % 4 >= limit) x[i] = -INFINITY;
      // no probability of a slot that the row does not see meets its step and lowest value, which may be anything
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int see = limit - (t0 + 16 * i + 4 * g);
#pragma unroll
        for (int f = 0; f < NG; ++f) {
          vs[i][f].x = see > 0 ? vs[i][f].x : 0;
          vs[i][f].y = see > 1 ? vs[i][f].y : 0;
          vs[i][f].z = see > 2 ? vs[i][f].z : 0;
          vs[i][f].w = see > 3 ? vs[i][f].w : 0;
        }
      }
    }
    if constexpr (LOGITS) {   // one tile of rows
      if (n < a.R) {
        float4* dst = reinterpret_cast<float4*>(a.logits + ((size_t)bh * a.R + n) * ((a.max_len + 31) / 32 * 32) + t0 + 4 * g);
        dst[0] = make_float4(x[0] * a.scale, x[1] * a.scale, x[2] * a.scale, x[3] * a.scale);
        dst[4] = make_float4(x[4] * a.scale, x[5] * a.scale, x[6] * a.scale, x[7] * a.scale);
      }
    }
    float top = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7]))) * a.scale;
    if (__any(top > m + 8.0f)) {
      top = fmaxf(top, __shfl_xor(top, 16, kWave));
      top = fmaxf(top, __shfl_xor(top, 32, kWave));
      top = fmaxf(top, m);
      const float f = top == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m - top);
      m = top;
      l *= f;
#pragma unroll
      for (int e = 0; e < NG; ++e) {
        low[e] *= f;
        one[e] *= f;
      }
#pragma unroll
      for (int j = 0; j < JV; ++j) o[j] *= f;
    }
    const float base = m == -INFINITY ? 0.0f : m;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      x[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[i], a.scale, -base));
      l += x[i];
    }
    // group by group: the probabilities times the group's steps, in pieces, and their products with the group's channels
#pragma unroll
    for (int e = 0; e < NG; ++e) {
      uint4 piece[P];
      uint32_t p[4][P];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t s0 = word_of(vs[i / 2][e], 2 * (i % 2)), s1 = word_of(vs[i / 2][e], 2 * (i % 2) + 1);
        low[e] = __builtin_fmaf(half_hi(s0), x[2 * i], low[e]);
        low[e] = __builtin_fmaf(half_hi(s1), x[2 * i + 1], low[e]);
        split_bf16<P>(half_lo(s0) * x[2 * i], half_lo(s1) * x[2 * i + 1], p[i]);
      }
#pragma unroll
      for (int c = 0; c < P; ++c) {
        piece[c] = make_uint4(p[0][c], p[1][c], p[2][c], p[3][c]);
        if constexpr (OPV != kOpExact) one[e] = mfma_q4<OPV>(ones, piece[c], one[e]);
      }
#pragma unroll
      for (int j = e * (GR / 16); j < (e + 1) * (GR / 16); ++j) {
        const uint4 vop = JOINED ? value_operand<OPV, D>(v, j, mv) : operands[step & 1][2 * JK + j][lane];
#pragma unroll
        for (int c = 0; c < P; ++c) o[j] = mfma_q4<OPV>(vop, piece[c], o[j]);
      }
    }
    if constexpr (JOINED) load_values(after);
    if (++unfolded == kFold<OPV>) {
      fold();
      unfolded = 0;
    }
  }

  l += __shfl_xor(l, 16, kWave);
  l += __shfl_xor(l, 32, kWave);
  fold();
  const size_t part = (size_t)blockIdx.x * a.row_tiles * 16;
  if constexpr (!JOINED) {
    if (row0 + n >= a.R) return;
    if (pieces > 1) {
      if (g == 0) a.m[part + row] = m, a.l[part + row] = l;
#pragma unroll
      for (int j = 0; j < JV; ++j)
        *reinterpret_cast<float4*>(a.o + (part + row) * D + 16 * j + 4 * g) = make_float4(o[j][0], o[j][1], o[j][2], o[j][3]);
    } else {
      const float inv = l == 0.0f ? 0.0f : 1.0f / l, z = log_sum(m, l);
#pragma unroll
      for (int j = 0; j < JV; ++j) store_out<T>(a, D, b, h, row, 16 * j + 4 * g, o[j] * inv);
      if (g == 0) {
        store_lse(a, b, h, row, z);
        if (a.weights) a.z[(size_t)bh * a.R + row] = z;
      }
    }
    return;
  }

  // the waves' sums
  float4* shared = reinterpret_cast<float4*>(smem);   // [wave][j][lane]
  if (g == 0) ml[0][wave][n] = m, ml[1][wave][n] = l;
  __syncthreads();
  if (row0 + n < a.R) {
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < 4; ++w) top = fmaxf(top, ml[0][w][n]);
    const float f = m == -INFINITY ? (l != l ? l : 0.0f) : __builtin_amdgcn_exp2f(m - top);   // a row of NaNs stays one
#pragma unroll
    for (int j = 0; j < JV; ++j)
      shared[(wave * JV + j) * 64 + lane] = make_float4(o[j][0] * f, o[j][1] * f, o[j][2] * f, o[j][3] * f);
  }
  __syncthreads();
  for (int i = threadIdx.x; i < min(16, a.R - row0) * (D / 4); i += 256) {
    const int col = i / (D / 4), d = i % (D / 4) * 4, row = row0 + col, at = d / 16 * 64 + d % 16 / 4 * 16 + col;
    float top = -INFINITY, total = 0.0f;
#pragma unroll
    for (int w = 0; w < 4; ++w) top = fmaxf(top, ml[0][w][col]);
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float mw = ml[0][w][col], lw = ml[1][w][col];
      total += mw == -INFINITY ? lw : lw * __builtin_amdgcn_exp2f(mw - top);   // no maximum: 0, or NaN
    }
    f32x4q v = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float4 s = shared[w * JV * 64 + at];
      v[0] += s.x; v[1] += s.y; v[2] += s.z; v[3] += s.w;
    }
    if (pieces > 1) {
      *reinterpret_cast<f32x4q*>(a.o + (part + row) * D + d) = v;
      if (d == 0) a.m[part + row] = top, a.l[part + row] = total;
    } else {
      const float z = log_sum(top, total);
      store_out<T>(a, D, b, h, row, d, v * (total == 0.0f ? 0.0f : 1.0f / total));
      if (d == 0) {
        store_lse(a, b, h, row, z);
        if (a.weights) a.z[(size_t)bh * a.R + row] = z;
      }
    }
  }
}

// The pieces' results in their order (workgroups x < join_blocks), and the weights that up to 16 rows give each slot, from the stored logits
// (the others, 256 slots each).  Latency is all of it, so whatever does not depend on the rows' sums is requested ahead of them, and
// workgroups are a wave each, for as many as possible to wait at a time.
template <class T, int D>
__global__ __launch_bounds__(64) void kv4_join_kernel(Kv4Attend a, int join_blocks) {
  const int bh = blockIdx.y, b = bh / a.c.H, h = bh % a.c.H;
  const int2 place = a.wanted == 0 ? make_int2(b * a.c.H, 1) : a.place[b];
  const int pieces = place.y;
  const size_t next = (size_t)a.c.H * a.row_tiles * 16, base = ((size_t)place.x + h) * a.row_tiles * 16;
  if ((int)blockIdx.x < join_blocks) {
    if (pieces == 1) return;   // written where it was computed
    constexpr int N = D / 4, ROWS = 64 / N, AHEAD = 8;   // lanes of a row
    const int r = blockIdx.x * ROWS + threadIdx.x / N, row = min(r, a.R - 1), d = threadIdx.x % N * 4;
    const size_t at = base + row;
    f32x4q p[AHEAD], v = {0.0f, 0.0f, 0.0f, 0.0f};
    auto piece = [&](int s) { return *reinterpret_cast<const f32x4q*>(a.o + (at + s * next) * D + d); };
#pragma unroll
    for (int s = 0; s < AHEAD; ++s) p[s] = piece(min(s, pieces - 1));
    float top, total, factor[kMaxSplits / N];
    join_pieces<N>(a.m + at, a.l + at, next, pieces, &top, &total, factor);
    auto factor_of = [&](float f, int s) { return __shfl(f, (threadIdx.x & 63) / N * N + s % N, kWave); };
#pragma unroll
    for (int s = 0; s < AHEAD; ++s) {
      const float f = factor_of(factor[0], s);
      if (s < pieces) v += p[s] * f;
    }
#pragma unroll
    for (int i = 0; i < kMaxSplits / N; ++i)
#pragma unroll 8
      for (int s = max(AHEAD, N * i); s < min(pieces, N * (i + 1)); ++s) v += piece(s) * factor_of(factor[i], s);
    if (r >= a.R) return;
    const float z = log_sum(top, total);
    store_out<T>(a, D, b, h, row, d, v * (total == 0.0f ? 0.0f : 1.0f / total));
    if (d == 0) {
      store_lse(a, b, h, row, z);
      if (a.weights == 2) a.z[(size_t)bh * a.R + row] = z;
    }
    return;
  }
  __shared__ float zs[16];
  const int len = min(max(a.lens[b], 0), a.max_len);
  const int t0 = ((int)blockIdx.x - join_blocks) * 256 + threadIdx.x * 4, pitch = (a.max_len + 31) / 32 * 32;
  if (t0 - (int)threadIdx.x * 4 >= len) return;   // the whole workgroup
  const float* logits = a.logits + (size_t)bh * a.R * pitch + min(t0, pitch - 4);
  const float* before = a.c.weight + (size_t)bh * a.c.cap + min(t0, pitch - 4);
  constexpr int AHEAD = 4;
  f32x4q x[AHEAD];
#pragma unroll
  for (int r = 0; r < AHEAD; ++r) x[r] = *reinterpret_cast<const f32x4q*>(logits + (size_t)min(r, a.R - 1) * pitch);
  float w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = before[i];
  if (pieces > 1) {
    const int r = threadIdx.x >> 2;   // four lanes a row
    const size_t at = base + min(r, a.R - 1);
    float top, total, factor[kMaxSplits / 4];
    join_pieces<4>(a.m + at, a.l + at, next, pieces, &top, &total, factor);
    if ((threadIdx.x & 3) == 0) zs[r] = log_sum(top, total);
  } else if ((int)threadIdx.x < a.R) {
    zs[threadIdx.x] = a.z[(size_t)bh * a.R + threadIdx.x];
  }
  __syncthreads();
  f32x4q sum = {0.0f, 0.0f, 0.0f, 0.0f};
  auto add = [&](int r, const f32x4q& y) {
    if (t0 >= row_limit(a, len, r)) return;   // also: no logits were stored there
#pragma unroll
    for (int i = 0; i < 4; ++i) sum[i] += __builtin_amdgcn_exp2f(y[i] - zs[r]);
  };
#pragma unroll
  for (int r = 0; r < AHEAD; ++r)
    if (r < a.R) add(r, x[r]);
#pragma unroll 4
  for (int r = AHEAD; r < a.R; ++r) add(r, *reinterpret_cast<const f32x4q*>(logits + (size_t)r * pitch));
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (t0 + i < len) a.weight_out[(size_t)bh * a.c.cap + t0 + i] = w[i] + sum[i];
}

// Weights of many rows: the logits are computed again, 32 slots a wave against all rows that see them, and every slot's sum stays in its
// lane until the end, so there is no order to depend on and nothing of S x T is stored.  The rows go through the LDS, each wave fetching
// a quarter of a tile of 16 for all four: every wave fetching its own is bound by the L2 (512 rows, 2048 slots, 32 heads: 36 us; of 16 slots
// a wave 64).
template <class T, int D, int GR>
__global__ __launch_bounds__(256) void gemm_q4_weights_kernel(Kv4Attend a) {
  constexpr int OP = Q4Type<T>::OP, PIECES = Q4Type<T>::PIECES, NG = D / GR, JK = D / 32, V = 8 / T::VEC;
  __shared__ uint4 tile_of_q[2][JK][V][64];
  const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int bh = blockIdx.x, b = bh / a.c.H, h = bh % a.c.H;   // heads fastest: a head's rows stay in one L2
  const int len = min(max(a.lens[b], 0), a.max_len);
  const int t_block = (int)(blockIdx.z * gridDim.y + blockIdx.y) * 128, t0 = t_block + wave * 32;
  if (t_block >= len) return;   // the whole workgroup; t0 + 32 may pass len, but not a multiple of 32 that holds it, so not the capacity
  const bool idle = t0 >= len;
  const Q4Magic mk = q4_magic<OP>();
  const int from = idle ? t_block : t0;
  const uint32_t* kp = a.c.k + ((size_t)bh * a.c.cap + from + n) * (D / 8) + g * (D / 32);
  const uint32_t* ksp = a.c.ks + (size_t)bh * NG * a.c.cap + from + 4 * g;
  uint4 kop[2][JK], ks[2][NG];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint4 k = ld_row<D>(kp + (size_t)(16 * i) * (D / 8));
#pragma unroll
    for (int j = 0; j < JK; ++j) kop[i][j] = q4_operand<OP>(word_of(k, j), mk);
#pragma unroll
    for (int f = 0; f < NG; ++f) ks[i][f] = ld16(ksp + (size_t)f * a.c.cap + 16 * i);
  }
  float rest[2][NG][4];
#pragma unroll
  for (int i = 0; i < 2; ++i) rests_of<T, D, GR>(ks[i], rest[i]);
  float w[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
  const int first = max(0, t_block - (len - a.S)) * a.G / 16;   // rows of earlier tiles see none of these slots
  uint4 mine[V];
  float z = 0.0f;
  auto request = [&](int tile) {
    const int row = min(tile * 16 + n, a.R - 1);
    if (JK == 4 || wave < JK) load_channels<T>(a, b, h, row, 32 * wave + 8 * g, mine);
    z = a.z[(size_t)bh * a.R + row];
  };
  if (first < a.row_tiles) request(first);
  for (int tile = first; tile < a.row_tiles; ++tile) {
    const int at = tile & 1;   // two places by turns: one barrier a tile
    if (JK == 4 || wave < JK)
#pragma unroll
      for (int v = 0; v < V; ++v) tile_of_q[at][wave][v][lane] = mine[v];
    const float zr = tile * 16 + n < a.R ? z : INFINITY;
    __syncthreads();
    request(min(tile + 1, a.row_tiles - 1));   // ahead of its use
    RawRow<T, D> raw;
#pragma unroll
    for (int j = 0; j < JK; ++j)
#pragma unroll
      for (int v = 0; v < V; ++v) raw.raw[j][v] = tile_of_q[at][j][v][lane];
    uint4 q[JK][PIECES];
    float sums[NG];
    make_rows<T, D, GR>(raw, q, sums);
    const int limit = idle ? 0 : row_limit(a, len, min(tile * 16 + n, a.R - 1));
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const f32x4q x = logits_of<T, D, GR>(kop[i], ks[i], rest[i], q, sums);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(x[r], a.scale, -zr));
        w[4 * i + r] += t0 + 16 * i + 4 * g + r < limit ? p : 0.0f;
      }
    }
  }
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int off = 1; off < 16; off <<= 1) w[i] += __shfl_xor(w[i], off, kWave);
  if (n == 0)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int t = t0 + 16 * (i / 4) + 4 * g + i % 4;
      const size_t at = (size_t)bh * a.c.cap + t;
      if (t < len) a.weight_out[at] = a.c.weight[at] + w[i];
    }
}

template <class T, int D, int GR, int SHARE>
int launch_attend(const Kv4Attend& a, hipStream_t s) {
  const int tiles = (a.R + 15) / 16, per = SHARE == kTiles ? 4 : 1;
  const dim3 grid(a.blocks, (tiles + per - 1) / per);
  const size_t lds = SHARE == kTiles ? 2 * (D / 8) * 1024 + 2 * 16 * (D / GR) * 16 : 4 * D * 64;   // D / 16 operands each
  hipLaunchKernelGGL((gemm_q4_attend_kernel<T, D, GR, SHARE>), grid, dim3(256), lds, s, a);
  CI_HIP_CHECK_LAUNCH();
  if (a.wanted || a.weights == 1) {
    constexpr int ROWS = 64 / (D / 4);
    const int join = a.wanted ? (a.R + ROWS - 1) / ROWS : 0, weight = a.weights == 1 ? (a.max_len + 255) / 256 : 0;
    hipLaunchKernelGGL((kv4_join_kernel<T, D>), dim3(join + weight, a.c.B * a.c.H), dim3(64), 0, s, a, join);
    CI_HIP_CHECK_LAUNCH();
  }
  if (a.weights == 2) {
    // up to 2^16 heads and 2^17 workgroups along the slots: together more threads than one dimension of a launch may have, of which the rest
    // would be left out without an error
    const uint32_t along = (uint32_t)(a.max_len + 127) / 128, most = 32768;
    hipLaunchKernelGGL((gemm_q4_weights_kernel<T, D, GR>), dim3(a.c.B * a.c.H, along < most ? along : most, (along + most - 1) / most), dim3(256),
                       0, s, a);
    CI_HIP_CHECK_LAUNCH();
  }
  return CI_OK;
}

template <class T, int D, int GR>
int launch_attend_rows(const Kv4Attend& a, hipStream_t s) {
  if (a.token_waves == 1) return launch_attend<T, D, GR, kTiles>(a, s);
  return a.weights == 1 ? launch_attend<T, D, GR, kSlotsAndLogits>(a, s) : launch_attend<T, D, GR, kSlots>(a, s);
}

}  // namespace

template <class T>
int launch_kv4_attend_type(const Kv4Attend& a, int D, int group, hipStream_t s) {
  if (D == 64) return group == 32 ? launch_attend_rows<T, 64, 32>(a, s) : launch_attend_rows<T, 64, 64>(a, s);
  if (group == 32) return launch_attend_rows<T, 128, 32>(a, s);
  return group == 64 ? launch_attend_rows<T, 128, 64>(a, s) : launch_attend_rows<T, 128, 128>(a, s);
}

}  // namespace ci
