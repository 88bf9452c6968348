// Writing keys and values to a cache in 4 bits, reading them back, and evicting the slots that got the least weight (kv4.hpp).
// Reading is bound by its bytes (8 x 40 heads x 1024 slots, 220 MB: 46 us, 4.8 TB/s); writing from a few hundred tokens on by the packing's
// instructions, about half of it, and by the rows' latency (1023 tokens of 32 heads 12.3 us, 6.4 of them instructions; four waves a SIMD, which
// wait in half of their cycles), and by latency alone below (one token of 8 x 72 heads 4.0 us); eviction by the chain of barriers
// in which a head's slots are chosen (one of 1025 slots 6 us with its move, 6144 of 8192 21 us and 18 for the moves).
#include <algorithm>
#include <type_traits>

#include "kv4.hpp"

namespace ci {
namespace {

// ---- writing ---------------------------------------------------------------------------------------------------------------------

struct AppendArgs {
  Kv4 c;
  const void *k, *v;
  int64_t s_b, s_s, s_h;  // strides of k and v in elements
  const int32_t *start, *lens, *next;
  int S, vectors;
};

// A workgroup has 16 slots of a head: one wave their keys, the other their values.  A slot's D channels are held by D / 8 neighbouring lanes.
// Workgroups that run together have neighbouring heads, whose rows are neighbours in memory.
template <class T, int D, int GR>
__global__ __launch_bounds__(128) void kv4_append_kernel(AppendArgs a) {
  constexpr int LPT = D / 8, TP = 64 / LPT, PASSES = 16 / TP, NG = D / GR;
  __shared__ __attribute__((aligned(16))) uint8_t code[16][D];  // of the values, on the way to their quads
  const int lane = threadIdx.x & 63, h = blockIdx.x, b = blockIdx.z;
  const bool values = threadIdx.x >= 64;
  const int64_t len = a.lens[b], from = len - a.S;   // slot of the first token
  const int64_t start = a.start ? a.start[b] : 0;
  const int64_t first = max(max(from, start), (int64_t)0), last = min(len, (int64_t)a.c.cap);
  const int64_t slot0 = (first / 16 + blockIdx.y) * 16;
  if (slot0 >= last) return;   // the whole workgroup
  const size_t head = (size_t)b * a.c.H + h;
  const typename T::T* src = reinterpret_cast<const typename T::T*>(values ? a.v : a.k) + b * a.s_b + h * a.s_h;
  uint32_t* scales = (values ? a.c.vs : a.c.ks) + head * NG * a.c.cap;
  const int d0 = (lane % LPT) * 8;
  // all rows on their way before the first is used; slots that are not written read a neighbour's
  uint4 raw[PASSES][8 / T::VEC];
  auto any_in = [&](int p) { return slot0 + (p + 1) * TP > first && slot0 + p * TP < last; };
#pragma unroll
  for (int p = 0; p < PASSES; ++p) {
    if (!any_in(p)) continue;
    const int64_t slot = min(max(slot0 + p * TP + lane / LPT, first), last - 1);
    const typename T::T* row = src + (slot - from) * a.s_s + d0;
    if (a.vectors) {
#pragma unroll
      for (int i = 0; i < 8 / T::VEC; ++i) raw[p][i] = ld16(row + i * T::VEC);
    } else {
      typename T::T e[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) e[i] = row[i];
      __builtin_memcpy(raw[p], e, sizeof(e));
    }
  }
#pragma unroll
  for (int p = 0; p < PASSES; ++p) {
    if (!any_in(p)) continue;   // nothing of its places in the LDS is used
    const int at = p * TP + lane / LPT;
    const int64_t slot = slot0 + at;
    const bool in = slot >= first && slot < last;
    float x[8];
#pragma unroll
    for (int i = 0; i < 8 / T::VEC; ++i) {
      float f[T::VEC];
      unpack<T>(raw[p][i], f);
#pragma unroll
      for (int e = 0; e < T::VEC; ++e) x[i * T::VEC + e] = f[e];
    }
    float lo = x[0], hi = x[0];
#pragma unroll
    for (int e = 1; e < 8; ++e) lo = min_nan(lo, x[e]), hi = max_nan(hi, x[e]);
    // over the lanes of a group, by moves within sixteen lanes: the neighbour, the other pair, the other four, the other eight
    auto both = [&](auto ctrl) {
      lo = min_nan(lo, u2f((uint32_t)__builtin_amdgcn_mov_dpp((int)f2u(lo), decltype(ctrl)::value, 0xf, 0xf, true)));
      hi = max_nan(hi, u2f((uint32_t)__builtin_amdgcn_mov_dpp((int)f2u(hi), decltype(ctrl)::value, 0xf, 0xf, true)));
    };
    both(std::integral_constant<int, 0xb1>{});
    both(std::integral_constant<int, 0x4e>{});
    if constexpr (GR >= 64) both(std::integral_constant<int, 0x141>{});
    if constexpr (GR >= 128) both(std::integral_constant<int, 0x140>{});
    const uint32_t scale = q4_scale(lo, hi);
    uint32_t n[8];
    q4_codes(x, scale, n);
    if (in && d0 % GR == 0) scales[(size_t)(d0 / GR) * a.c.cap + slot] = scale;
    if (values) {
      *reinterpret_cast<uint2*>(&code[at][d0]) = make_uint2(n[0] | n[1] << 8 | n[2] << 16 | n[3] << 24,
                                                            n[4] | n[5] << 8 | n[6] << 16 | n[7] << 24);
    } else if (in) {
      uint32_t word = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) word |= n[e] << (4 * q4_nibble(e));
      const int j = d0 / 32, g = d0 / 8 % 4;
      a.c.k[(head * a.c.cap + slot) * (D / 8) + (D / 32) * g + j] = word;
      if (d0 == 0) {
        if (a.c.weight) a.c.weight[head * a.c.cap + slot] = 0.0f;
        if (a.c.pos) a.c.pos[head * a.c.cap + slot] = (int32_t)((a.next ? (int64_t)a.next[b] : len) - a.S + (slot - from));
      }
    }
  }
  __syncthreads();
  if (!values) return;
  // lane 16 q + n: quad q's word pairs of n
  const int n = lane & 15, q = lane >> 4;
  const int64_t quad = slot0 / 4 + q;
  uint32_t half[4][D / 64];
#pragma unroll
  for (int t = 0; t < 4; ++t)
#pragma unroll
    for (int f = 0; f < D / 64; ++f) {
      half[t][f] = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) half[t][f] |= (uint32_t)code[4 * q + t][64 * f + 16 * i + n] << (4 * i);
    }
  uint32_t* dst = a.c.v + ((head * (a.c.cap / 4) + quad) * 16 + n) * (D / 32);
  if (quad * 4 >= first && quad * 4 + 4 <= last) {
    if constexpr (D == 128)
      *reinterpret_cast<uint4*>(dst) = make_uint4(half[0][0] | half[1][0] << 16, half[0][1] | half[1][1] << 16,
                                                  half[2][0] | half[3][0] << 16, half[2][1] | half[3][1] << 16);
    else
      *reinterpret_cast<uint2*>(dst) = make_uint2(half[0][0] | half[1][0] << 16, half[2][0] | half[3][0] << 16);
  } else {
#pragma unroll
    for (int t = 0; t < 4; ++t)
      if (quad * 4 + t >= first && quad * 4 + t < last)
#pragma unroll
        for (int f = 0; f < D / 64; ++f)
          reinterpret_cast<uint16_t*>(dst)[2 * ((D / 64) * (t >> 1) + f) + (t & 1)] = (uint16_t)half[t][f];
  }
}

// ---- reading ---------------------------------------------------------------------------------------------------------------------

// Slots first .. first + count - 1 as values of type T, [B, H, count, D]; zeros from the sentence's length on.
template <class T, int D, int GR>
__global__ __launch_bounds__(128) void kv4_read_kernel(Kv4 c, const int32_t* lens, int first, int count, typename T::T* k,
                                                       typename T::T* v) {
  constexpr int LPT = D / 8, TP = 64 / LPT, PASSES = 16 / TP, NG = D / GR;
  __shared__ __attribute__((aligned(16))) uint8_t code[16][D];
  const int lane = threadIdx.x & 63, h = blockIdx.y, b = blockIdx.z;
  const bool values = threadIdx.x >= 64;
  const int slot0 = (first / 16 + (int)blockIdx.x) * 16, end = first + count;   // end <= cap, which is whole tiles
  const int len = min(max(lens[b], 0), c.cap);
  const size_t head = (size_t)b * c.H + h;
  if (values) {
    const int n = lane & 15, q = lane >> 4;
    const uint32_t* src = c.v + ((head * (c.cap / 4) + slot0 / 4 + q) * 16 + n) * (D / 32);
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int f = 0; f < D / 64; ++f) {
        const uint32_t half = src[(D / 64) * (t >> 1) + f] >> (16 * (t & 1));
#pragma unroll
        for (int i = 0; i < 4; ++i) code[4 * q + t][64 * f + 16 * i + n] = (half >> (4 * i)) & 15u;
      }
  }
  __syncthreads();
  const uint32_t* scales = (values ? c.vs : c.ks) + head * NG * c.cap;
  const int d0 = (lane % LPT) * 8;
#pragma unroll
  for (int p = 0; p < PASSES; ++p) {
    const int at = p * TP + lane / LPT, slot = slot0 + at;
    if (slot < first || slot >= end) continue;
    uint32_t n[8];
    if (values) {
#pragma unroll
      for (int e = 0; e < 8; ++e) n[e] = code[at][d0 + e];
    } else {
      const uint32_t word = c.k[(head * c.cap + slot) * (D / 8) + (D / 32) * (d0 / 8 % 4) + d0 / 32];
#pragma unroll
      for (int e = 0; e < 8; ++e) n[e] = (word >> (4 * q4_nibble(e))) & 15u;
    }
    const uint32_t scale = scales[(size_t)(d0 / GR) * c.cap + slot];
    typename T::T* dst = (values ? v : k) + ((head * count + (slot - first)) * D + d0);
    typename T::T y[8] __attribute__((aligned(16)));
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = slot < len ? from_float<T>(q4_value(n[e], scale)) : from_float<T>(0.0f);
#pragma unroll
    for (int i = 0; i < 8 / T::VEC; ++i) reinterpret_cast<uint4*>(dst)[i] = reinterpret_cast<const uint4*>(y)[i];
  }
}

// ---- eviction --------------------------------------------------------------------------------------------------------------------

constexpr int kFew = 4;
constexpr int kMovedHere = 256;  // moves of a head that the workgroup which plans them does itself

struct EvictArgs {
  Kv4 c;
  const int32_t *lens, *next;
  int32_t* lens_out;
  float* weight_out;
  int32_t* pos_out;
  int recent, budget, max_len, max_moves;
  int32_t *count, *holes, *movers;   // [B H], [B H, max_moves] twice
};

// Inclusive sum over the lanes of a wave, without the LDS.
__device__ __forceinline__ uint32_t wave_scan(uint32_t v) {
  auto add = [&](auto ctrl, auto rows) {
    v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, decltype(ctrl)::value, decltype(rows)::value, 0xf, false);
  };
  constexpr std::integral_constant<int, 0xf> all{};
  add(std::integral_constant<int, 0x111>{}, all);   // from 1, 2, 4 and 8 lanes below within sixteen
  add(std::integral_constant<int, 0x112>{}, all);
  add(std::integral_constant<int, 0x114>{}, all);
  add(std::integral_constant<int, 0x118>{}, all);
  add(std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xa>{});   // the sums of the sixteens before
  add(std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xc>{});
  return v;
}

// The least (LEAST) or greatest of a wave's values, in every lane.
template <bool LEAST>
__device__ __forceinline__ uint32_t wave_extreme(uint32_t v) {
  auto with = [&](auto ctrl, auto rows) {
    const uint32_t u = (uint32_t)__builtin_amdgcn_update_dpp(LEAST ? -1 : 0, (int)v, decltype(ctrl)::value, decltype(rows)::value, 0xf, false);
    v = LEAST ? min(v, u) : max(v, u);
  };
  constexpr std::integral_constant<int, 0xf> all{};
  with(std::integral_constant<int, 0x111>{}, all);
  with(std::integral_constant<int, 0x112>{}, all);
  with(std::integral_constant<int, 0x114>{}, all);
  with(std::integral_constant<int, 0x118>{}, all);
  with(std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xa>{});
  with(std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xc>{});
  return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}

// Exclusive sums over the workgroup; all threads take part.  sums: THREADS / 64 words that no other call uses.  Returns the total.
template <int THREADS>
__device__ __forceinline__ uint32_t block_scan(uint32_t x, uint32_t* sums, uint32_t* before) {
  const uint32_t v = wave_scan(x);
  const int wave = threadIdx.x >> 6;
  if ((threadIdx.x & 63) == 63) sums[wave] = v;
  __syncthreads();
  uint32_t lower = 0, all = 0;
#pragma unroll
  for (int w = 0; w < THREADS / 64; ++w) {
    const uint32_t s = sums[w];
    lower += w < wave ? s : 0;
    all += s;
  }
  *before = lower + v - x;
  return all;
}

// A head's slot moved to another: sixteen lanes take the row of keys, the half-words of the values, the scales.
template <int D, int GR>
__device__ __forceinline__ void move_slot(const Kv4& c, size_t head, size_t to, size_t of, int n) {
  constexpr int NG = D / GR;
  const size_t cap = c.cap;
  uint32_t* k = c.k + head * cap * (D / 8);
  uint16_t* v = reinterpret_cast<uint16_t*>(c.v + head * cap * (D / 8));
  uint32_t* s = (n < NG ? c.ks : c.vs) + (head * NG + n % NG) * cap;
  auto half = [&](size_t slot, int f) { return (slot / 4 * 16 + n) * (D / 16) + 2 * ((D / 64) * ((slot & 3) >> 1) + f) + (slot & 1); };
  const uint32_t kw = n < D / 8 ? k[of * (D / 8) + n] : 0, sw = n < 2 * NG ? s[of] : 0;
  uint16_t vw[D / 64];
#pragma unroll
  for (int f = 0; f < D / 64; ++f) vw[f] = v[half(of, f)];
  if (n < D / 8) k[to * (D / 8) + n] = kw;
#pragma unroll
  for (int f = 0; f < D / 64; ++f) v[half(to, f)] = vw[f];
  if (n < 2 * NG) s[to] = sw;
}

// Which slots of a head stay, which move where.  Keys: the last `recent` positions first, then by weight, NaN last; equal keys by the
// lower slot.  The budget-th key is found eleven bits at a time from histograms in the LDS; the recent ones, all alike, and zeros, of which
// there may be many, are counted by wave, or every lane would wait for all others at one bin.  CACHED: the keys of a head are kept in
// the LDS.  MOVE: the rows are moved here as well (few of them, and nobody reads a length that this launch writes), from lists in the LDS, whose
// 16 bits a slot hold what CACHED allows.  FEW: no more than
// kFew slots can leave, as in a cache that is cut at every step, so these are looked for one by one (one of 1025 slots of 320 heads: 6 us
// instead of 13).
template <int THREADS, bool CACHED, int D, int GR, bool MOVE, bool FEW>
__global__ __launch_bounds__(THREADS) void kv4_plan_kernel(EvictArgs a) {
  static_assert(CACHED || !MOVE, "without lists in the LDS the moves are another launch's, from those in memory");
  extern __shared__ uint32_t cache[];
  constexpr int kBins = 2048;
  __shared__ __attribute__((aligned(16))) uint32_t hist[3][kBins];   // of the three passes; the last uses half of its
  __shared__ uint32_t sums[6][THREADS / 64], chosen[3][2], recents;
  constexpr uint32_t kRecent = 0xffffffffu, kZero = 0x80000000u;
  const int tid = threadIdx.x, lane = tid & 63, h = blockIdx.x % a.c.H, b = blockIdx.x / a.c.H;
  const size_t head = blockIdx.x;
  const float* weight = a.c.weight + head * a.c.cap;
  const int32_t* pos = a.c.pos + head * a.c.cap;
  float* weight_out = a.weight_out + head * a.c.cap;
  int32_t* pos_out = a.pos_out + head * a.c.cap;
  const int len = min(max(a.lens[b], 0), a.max_len);
  const bool copy = weight_out != weight, copy_pos = pos_out != pos;
  if (MOVE && h == 0 && tid == 0 && a.lens_out) a.lens_out[b] = min(len, a.budget);
  if (len <= a.budget) {
    for (int t = tid; t < len; t += THREADS) {
      if (copy) weight_out[t] = weight[t];
      if (copy_pos) pos_out[t] = pos[t];
    }
    if (!MOVE && tid == 0) a.count[head] = 0;
    return;
  }
  const int64_t protect = (int64_t)a.next[b] - a.recent;
  auto key_of = [&](float w, int p) -> uint32_t {
    if (p >= protect) return kRecent;
    if (w != w) return 0u;
    const uint32_t u = f2u(w + 0.0f);   // one zero
    return u & 0x80000000u ? ~u : u | 0x80000000u;
  };
  auto key_at = [&](int t) { return CACHED ? cache[t] : key_of(weight[t], pos[t]); };
  for (int i = tid; i < 3 * kBins / 4; i += THREADS) reinterpret_cast<uint4*>(hist)[i] = make_uint4(0, 0, 0, 0);
  if (tid == 0) recents = 0;
  __syncthreads();
  // what does not depend on the choice goes out at once: slots that stay, and those cleared, unless their old values are yet to move
  constexpr int AHEAD = 8;   // all loads of a round before its first store, which might be to the same place for all the compiler knows
  for (int t0 = tid; t0 - tid < len; t0 += AHEAD * THREADS) {
    float w[AHEAD];
    int32_t p[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      const int t = min(t0 + i * THREADS, len - 1);
      w[i] = weight[t];
      p[i] = pos[t];
    }
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      const int t = t0 + i * THREADS;
      const bool in = t < len;
      const uint32_t key = key_of(w[i], p[i]);
      if (CACHED && in) cache[t] = key;
      const uint64_t all = __ballot(in && key == kRecent);
      if (lane == 0 && all) atomicAdd(&recents, (uint32_t)__popcll(all));
      if (in && copy) weight_out[t] = t < a.budget ? w[i] : 0.0f;
      if (in && copy_pos) pos_out[t] = t < a.budget ? p[i] : -1;
    }
  }
  __syncthreads();

  // lists of the moves: in the LDS, where the histograms were, if they fit there (16 bits a slot)
  constexpr int kListed = 3 * kBins * 4 / 4, WAVES = THREADS / 64;
  uint16_t* lists = reinterpret_cast<uint16_t*>(hist);
  int32_t* holes = a.holes + head * a.max_moves;
  int32_t* movers = a.movers + head * a.max_moves;
  const int wave = tid >> 6;
  int moves;
  bool small;
  if constexpr (FEW) {
    static_assert(MOVE, "rows moved here");
    __shared__ uint32_t least[2][WAVES][2];   // by turns: one barrier a slot
    int gone[kFew];
#pragma unroll
    for (int r = 0; r < kFew; ++r) {
      gone[r] = -1;
      if (r >= len - a.budget) continue;
      uint32_t key = kRecent, place = 0;   // of the last of the least, its number counted from one
      for (int t = tid; t < len; t += THREADS) {
        bool left = false;
#pragma unroll
        for (int q = 0; q < r; ++q) left |= t == gone[q];
        const uint32_t k = cache[t];
        if (!left && k <= key) key = k, place = (uint32_t)t + 1;
      }
      const uint32_t wave_key = wave_extreme<true>(key), wave_place = wave_extreme<false>(key == wave_key ? place : 0u);
      if (lane == 0) least[r & 1][wave][0] = wave_key, least[r & 1][wave][1] = wave_place;
      __syncthreads();
      key = kRecent, place = 0;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) {
        const uint32_t k = least[r & 1][w][0], at = least[r & 1][w][1];
        place = k < key ? at : k == key ? max(place, at) : place;
        key = min(key, k);
      }
      gone[r] = (int)place - 1;
    }
    // the holes in ascending order, and the slots from the budget on that have not left
    small = true;
    moves = 0;
#pragma unroll
    for (int r = 0; r < kFew; ++r) {
      if (gone[r] < 0 || gone[r] >= a.budget) continue;
      int before = 0;
#pragma unroll
      for (int q = 0; q < kFew; ++q) before += gone[q] >= 0 && gone[q] < gone[r];
      if (tid == 0) lists[before] = (uint16_t)gone[r];
      ++moves;
    }
    int of = 0;
    for (int t = a.budget; t < len; ++t) {
      bool left = false;
#pragma unroll
      for (int q = 0; q < kFew; ++q) left |= t == gone[q];
      if (left) continue;
      if (tid == 0) lists[kListed + of] = (uint16_t)t;
      ++of;
    }
  } else {
    uint32_t prefix = 0, want = (uint32_t)a.budget;
    if (recents >= want) {
      prefix = kRecent;
    } else {
      want -= recents;
#pragma unroll
      for (int pass = 0; pass < 3; ++pass) {
        const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
        const uint32_t mask = pass == 2 ? 1023u : 2047u;
#pragma unroll 4
        for (int t0 = 0; t0 < len; t0 += THREADS) {
          const int t = t0 + tid;
          const uint32_t key = t < len ? key_at(t) : kRecent;
          const bool in = key != kRecent && (pass == 0 || key >> (pass == 1 ? 21 : 10) == prefix);
          if (!__any(in)) continue;   // most rounds of the later passes
          const uint64_t zeros = __ballot(in && key == kZero);
          if (zeros && lane == 0) atomicAdd(&hist[pass][kZero >> shift & mask], (uint32_t)__popcll(zeros));
          if (in && key != kZero) atomicAdd(&hist[pass][key >> shift & mask], 1u);
        }
        __syncthreads();
        // a run of bins a thread, from the largest down
        constexpr int RUN = kBins / THREADS;
        const int i0 = kBins - RUN * (tid + 1);
        uint32_t c[RUN], mine = 0, before;
#pragma unroll
        for (int i = 0; i < RUN; ++i) c[i] = hist[pass][i0 + RUN - 1 - i], mine += c[i];
        block_scan<THREADS>(mine, sums[pass], &before);
        if (before < want && before + mine >= want) {
          int i = 0;
#pragma unroll
          for (int j = 0; j < RUN - 1; ++j)
            if (i == j && before + c[j] < want) before += c[j], ++i;
          chosen[pass][0] = (uint32_t)(i0 + RUN - 1 - i);
          chosen[pass][1] = want - before;
        }
        __syncthreads();
        prefix = pass == 0 ? chosen[pass][0] : prefix << (pass == 1 ? 11 : 10) | chosen[pass][0];
        want = chosen[pass][1];
      }
    }

    // A stretch of slots a wave, 64 at a time in order: the equal ones before it, then the holes and the slots that move, counted by ballots.
    const int stretch = ((len + THREADS - 1) / THREADS) * 64;
    const int t0 = wave * stretch, t1 = min(t0 + stretch, len);
    const uint64_t lower = lanemask_lt();
    auto over_waves = [&](uint32_t mine, uint32_t* of, uint32_t* all) {   // the sum over the waves before this one; a barrier
      if (lane == 0) of[wave] = mine;
      __syncthreads();
      uint32_t sum = 0, total = 0;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) {
        sum += w < wave ? of[w] : 0;
        total += of[w];
      }
      *all = total;
      return sum;
    };
    uint32_t equal = 0, total;
#pragma unroll 4
    for (int t = t0 + lane; t - lane < t1; t += 64) equal += (uint32_t)__popcll(__ballot(t < t1 && key_at(t) == prefix));
    const uint32_t equal_before = over_waves(equal, sums[3], &total);
    auto walk = [&](auto&& visit) {   // visit(slot, is a hole, moves)
      uint32_t e = equal_before;
#pragma unroll 4
      for (int t = t0 + lane; t - lane < t1; t += 64) {
        const uint32_t key = t < t1 ? key_at(t) : 0u;
        const uint64_t same = __ballot(t < t1 && key == prefix);
        const bool kept = key > prefix || (key == prefix && e + (uint32_t)__popcll(same & lower) < want);
        e += (uint32_t)__popcll(same);
        visit(t, t < t1 && !kept && t < a.budget, t < t1 && kept && t >= a.budget);
      }
    };
    uint32_t n_holes = 0, n_movers = 0;
    walk([&](int, bool hole, bool mover) {
      n_holes += (uint32_t)__popcll(__ballot(hole));
      n_movers += (uint32_t)__popcll(__ballot(mover));
    });
    uint32_t ih, im;
    im = over_waves(n_movers, sums[4], &total);
    ih = over_waves(n_holes, sums[5], &total);   // as many holes as slots that move
    moves = (int)total;
    // rows that are not moved here need the lists in memory too
    small = CACHED && moves <= kListed;
    walk([&](int t, bool hole, bool mover) {
      const uint64_t all_holes = __ballot(hole), all_movers = __ballot(mover);
      const uint32_t to = ih + (uint32_t)__popcll(all_holes & lower), of = im + (uint32_t)__popcll(all_movers & lower);
      if (hole) {
        if (small) lists[to] = (uint16_t)t;
        if (!MOVE) holes[to] = t;
      }
      if (mover) {
        if (small) lists[kListed + of] = (uint16_t)t;
        if (!MOVE) movers[of] = t;
      }
      ih += (uint32_t)__popcll(all_holes);
      im += (uint32_t)__popcll(all_movers);
    });
    if (!MOVE && tid == 0) a.count[head] = moves;
  }
  auto hole_at = [&](int i) { return small ? (int)lists[i] : holes[i]; };
  auto mover_at = [&](int i) { return small ? (int)lists[kListed + i] : movers[i]; };
  __syncthreads();   // the lists, every read of a weight or position for a key, and what the copies stored
  if constexpr (MOVE)
    for (int i = tid >> 4; i < moves; i += THREADS / 16) move_slot<D, GR>(a.c, head, hole_at(i), mover_at(i), tid & 15);
  for (int i0 = tid; i0 < moves; i0 += 4 * THREADS) {
    int to[4], p[4];
    float w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int i = min(i0 + j * THREADS, moves - 1), of = mover_at(i);
      to[j] = hole_at(i);
      w[j] = weight[of];
      p[j] = pos[of];
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (i0 + j * THREADS < moves) {
        weight_out[to[j]] = w[j];
        pos_out[to[j]] = p[j];
      }
  }
  if (copy && copy_pos) return;
  __syncthreads();
  for (int t = a.budget + tid; t < len; t += THREADS) {
    if (!copy) weight_out[t] = 0.0f;
    if (!copy_pos) pos_out[t] = -1;
  }
}

// Sixteen lanes a move.  Sources lie from the budget on and places below it.
template <int D, int GR>
__global__ __launch_bounds__(256) void kv4_move_kernel(EvictArgs a) {
  const size_t head = blockIdx.y;
  if (blockIdx.x == 0 && head % a.c.H == 0 && threadIdx.x == 0 && a.lens_out) {
    const int b = (int)(head / a.c.H);
    a.lens_out[b] = min(min(max(a.lens[b], 0), a.max_len), a.budget);
  }
  const int i = blockIdx.x * 16 + (threadIdx.x >> 4);
  if (i >= a.count[head]) return;
  move_slot<D, GR>(a.c, head, a.holes[head * a.max_moves + i], a.movers[head * a.max_moves + i], threadIdx.x & 15);
}

constexpr int kCachedKeys = 32768;   // 128 KB of the LDS

template <class T, class F>
int by_shape(int D, int group, F&& f) {
  if (D == 64) return group == 32 ? f.template operator()<T, 64, 32>() : f.template operator()<T, 64, 64>();
  if (group == 32) return f.template operator()<T, 128, 32>();
  return group == 64 ? f.template operator()<T, 128, 64>() : f.template operator()<T, 128, 128>();
}
template <class F>
int by_type(int dtype, int D, int group, F&& f) {
  switch (dtype) {
    case CI_F32: return by_shape<F32>(D, group, f);
    case CI_F16: return by_shape<F16>(D, group, f);
    default: return by_shape<BF16>(D, group, f);
  }
}

struct AppendLaunch {
  AppendArgs a;
  hipStream_t s;
  template <class T, int D, int GR>
  int operator()() const {
    hipLaunchKernelGGL((kv4_append_kernel<T, D, GR>), dim3(a.c.H, (a.S + 14) / 16 + 1, a.c.B), dim3(128), 0, s, a);
    CI_HIP_CHECK_LAUNCH();
    return CI_OK;
  }
};

struct ReadLaunch {
  Kv4 c;
  const int32_t* lens;
  int first, count;
  void *k, *v;
  hipStream_t s;
  template <class T, int D, int GR>
  int operator()() const {
    const int tiles = (first + count + 15) / 16 - first / 16;
    hipLaunchKernelGGL((kv4_read_kernel<T, D, GR>), dim3(tiles, c.H, c.B), dim3(128), 0, s, c, lens, first, count,
                       reinterpret_cast<typename T::T*>(k), reinterpret_cast<typename T::T*>(v));
    CI_HIP_CHECK_LAUNCH();
    return CI_OK;
  }
};

struct EvictLaunch {
  EvictArgs a;
  hipStream_t s;
  bool here;
  template <int THREADS, bool CACHED, int D, int GR, bool MOVE, bool FEW>
  int plan() const {
    auto* kernel = kv4_plan_kernel<THREADS, CACHED, D, GR, MOVE, FEW>;
    const size_t lds = CACHED ? (size_t)a.max_len * sizeof(uint32_t) : 0;
    static std::atomic<uint64_t> seen{0};
    if (lds > 32768) {   // with the kernel's own, more than a launch may have unasked
      const int rc = allow_dynamic_lds(seen, reinterpret_cast<const void*>(kernel), kCachedKeys * sizeof(uint32_t));
      if (rc != CI_OK) return rc;
    }
    hipLaunchKernelGGL(kernel, dim3(a.c.B * a.c.H), dim3(THREADS), lds, s, a);
    CI_HIP_CHECK_LAUNCH();
    return CI_OK;
  }
  template <int D, int GR, bool MOVE>
  int plan_any() const {   // MOVE: max_len <= kCachedKeys
    if constexpr (MOVE)
      if (a.max_len - a.budget <= kFew)
        return a.max_len <= 2048 ? plan<256, true, D, GR, true, true>() : plan<1024, true, D, GR, true, true>();
    // a wave's share of the steps against the barriers' cost
    if (a.max_len <= 2048) return plan<256, true, D, GR, MOVE, false>();
    if constexpr (!MOVE)
      if (a.max_len > kCachedKeys) return plan<1024, false, D, GR, false, false>();
    return plan<1024, true, D, GR, MOVE, false>();
  }
  template <class T, int D, int GR>
  int operator()() const {
    if (here) return plan_any<D, GR, true>();
    const int rc = plan_any<D, GR, false>();
    if (rc != CI_OK) return rc;
    hipLaunchKernelGGL((kv4_move_kernel<D, GR>), dim3((std::max(a.max_moves, 1) + 15) / 16, a.c.B * a.c.H), dim3(256), 0, s, a);
    CI_HIP_CHECK_LAUNCH();
    return CI_OK;
  }
};

Kv4 kv4_of(const ci_kv4& c) {
  return Kv4{reinterpret_cast<uint32_t*>(c.k), reinterpret_cast<uint32_t*>(c.v), c.k_scale, c.v_scale, c.weight, c.pos,
             (int)c.B, (int)c.H, (int)c.cap};
}

// A slot moves only into a hole below the budget and only from above it.
int64_t moves_bound(int64_t max_len, int64_t budget) { return std::max<int64_t>(0, std::min(budget, max_len - budget)); }
size_t words256(size_t n) { return (n + 63) / 64 * 64; }

}  // namespace

int launch_kv4_append(const ci_kv4& c, const void* k, const void* v, int64_t S, const int64_t (&stride)[3], int dtype,
                      const int32_t* start, const int32_t* lens, const int32_t* next, hipStream_t s) {
  const int e = elem_bytes(dtype);
  const int vectors = aligned16(k) && aligned16(v) && stride[0] * e % 16 == 0 && stride[1] * e % 16 == 0 && stride[2] * e % 16 == 0;
  return by_type(dtype, c.D, c.group,
                 AppendLaunch{{kv4_of(c), k, v, stride[0], stride[1], stride[2], start, lens, next, (int)S, vectors}, s});
}

int launch_kv4_read(const ci_kv4& c, const int32_t* lens, int64_t first, int64_t count, void* k, void* v, int dtype, hipStream_t s) {
  return by_type(dtype, c.D, c.group, ReadLaunch{kv4_of(c), lens, (int)first, (int)count, k, v, s});
}

size_t kv4_evict_ws_bytes(int64_t heads, int64_t max_len, int64_t budget) {
  return (words256(heads) + 2 * words256((size_t)heads * moves_bound(max_len, budget))) * sizeof(int32_t);
}

int launch_kv4_evict(const ci_kv4& c, const int32_t* lens, const int32_t* next, int64_t max_len, int64_t budget, int64_t recent,
                     float* weight_out, int32_t* pos_out, int32_t* lens_out, void* ws, hipStream_t s) {
  EvictArgs a;
  a.c = kv4_of(c);
  a.lens = lens;
  a.next = next;
  a.lens_out = lens_out;
  a.weight_out = weight_out;
  a.pos_out = pos_out;
  a.recent = (int)recent;
  a.budget = (int)budget;
  a.max_len = (int)max_len;
  a.max_moves = (int)moves_bound(max_len, budget);
  const size_t heads = (size_t)c.B * c.H;
  a.count = reinterpret_cast<int32_t*>(ws);
  a.holes = a.count + words256(heads);
  a.movers = a.holes + words256(heads * a.max_moves);
  // In one launch where a workgroup's own moves are few and the keys fit the LDS, unless it would write what others have yet to read.
  auto apart = [&](const int32_t* in) {
    const uintptr_t from = reinterpret_cast<uintptr_t>(in), to = reinterpret_cast<uintptr_t>(lens_out), bytes = c.B * sizeof(int32_t);
    return !lens_out || to + bytes <= from || from + bytes <= to;
  };
  const bool here = max_len <= kCachedKeys && a.max_moves <= kMovedHere && apart(lens) && apart(next);
  return by_shape<F32>(c.D, c.group, EvictLaunch{a, s, here});
}

}  // namespace ci
