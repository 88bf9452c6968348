// Writing keys and values to a cache in 4 bits, reading them back, and evicting the slots that got the least weight (kv4.hpp).
// All three are bound by the bytes they move, or, for single tokens, by their launches.
#include <algorithm>

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
template <class T, int D, int GR>
__global__ __launch_bounds__(128) void kv4_append_kernel(AppendArgs a) {
  constexpr int LPT = D / 8, TP = 64 / LPT, PASSES = 16 / TP, NG = D / GR;
  __shared__ __attribute__((aligned(16))) uint8_t code[16][D];  // of the values, on the way to their quads
  const int lane = threadIdx.x & 63, h = blockIdx.y, b = blockIdx.z;
  const bool values = threadIdx.x >= 64;
  const int64_t len = a.lens[b], from = len - a.S;   // slot of the first token
  const int64_t start = a.start ? a.start[b] : 0;
  const int64_t first = max(max(from, start), (int64_t)0), last = min(len, (int64_t)a.c.cap);
  const int64_t slot0 = (first / 16 + blockIdx.x) * 16;
  if (slot0 >= last) return;   // the whole workgroup
  const size_t head = (size_t)b * a.c.H + h;
  const typename T::T* src = reinterpret_cast<const typename T::T*>(values ? a.v : a.k) + b * a.s_b + h * a.s_h;
  uint32_t* scales = (values ? a.c.vs : a.c.ks) + head * NG * a.c.cap;
  const int d0 = (lane % LPT) * 8;
#pragma unroll
  for (int p = 0; p < PASSES; ++p) {
    const int at = p * TP + lane / LPT;
    const int64_t slot = slot0 + at;
    const bool in = slot >= first && slot < last;
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = 0.0f;
    if (in) {
      const typename T::T* row = src + (slot - from) * a.s_s + d0;
      if (a.vectors) {
        float f[T::VEC];
#pragma unroll
        for (int i = 0; i < 8 / T::VEC; ++i) {
          unpack<T>(ld16(row + i * T::VEC), f);
#pragma unroll
          for (int e = 0; e < T::VEC; ++e) x[i * T::VEC + e] = f[e];
        }
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = to_float<T>(row[e]);
      }
    }
    float lo = x[0], hi = x[0];
#pragma unroll
    for (int e = 1; e < 8; ++e) lo = min_nan(lo, x[e]), hi = max_nan(hi, x[e]);
#pragma unroll
    for (int off = 1; off < GR / 8; off <<= 1) {
      lo = min_nan(lo, __shfl_xor(lo, off, kWave));
      hi = max_nan(hi, __shfl_xor(hi, off, kWave));
    }
    const uint32_t scale = q4_scale(lo, hi);
    uint32_t n[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) n[e] = q4_code(x[e], scale);
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

struct EvictArgs {
  Kv4 c;
  const int32_t *lens, *next;
  int32_t* lens_out;
  float* weight_out;
  int32_t* pos_out;
  int recent, budget, max_len, max_moves;
  int32_t *count, *holes, *movers;   // [B H], [B H, max_moves] twice
};

constexpr int kPlanThreads = 1024;

// Exclusive sum over the workgroup of a pair of counts below 2^32 in one word each; all threads take part.
__device__ __forceinline__ uint64_t block_scan(uint64_t x, uint64_t* sums, uint64_t* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint64_t v = x;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const uint64_t u = __shfl_up(v, off, kWave);
    if (lane >= off) v += u;
  }
  __syncthreads();
  if (lane == 63) sums[wave] = v;
  __syncthreads();
  uint64_t before = 0, all = 0;
  for (int w = 0; w < kPlanThreads / 64; ++w) {
    const uint64_t s = sums[w];
    before += w < wave ? s : 0;
    all += s;
  }
  *total = all;
  return before + v - x;
}

// Which slots of a head stay, which move where.  Keys: the last `recent` positions first, then by weight, NaN last; equal keys by the
// lower slot.  CACHED: the keys of a head are kept in the LDS.
template <bool CACHED>
__global__ __launch_bounds__(kPlanThreads) void kv4_plan_kernel(EvictArgs a) {
  extern __shared__ uint32_t cache[];
  __shared__ uint32_t hist[2048];
  __shared__ uint64_t sums[kPlanThreads / 64];
  __shared__ uint32_t chosen[2];
  const int tid = threadIdx.x, b = blockIdx.x / a.c.H;
  const size_t head = blockIdx.x;
  const float* weight = a.c.weight + head * a.c.cap;
  const int32_t* pos = a.c.pos + head * a.c.cap;
  float* weight_out = a.weight_out + head * a.c.cap;
  int32_t* pos_out = a.pos_out + head * a.c.cap;
  const int len = min(max(a.lens[b], 0), a.max_len);
  const bool copy = weight_out != weight, copy_pos = pos_out != pos;
  if (len <= a.budget) {
    for (int t = tid; t < len; t += kPlanThreads) {
      if (copy) weight_out[t] = weight[t];
      if (copy_pos) pos_out[t] = pos[t];
    }
    if (tid == 0) a.count[head] = 0;
    return;
  }
  const int64_t protect = (int64_t)a.next[b] - a.recent;
  auto make_key = [&](int t) -> uint32_t {
    if (pos[t] >= protect) return 0xffffffffu;
    const float w = weight[t];
    if (w != w) return 0u;
    const uint32_t u = f2u(w + 0.0f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
  };
  if (CACHED) {
    for (int t = tid; t < len; t += kPlanThreads) cache[t] = make_key(t);
    __syncthreads();
  }
  auto key_at = [&](int t) { return CACHED ? cache[t] : make_key(t); };

  // the budget-th largest key, eleven bits at a time, and how many equal to it are kept
  uint32_t prefix = 0, want = (uint32_t)a.budget;
#pragma unroll
  for (int pass = 0; pass < 3; ++pass) {
    const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bins = pass == 2 ? 1024 : 2048;
    for (int i = tid; i < bins; i += kPlanThreads) hist[i] = 0;
    __syncthreads();
    for (int t = tid; t < len; t += kPlanThreads) {
      const uint32_t key = key_at(t);
      if (pass == 0 || key >> (pass == 1 ? 21 : 10) == prefix) atomicAdd(&hist[key >> shift & (uint32_t)(bins - 1)], 1u);
    }
    __syncthreads();
    // two bins a thread, from the largest down
    const int i0 = bins - 1 - 2 * tid;
    uint32_t c0 = 0, c1 = 0;
    if (i0 > 0) c0 = hist[i0], c1 = hist[i0 - 1];
    uint64_t total;
    const uint64_t before = block_scan(c0 + c1, sums, &total);
    if (before < want && before + c0 + c1 >= want) {
      const bool second = before + c0 < want;
      chosen[0] = (uint32_t)(second ? i0 - 1 : i0);
      chosen[1] = want - (uint32_t)before - (second ? c0 : 0);
    }
    __syncthreads();
    prefix = pass == 0 ? chosen[0] : prefix << (pass == 1 ? 11 : 10) | chosen[0];
    want = chosen[1];
    __syncthreads();
  }

  // a run of slots a thread: the equal ones before it, then the holes and the slots that move
  const int run = ((len + kPlanThreads - 1) / kPlanThreads) | 1;   // odd: the runs start in different banks
  const int t0 = min(tid * run, len), t1 = min(t0 + run, len);
  uint32_t equal = 0;
  for (int t = t0; t < t1; ++t) equal += key_at(t) == prefix;
  uint64_t total;
  const uint32_t equal_before = (uint32_t)block_scan(equal, sums, &total);
  auto walk = [&](auto&& hole, auto&& mover) {
    uint32_t e = equal_before;
    for (int t = t0; t < t1; ++t) {
      const uint32_t key = key_at(t);
      const bool kept = key > prefix || (key == prefix && e < want);
      e += key == prefix;
      if (!kept && t < a.budget) hole(t);
      if (kept && t >= a.budget) mover(t);
    }
  };
  uint64_t mine = 0;
  walk([&](int) { mine += 1; }, [&](int) { mine += 1ull << 32; });
  const uint64_t at = block_scan(mine, sums, &total);
  int32_t* holes = a.holes + head * a.max_moves;
  int32_t* movers = a.movers + head * a.max_moves;
  uint32_t ih = (uint32_t)at, im = (uint32_t)(at >> 32);
  walk([&](int t) { holes[ih++] = t; }, [&](int t) { movers[im++] = t; });
  const int moves = (int)(uint32_t)total;   // as many holes as slots that move
  if (tid == 0) a.count[head] = moves;
  __syncthreads();   // the lists, and every read of a weight or position for a key
  if (copy || copy_pos)
    for (int t = tid; t < a.budget; t += kPlanThreads) {
      if (copy) weight_out[t] = weight[t];
      if (copy_pos) pos_out[t] = pos[t];
    }
  __syncthreads();
  for (int i = tid; i < moves; i += kPlanThreads) {
    const int to = holes[i], of = movers[i];
    weight_out[to] = weight[of];
    pos_out[to] = pos[of];
  }
  __syncthreads();
  for (int t = a.budget + tid; t < len; t += kPlanThreads) {
    weight_out[t] = 0.0f;
    pos_out[t] = -1;
  }
}

// Sixteen lanes a move: a row of keys, the half-words of the values, the scales.  Sources lie from the budget on and places below it.
template <int D, int GR>
__global__ __launch_bounds__(256) void kv4_move_kernel(EvictArgs a) {
  constexpr int NG = D / GR;
  const size_t head = blockIdx.y;
  if (blockIdx.x == 0 && head % a.c.H == 0 && threadIdx.x == 0 && a.lens_out) {
    const int b = (int)(head / a.c.H);
    a.lens_out[b] = min(min(max(a.lens[b], 0), a.max_len), a.budget);
  }
  const int i = blockIdx.x * 16 + (threadIdx.x >> 4), n = threadIdx.x & 15;
  if (i >= a.count[head]) return;
  const size_t to = a.holes[head * a.max_moves + i], of = a.movers[head * a.max_moves + i], cap = a.c.cap;
  uint32_t* k = a.c.k + head * cap * (D / 8);
  if (n < D / 8) k[to * (D / 8) + n] = k[of * (D / 8) + n];
  uint16_t* v = reinterpret_cast<uint16_t*>(a.c.v + head * cap * (D / 8));
  auto half = [&](size_t slot, int f) { return (slot / 4 * 16 + n) * (D / 16) + 2 * ((D / 64) * ((slot & 3) >> 1) + f) + (slot & 1); };
#pragma unroll
  for (int f = 0; f < D / 64; ++f) v[half(to, f)] = v[half(of, f)];
  if (n < 2 * NG) {
    uint32_t* s = (n < NG ? a.c.ks : a.c.vs) + (head * NG + n % NG) * cap;
    s[to] = s[of];
  }
}

constexpr int kCachedKeys = 32768;

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
    hipLaunchKernelGGL((kv4_append_kernel<T, D, GR>), dim3((a.S + 14) / 16 + 1, a.c.H, a.c.B), dim3(128), 0, s, a);
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

struct MoveLaunch {
  EvictArgs a;
  hipStream_t s;
  template <class T, int D, int GR>
  int operator()() const {
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
  if (max_len <= kCachedKeys) {
    static std::atomic<uint64_t> seen{0};
    const size_t lds = (size_t)max_len * sizeof(uint32_t);
    if (lds > 40960) {   // with the kernel's own, more than a launch may have unasked
      const int rc = allow_dynamic_lds(seen, reinterpret_cast<const void*>(kv4_plan_kernel<true>), kCachedKeys * sizeof(uint32_t));
      if (rc != CI_OK) return rc;
    }
    hipLaunchKernelGGL(kv4_plan_kernel<true>, dim3((uint32_t)heads), dim3(kPlanThreads), lds, s, a);
  } else {
    hipLaunchKernelGGL(kv4_plan_kernel<false>, dim3((uint32_t)heads), dim3(kPlanThreads), 0, s, a);
  }
  CI_HIP_CHECK_LAUNCH();
  return by_shape<F32>(c.D, c.group, MoveLaunch{a, s});
}

}  // namespace ci
