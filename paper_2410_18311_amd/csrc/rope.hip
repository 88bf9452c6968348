// Rotary positions with norms of heads (coreinfer_rope), and keys and values written to a cache in pages on the same way
// (coreinfer_kvp_append): a pair (a, c) of channels at position p becomes scale (a cos - c sin, c cos + a sin) of the angle p f.
//
// Both are bound by their bytes, or by the latency of one launch.  A lane holds two vectors of 16 bytes of a head, the two halves of its pairs
// (neighbouring pairs: two vectors of whole pairs), so a head is D / 2 elements' lanes and its norm a sum over them.  The sines and cosines are a token's,
// not a head's: a workgroup takes one or two tokens, computes each pair's once (one pair a thread) and hands them round through the LDS.
//
// Angles are whole 2^-64ths of a turn, so position times frequency is one 64-bit product whose overflow is whole turns: exact at any position.
// Its nearest quarter turn is taken off as bits; what is left, at most an eighth of a turn, goes through the Taylor series, whose
// first terms left out are below 2^-28.
//
// 4096 tokens of 40 heads of 128, bf16: 16.2 to 18 us for 84 MB, 4.7 to 5.2 TB/s, the rate of a large copy; 3584 tokens of 96 heads to pages 39.5 us for 176 MB.
// One token: 2.5 us of the kernel, 4.9 with the search for its sentence and page, the rest of a call's 5 to 7 us its launch.
#include <algorithm>

#include "kvp.hpp"

namespace ci {
namespace {

// One kind of heads of a call: queries, keys or values.
struct Heads {
  const void* x;
  void* y;                  // NULL: the slot of a page
  int64_t x_t, x_h, y_t, y_h;   // strides in elements
  const void* norm;
  int count, turned;
};
struct RopeCall {
  Heads kind[3];
  Kvp cache;
  const int32_t *pos, *first, *lens;
  const uint64_t* turns;
  float scale, sign, eps;
  int T, D, rot, heads;
  int lanes, tokens, per_group;   // lanes of a head (a power of two), tokens of a workgroup, heads of a workgroup and token
};

// The sine and cosine of turns p / 2^64 of a turn.
__device__ __forceinline__ void sin_cos(uint64_t turns, int p, float* sin, float* cos) {
  const uint64_t t = turns * (uint64_t)(int64_t)p;
  const int quarter = (int)((t + (1ull << 61)) >> 62);
  const int64_t rest = (int64_t)(t - ((uint64_t)quarter << 62));      // -2^61 .. 2^61
  const float r = (float)(int)(rest >> 30);                            // 2^-34ths of a turn
  // 2 pi / 2^34 in two parts
  const float a = __builtin_fmaf(r, 3.6572953e-10f, r * -1.0177351e-17f), q = a * a;
  float s = __builtin_fmaf(q, 2.75573192e-6f, -1.98412698e-4f);
  s = __builtin_fmaf(q, s, 8.33333333e-3f);
  s = __builtin_fmaf(q, s, -1.66666667e-1f);
  s = __builtin_fmaf(a * q, s, a);
  float c = __builtin_fmaf(q, -2.75573192e-7f, 2.48015873e-5f);
  c = __builtin_fmaf(q, c, -1.38888889e-3f);
  c = __builtin_fmaf(q, c, 4.16666667e-2f);
  c = __builtin_fmaf(q, c, -0.5f);
  c = __builtin_fmaf(q, c, 1.0f);
  const float x = quarter & 1 ? -s : c, y = quarter & 1 ? c : s;
  *cos = quarter & 2 ? -x : x;
  *sin = quarter & 2 ? -y : y;
}

// Where a token's keys and values go, and its position.
struct Place {
  int64_t at;   // elements from the pages' start to the slot of head 0; -1: nowhere
  int pos, mine;   // mine: the token is some sentence's
};
__device__ __forceinline__ Place place_of(const RopeCall& a, int t) {
  Place p{-1, 0, 0};
  int b, from, to, len;
  if (a.cache.B <= 64) {
    // everything that the sentence may be asked for comes with the search
    const int lane = threadIdx.x & 63, own = a.first[min(lane, a.cache.B)], next = a.first[min(lane + 1, a.cache.B)],
              held = a.lens[min(lane, a.cache.B - 1)];
    b = __popcll(__ballot(lane == 0 || (lane < a.cache.B && own <= t))) - 1;
    from = __builtin_amdgcn_readlane(own, b);
    to = __builtin_amdgcn_readlane(next, b);
    len = __builtin_amdgcn_readlane(held, b);
  } else {
    b = sentence_of(a.first, a.cache.B, t);
    from = a.first[b];
    to = a.first[b + 1];
    len = a.lens[b];
  }
  from = clamp_row(from, a.T);
  to = clamp_row(to, a.T);
  const int64_t slot = (int64_t)len - (to - from) + (t - from);
  if (t < from || t >= to) return p;
  p.mine = 1;
  p.pos = (int)slot;
  if (slot >= 0 && slot < (a.cache.most << a.cache.shift)) {
    const int64_t page = a.cache.table[b * a.cache.most + (slot >> a.cache.shift)];
    if ((uint64_t)page < a.cache.pages)
      p.at = ((page * a.cache.H << a.cache.shift) + (slot & ((1 << a.cache.shift) - 1))) * a.D;
  }
  return p;
}

template <class E>
__device__ __forceinline__ uint4 pack(const float (&f)[E::VEC]) {
  typename E::T x[E::VEC];
#pragma unroll
  for (int e = 0; e < E::VEC; ++e) x[e] = from_float<E>(f[e]);
  uint4 u;
  __builtin_memcpy(&u, x, sizeof(u));
  return u;
}

// A head's number among all kinds of heads as its kind and its number there.
__device__ __forceinline__ int kind_of(const RopeCall& a, int* head) {
  int kind = 0;
  if (*head >= a.kind[0].count) {
    *head -= a.kind[0].count;
    kind = 1;
    if (*head >= a.kind[1].count) {
      *head -= a.kind[1].count;
      kind = 2;
    }
  }
  return kind;
}

template <class E>
__device__ __forceinline__ const typename E::T* source(const RopeCall& a, const Heads& k, int t, int head) {
  return reinterpret_cast<const typename E::T*>(k.x) + t * k.x_t + head * k.x_h;
}
// NULL: nowhere
template <class E, bool APPEND>
__device__ __forceinline__ typename E::T* target(const RopeCall& a, const Heads& k, int which, int t, int head, const Place& p) {
  if (!APPEND || which == 0) return APPEND && !p.mine ? nullptr : reinterpret_cast<typename E::T*>(k.y) + t * k.y_t + head * k.y_h;
  if (p.at < 0) return nullptr;
  return reinterpret_cast<typename E::T*>(which == 1 ? a.cache.k : a.cache.v) + p.at + ((int64_t)head << a.cache.shift) * a.D;
}

// Vectors of 16 bytes: everything aligned to them, D and rot multiples of two of them.
template <class E, bool APPEND, bool INTERLEAVED>
__global__ __launch_bounds__(256) void rope_kernel(RopeCall a) {
  constexpr int V = E::VEC;
  extern __shared__ __attribute__((aligned(16))) float turned[];   // [tokens][cos, sin][rot / 2]
  __shared__ Place places[2];
  const int t0 = blockIdx.x * a.tokens, pairs = a.rot / 2;
  const int groups = 256 / a.lanes, lane = threadIdx.x & (a.lanes - 1), group = threadIdx.x / a.lanes;
  const int token = group & (a.tokens - 1), t = t0 + token, turning = a.rot / (2 * V);   // lanes that turn pairs
  const int from = blockIdx.y * a.per_group, to = min(a.heads, from + a.per_group), stride = groups / a.tokens;
  const bool live = t < a.T && 2 * V * lane < a.D;
  // channels of the two vectors
  const int first = lane < turning ? lane * V : a.rot + (lane - turning) * V;
  const int second = first + (lane < turning ? a.rot : a.D - a.rot) / 2;
  // A head's vectors are requested while the one before is worked on, the first before the angles are known.
  auto load = [&](int h, uint4* u, uint4* w) {
    if (!live || h >= to) return;
    int head = h;
    const Heads& k = a.kind[APPEND ? kind_of(a, &head) : 0];
    const typename E::T* x = source<E>(a, k, t, head);
    *u = ld16(x + first);
    *w = ld16(x + second);
  };
  int h = from + group / a.tokens;
  uint4 u = make_uint4(0, 0, 0, 0), w = u, next_u = u, next_w = u;
  load(h, &u, &w);

  if constexpr (APPEND) {
    const int wave = threadIdx.x >> 6;
    for (int i = wave; i < a.tokens && t0 + i < a.T; i += 4) {
      const Place p = place_of(a, t0 + i);
      if ((threadIdx.x & 63) == 0) places[i] = p;
    }
    __syncthreads();
  }
  for (int i = threadIdx.x; i < a.tokens * pairs; i += 256) {
    const int token = i / pairs, pair = i - token * pairs, t = t0 + token;
    if (t >= a.T) break;
    float s, c;
    sin_cos(a.turns[pair], a.pos ? a.pos[t] : places[token].pos, &s, &c);
    turned[2 * token * pairs + pair] = c * a.scale;
    turned[(2 * token + 1) * pairs + pair] = s * (a.scale * a.sign);
  }
  __syncthreads();

  Place p{-1, 0, 0};
  if (APPEND && live) p = places[token];
  const float* cs = turned + 2 * token * pairs;
  for (; h - group / a.tokens < to; h += stride) {
    int head = h;
    const int which = APPEND ? kind_of(a, &head) : 0;
    const Heads& k = a.kind[which];
    const bool here = live && h < to;
    load(h + stride, &next_u, &next_w);
    if (k.turned || k.norm) {
      float xa[V], xb[V];
      unpack<E>(u, xa);
      unpack<E>(w, xb);
      if (k.norm) {
        float sum = 0.0f;
#pragma unroll
        for (int e = 0; e < V; ++e) sum = __builtin_fmaf(xa[e], xa[e], __builtin_fmaf(xb[e], xb[e], sum));
        for (int off = 1; off < a.lanes; off <<= 1) sum += __shfl_xor(sum, off, kWave);
        const float r = 1.0f / sqrtf(sum / (float)a.D + a.eps);
        if (here) {
          float na[V], nb[V];
          unpack<E>(ld16(reinterpret_cast<const typename E::T*>(k.norm) + first), na);
          unpack<E>(ld16(reinterpret_cast<const typename E::T*>(k.norm) + second), nb);
#pragma unroll
          for (int e = 0; e < V; ++e) {
            xa[e] = xa[e] * r * na[e];
            xb[e] = xb[e] * r * nb[e];
          }
        }
      }
      if (k.turned && lane < turning) {
        if constexpr (!INTERLEAVED) {
#pragma unroll
          for (int e = 0; e < V; ++e) {
            const float c = cs[first + e], s = cs[pairs + first + e], x = xa[e];
            xa[e] = x * c - xb[e] * s;
            xb[e] = xb[e] * c + x * s;
          }
        } else {
#pragma unroll
          for (int e = 0; e < V; e += 2) {
            const int i = (first + e) / 2, j = (second + e) / 2;
            const float x = xa[e], y = xb[e];
            xa[e] = x * cs[i] - xa[e + 1] * cs[pairs + i];
            xa[e + 1] = xa[e + 1] * cs[i] + x * cs[pairs + i];
            xb[e] = y * cs[j] - xb[e + 1] * cs[pairs + j];
            xb[e + 1] = xb[e + 1] * cs[j] + y * cs[pairs + j];
          }
        }
      }
      u = pack<E>(xa);
      w = pack<E>(xb);
    }
    if (here) {
      typename E::T* y = target<E, APPEND>(a, k, which, t, head, p);
      if (y) {
        *reinterpret_cast<uint4*>(y + first) = u;
        *reinterpret_cast<uint4*>(y + second) = w;
      }
    }
    u = next_u;
    w = next_w;
  }
}

// Any alignment and any even rot: a wave a token and head, a pair or a channel a lane and step.
template <class E, bool APPEND>
__global__ __launch_bounds__(256) void rope_any_kernel(RopeCall a, int interleaved) {
  constexpr int N = CI_MAX_ROPE_CHANNELS / 128;   // pairs of a lane
  const int lane = threadIdx.x & 63, t = blockIdx.x, pairs = a.rot / 2;
  Place p{-1, 0, 1};
  if constexpr (APPEND) p = place_of(a, t);
  const int at = a.pos ? a.pos[t] : p.pos;
  for (int h = blockIdx.y * 4 + (threadIdx.x >> 6); h < a.heads; h += gridDim.y * 4) {
    int head = h;
    const int which = APPEND ? kind_of(a, &head) : 0;
    const Heads& k = a.kind[which];
    const typename E::T* x = source<E>(a, k, t, head);
    typename E::T* y = target<E, APPEND>(a, k, which, t, head, p);
    if (!y) continue;
    // the turned channels as pairs, the others as they come, in pairs of neighbours (the last may be one)
    float xa[N], xb[N];
    int ia[N], ib[N];
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int j = lane + 64 * i;
      if (j < pairs) {
        ia[i] = interleaved ? 2 * j : j;
        ib[i] = interleaved ? 2 * j + 1 : j + pairs;
      } else {
        ia[i] = 2 * j;      // behind rot, which is 2 pairs
        ib[i] = 2 * j + 1;
      }
      xa[i] = ia[i] < a.D ? to_float<E>(x[ia[i]]) : 0.0f;
      xb[i] = ib[i] < a.D ? to_float<E>(x[ib[i]]) : 0.0f;
      sum = __builtin_fmaf(xa[i], xa[i], __builtin_fmaf(xb[i], xb[i], sum));
    }
    float r = 1.0f;
    const typename E::T* norm = reinterpret_cast<const typename E::T*>(k.norm);
    if (norm) r = 1.0f / sqrtf(wave_sum(sum) / (float)a.D + a.eps);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if (ia[i] >= a.D) continue;
      const bool both = ib[i] < a.D;
      if (norm) {
        xa[i] = xa[i] * r * to_float<E>(norm[ia[i]]);
        if (both) xb[i] = xb[i] * r * to_float<E>(norm[ib[i]]);
      }
      if (k.turned && lane + 64 * i < pairs) {
        float s, c;
        sin_cos(a.turns[lane + 64 * i], at, &s, &c);
        c *= a.scale;
        s *= a.scale * a.sign;
        const float v = xa[i];
        xa[i] = v * c - xb[i] * s;
        xb[i] = xb[i] * c + v * s;
      }
      y[ia[i]] = from_float<E>(xa[i]);
      if (both) y[ib[i]] = from_float<E>(xb[i]);
    }
  }
}

template <class E, bool APPEND>
int launch_type(RopeCall& a, int style, hipStream_t s) {
  constexpr int V = E::VEC;
  auto whole = [](int64_t stride) { return stride * E::BYTES % 16 == 0; };
  bool vectors = a.D % (2 * V) == 0 && a.rot % (2 * V) == 0;
  for (const Heads& k : a.kind)
    vectors = vectors && (k.count == 0 || (aligned16(k.x) && aligned16(k.y) && aligned16(k.norm) && whole(k.x_t) && whole(k.x_h) &&
                                           whole(k.y_t) && whole(k.y_h)));
  if (!vectors) {
    const dim3 grid((unsigned)a.T, (unsigned)std::min(4096, (a.heads + 3) / 4));
    hipLaunchKernelGGL((rope_any_kernel<E, APPEND>), grid, dim3(256), 0, s, a, style == CI_ROPE_INTERLEAVED);
    CI_HIP_CHECK_LAUNCH();
    return CI_OK;
  }
  a.lanes = 1;
  while (a.lanes * 2 * V < a.D) a.lanes *= 2;
  const int groups = 256 / a.lanes;
  // Few tokens: one a workgroup, and as many heads as it has lanes for.  Many: two, and up to eight rounds of heads, so that the angles and the
  // first loads' time are shared: 3584 tokens of 96 heads to pages 39.5 us; one round 46, four tokens 48 to 52.
  a.tokens = a.T >= 1024 && groups >= 2 ? 2 : 1;
  const int once = groups / a.tokens;   // heads of a workgroup and token at a time
  const int rounds = a.T >= 1024 ? std::min(8, (a.heads + once - 1) / once) : 1;
  a.per_group = rounds * once;
  const dim3 grid((unsigned)((a.T + a.tokens - 1) / a.tokens), (unsigned)((a.heads + a.per_group - 1) / a.per_group));
  const size_t lds = (size_t)a.tokens * a.rot * sizeof(float);
  if (style == CI_ROPE_INTERLEAVED)
    hipLaunchKernelGGL((rope_kernel<E, APPEND, true>), grid, dim3(256), lds, s, a);
  else
    hipLaunchKernelGGL((rope_kernel<E, APPEND, false>), grid, dim3(256), lds, s, a);
  CI_HIP_CHECK_LAUNCH();
  return CI_OK;
}

template <bool APPEND>
int launch(RopeCall& a, const ci_rope* rope, float eps, bool backward, int dtype, hipStream_t s) {
  a.turns = rope ? rope->turns : nullptr;
  a.scale = rope ? rope->scale : 1.0f;
  a.rot = rope ? rope->rot : 0;
  a.sign = backward ? -1.0f : 1.0f;
  a.eps = eps;
  a.heads = a.kind[0].count + a.kind[1].count + a.kind[2].count;
  for (int i = 0; i < 2; ++i) a.kind[i].turned = a.rot > 0;
  const int style = rope ? rope->style : CI_ROPE_HALF;
  switch (dtype) {
    case CI_F32: return launch_type<F32, APPEND>(a, style, s);
    case CI_F16: return launch_type<F16, APPEND>(a, style, s);
    default: return launch_type<BF16, APPEND>(a, style, s);
  }
}

}  // namespace

int launch_rope(const void* x, const int64_t (&stride)[2], int64_t T, int64_t H, int64_t D, int dtype, const void* norm, float eps,
                const ci_rope* rope, const int32_t* pos, bool backward, void* y, const int64_t (&y_stride)[2], hipStream_t s) {
  RopeCall a = {};
  a.kind[0] = Heads{x, y, stride[0], stride[1], y_stride[0], y_stride[1], norm, (int)H, 0};
  a.pos = pos;
  a.T = (int)T;
  a.D = (int)D;
  return launch<false>(a, rope, eps, backward, dtype, s);
}

int launch_kvp_append(const ci_kvp& c, const void* k, const void* v, const int64_t (&stride)[2], int64_t T, const int32_t* first,
                      const int32_t* lens, const int32_t* pos, const ci_rope* rope, const void* k_norm, float eps, const void* q,
                      int64_t Hq, const int64_t (&q_stride)[2], const void* q_norm, void* q_out, hipStream_t s) {
  RopeCall a = {};
  a.kind[0] = Heads{q, q_out, q_stride[0], q_stride[1], Hq * c.D, c.D, q_norm, (int)Hq, 0};
  a.kind[1] = Heads{k, nullptr, stride[0], stride[1], 0, 0, k_norm, c.H, 0};
  a.kind[2] = Heads{v, nullptr, stride[0], stride[1], 0, 0, nullptr, c.H, 0};
  a.cache = make_kvp(c);
  a.pos = pos;
  a.first = first;
  a.lens = lens;
  a.T = (int)T;
  a.D = c.D;
  return launch<true>(a, rope, eps, false, c.dtype, s);
}

}  // namespace ci
