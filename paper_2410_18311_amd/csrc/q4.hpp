// Numbers in 4 bits, as the weights (w4.hip) and the cache (kv4.hip) hold them, and their matrix products on gfx950.
//
// A group of 32, 64 or 128 elements along a row is held as codes n = 0 .. 15 with low = fp16(min) and step = fp16((max - min) / 15),
// n = rint((x - low) / step) in fp32, and stands for low + step n.  A product with a row x of such groups is, per group,
//   step (sum n x) + low (sum x),
// so the matrix cores multiply the codes themselves and the two fp16 numbers enter once per group, in fp32.
//
// A code becomes an operand without a conversion: its bits at the top of the mantissa of 16 are 16 + n, and two instructions put two of them there.
// The constant comes out again with the sum of x, which the matrix cores form beside (a product with ones): one vector instruction an element,
// where a conversion takes more than 2.  At the bottom of the mantissa they would be 128 + n (fp16: 64 + n) and an eighth of the instructions less,
// but the sums lose what their size loses: 24 on average instead of the codes' own 9, 1.4 of 24 bits, not 4.  Operands for fp32 rows carry the
// codes exactly and take twice the instructions.
#pragma once

#include "common.hpp"

namespace ci {
namespace {

typedef float f32x4q __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8q __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8q __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2q __attribute__((ext_vector_type(2)));
typedef float f32x2q __attribute__((ext_vector_type(2)));

// What multiplies: bf16 with 16 + n, fp16 with 16 + n, bf16 with n.
enum { kOpBF16, kOpF16, kOpExact };
template <int OP> constexpr float kOffset = OP == kOpExact ? 0.0f : 16.0f;
template <int OP> constexpr uint32_t kMagic = OP == kOpF16 ? 0x4c004c00u : 0x41804180u;
template <int OP> constexpr int kCodeBit = OP == kOpF16 ? 6 : 3;   // where a code stands in its half-word
template <int OP> constexpr uint32_t kOnes = OP == kOpF16 ? 0x3c003c00u : 0x3f803f80u;

// The other operand in as many pieces as hold it whole: fp32 values in three bf16 ones, 16-bit values as they are.
template <class D> struct Q4Type;
template <> struct Q4Type<F32> { static constexpr int OP = kOpExact, PIECES = 3; };
template <> struct Q4Type<F16> { static constexpr int OP = kOpF16, PIECES = 1; };
template <> struct Q4Type<BF16> { static constexpr int OP = kOpBF16, PIECES = 1; };

template <int OP>
__device__ __forceinline__ f32x4q mfma_q4(const uint4& a, const uint4& b, f32x4q c) {
  if constexpr (OP == kOpF16)
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8q, a), __builtin_bit_cast(f16x8q, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8q, a), __builtin_bit_cast(bf16x8q, b), c, 0, 0, 0);
}

// Mask and constant in registers of their own: an instruction with two literals does not exist, and with the constants known the compiler
// makes two of it.
struct Q4Magic {
  uint32_t mask, magic;
};
template <int OP>
__device__ __forceinline__ Q4Magic q4_magic() {
  Q4Magic m{0x000f000fu << kCodeBit<OP>, kMagic<OP>};
  asm("" : "+s"(m.mask), "+v"(m.magic));
  return m;
}

// The two codes at bits 4 i and 16 + 4 i of w.
template <int OP>
__device__ __forceinline__ uint32_t q4_pair(uint32_t w, int i, const Q4Magic& m) {
  const int up = kCodeBit<OP> - 4 * i;
  return ((up > 0 ? w << up : w >> -up) & m.mask) | m.magic;
}

// Eight codes as an operand's eight elements: element 2 i is the nibble i of w, element 2 i + 1 the nibble i + 4.
template <int OP>
__device__ __forceinline__ uint4 q4_operand(uint32_t w, const Q4Magic& m) {
  if constexpr (OP != kOpExact) {
    return make_uint4(q4_pair<OP>(w, 0, m), q4_pair<OP>(w, 1, m), q4_pair<OP>(w, 2, m), q4_pair<OP>(w, 3, m));
  } else {
    // bytes 0 .. 3 of even: nibbles 0, 2, 4, 6; a code below 16 is exact in the upper half of its fp32 image
    const uint32_t even = w & 0x0f0f0f0fu, odd = (w >> 4) & 0x0f0f0f0fu;
    auto pair = [](uint32_t a, uint32_t b) {
      return __builtin_amdgcn_perm(f2u((float)(b & 0xffu)), f2u((float)(a & 0xffu)), 0x07060302u);
    };
    return make_uint4(pair(even, even >> 16), pair(odd, odd >> 16), pair(even >> 8, even >> 24), pair(odd >> 8, odd >> 24));
  }
}
// Where an element e of eight goes in the word.
__device__ __forceinline__ int q4_nibble(int e) { return (e >> 1) + 4 * (e & 1); }

__device__ __forceinline__ uint32_t pk_bf16(float a, float b) {
  f32x2q f;
  f.x = a;
  f.y = b;
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, bf16x2q));
}
__device__ __forceinline__ float bf16_lo(uint32_t p) { return u2f(p << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t p) { return u2f(p & 0xffff0000u); }

// Two fp32 values in N bf16 pieces, each the rounded rest of the ones before: 8 bits more with every piece.
template <int N>
__device__ __forceinline__ void split_bf16(float a, float b, uint32_t (&piece)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    piece[i] = pk_bf16(a, b);
    if (i + 1 < N) {
      a -= bf16_lo(piece[i]);
      b -= bf16_hi(piece[i]);
    }
  }
}

__device__ __forceinline__ float half_lo(uint32_t p) { return (float)__builtin_bit_cast(half2_t, p)[0]; }
__device__ __forceinline__ float half_hi(uint32_t p) { return (float)__builtin_bit_cast(half2_t, p)[1]; }

// Step (lower half) and lowest value (upper half) of a group from its extremes; what fp16 does not hold is held at its largest.  NaN
// extremes make both NaN.
__device__ __forceinline__ uint32_t q4_scale(float lo, float hi) {
  constexpr float kMax = 65504.0f;
  float step = (hi - lo) / 15.0f;
  if (step > kMax) step = kMax;
  if (lo > kMax) lo = kMax;
  if (lo < -kMax) lo = -kMax;
  half2_t h;
  h[0] = (_Float16)step;
  h[1] = (_Float16)lo;
  return __builtin_bit_cast(uint32_t, h);
}
__device__ __forceinline__ uint32_t q4_code(float x, uint32_t scale) {
  const float step = half_lo(scale);
  if (!(step > 0.0f)) return 0;
  const float n = rintf((x - half_hi(scale)) / step);
  return (uint32_t)fminf(fmaxf(n, 0.0f), 15.0f);
}
// The codes of eight elements of a group.  A product with the reciprocal differs from the quotient by the reciprocal's 2^-23, the product's 2^-24
// and the quotient's own 2^-24, 2^-22 of it together: at most 2^-18 = 3.8e-6 for what counts (up to 16).  Only where it lies within twice that of the
// middle between two codes do the divisions decide; a fifth of the instructions otherwise.
__device__ __forceinline__ void q4_codes(const float (&x)[8], uint32_t scale, uint32_t (&n)[8]) {
  const float step = half_lo(scale), low = half_hi(scale), inv = __builtin_amdgcn_rcpf(step);
  bool close = false;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float q = (x[e] - low) * inv, r = rintf(q);
    close |= fabsf(fabsf(q - r) - 0.5f) < 8e-6f;
    n[e] = step > 0.0f ? (uint32_t)fminf(fmaxf(r, 0.0f), 15.0f) : 0u;
  }
  if (__any(close)) {
#pragma unroll
    for (int e = 0; e < 8; ++e) n[e] = q4_code(x[e], scale);
  }
}
__device__ __forceinline__ float q4_value(uint32_t code, uint32_t scale) {
  return __builtin_fmaf(half_lo(scale), (float)code, half_hi(scale));
}
// Extremes that a NaN takes over, in one instruction.
__device__ __forceinline__ float min_nan(float a, float b) { return __builtin_elementwise_minimum(a, b); }
__device__ __forceinline__ float max_nan(float a, float b) { return __builtin_elementwise_maximum(a, b); }

}  // namespace
}  // namespace ci
