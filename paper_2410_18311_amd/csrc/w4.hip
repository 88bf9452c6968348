// Products of one to 64 rows with 4-bit weights (q4.hpp): y = act(W x + b), or SiLU(G x) * (U x).  The projections of a decode step and the
// up, gate and down matrices of deployed core neurons; what a token reads is a fifth of the 16-bit weights' bytes and more.
//
// Layout.  Rows by 16 and columns by 128 make a block of 1 KB, which a wave loads with one instruction: lane 16 g + n holds row n, word j
// the columns 32 j + 8 g .. + 7, so that the word is the matrix cores' operand (16 rows, 32 columns) once its codes are unpacked and
// a group is a whole number of words.  Blocks lie along the columns; behind all of them, in the same order, the steps and lowest values of
// the 16 rows, group by group.  Rows and columns that fill up the last blocks hold code, step and lowest value 0.
#include <algorithm>

#include "q4.hpp"

namespace ci {
namespace {

constexpr int kBlockCols = 128, kBlockBytes = 1024;
inline int64_t row_tiles(int64_t R) { return (R + 15) / 16; }
inline int64_t col_blocks(int64_t C) { return (C + kBlockCols - 1) / kBlockCols; }

// ---- packing ---------------------------------------------------------------------------------------------------------------------

template <class D, int G>
__global__ __launch_bounds__(256) void w4_quantize_kernel(const typename D::T* w, int64_t ld, int R, int C, int nb, int64_t blocks,
                                                          uint32_t* codes, uint32_t* scales, int vectors) {
  const int64_t block = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (block >= blocks) return;
  const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
  const int64_t row = block / nb * 16 + n;
  const int col0 = (int)(block % nb) * kBlockCols;
  const typename D::T* src = w + row * ld;
  float x[4][8], lo[4], hi[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int c = col0 + 32 * j + 8 * g;
    const int have = row < R ? min(8, C - c) : 0;   // elements of the eight that are there
    if (vectors && have == 8) {
      if constexpr (D::VEC == 8) {
        unpack<D>(ld16(src + c), x[j]);
      } else {
        float a[4], b[4];
        unpack<D>(ld16(src + c), a);
        unpack<D>(ld16(src + c + 4), b);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[j][e] = a[e], x[j][4 + e] = b[e];
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[j][e] = e < have ? to_float<D>(src[c + e]) : 0.0f;
    }
    lo[j] = INFINITY;
    hi[j] = -INFINITY;
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < have) {
        lo[j] = min_nan(lo[j], x[j][e]);
        hi[j] = max_nan(hi[j], x[j][e]);
      }
#pragma unroll
    for (int off = 16; off <= 32; off <<= 1) {
      lo[j] = min_nan(lo[j], __shfl_xor(lo[j], off, kWave));
      hi[j] = max_nan(hi[j], __shfl_xor(hi[j], off, kWave));
    }
  }
  constexpr int J = G / 32;   // words of a group
  uint32_t word[4];
#pragma unroll
  for (int s = 0; s < 4 / J; ++s) {
    float l = lo[s * J], h = hi[s * J];
#pragma unroll
    for (int j = 1; j < J; ++j) l = min_nan(l, lo[s * J + j]), h = max_nan(h, hi[s * J + j]);
    const uint32_t scale = l > h ? 0u : q4_scale(l, h);   // l > h: a group of nothing
#pragma unroll
    for (int j = s * J; j < s * J + J; ++j) {
      const int c = col0 + 32 * j + 8 * g;
      word[j] = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (row < R && c + e < C) word[j] |= q4_code(x[j][e], scale) << (4 * q4_nibble(e));
    }
    if (g == s % 4) scales[(block * (4 / J) + s) * 16 + n] = scale;
  }
  *reinterpret_cast<uint4*>(codes + block * (kBlockBytes / 4) + lane * 4) = make_uint4(word[0], word[1], word[2], word[3]);
}

template <class D>
__global__ __launch_bounds__(256) void w4_read_kernel(const uint32_t* codes, const uint32_t* scales, int J, int R, int C, int nb,
                                                      int64_t blocks, typename D::T* w, int64_t ld) {
  const int64_t block = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (block >= blocks) return;
  const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
  const int64_t row = block / nb * 16 + n;
  if (row >= R) return;
  const int col0 = (int)(block % nb) * kBlockCols;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t word = codes[block * (kBlockBytes / 4) + lane * 4 + j], scale = scales[(block * (4 / J) + j / J) * 16 + n];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int c = col0 + 32 * j + 8 * g + e;
      if (c < C) w[row * ld + c] = from_float<D>(q4_value((word >> (4 * q4_nibble(e))) & 15u, scale));
    }
  }
}

// ---- products --------------------------------------------------------------------------------------------------------------------

struct RowsArgs {
  const void* x;
  int64_t ldx;
  const uint32_t* w[2];   // up (or the one matrix), gate
  size_t scales;          // words from a matrix's start to its steps and lowest values
  const void* bias;
  void* y;
  int64_t ldy;
  int M, R, C, nb, tiles; // nb blocks of columns, tiles of 16 rows
  int x_vectors, y_vectors, bias_dtype, y_dtype, act;
};

// Eight elements of x from column c on as the pieces of an operand; zeros past the end.
template <class D>
__device__ __forceinline__ void x_pieces(const typename D::T* src, int c, int C, int vectors, uint4 (&out)[Q4Type<D>::PIECES]) {
  if constexpr (D::VEC == 8) {
    if (vectors && c + 8 <= C) {
      out[0] = ld16(src + c);
      return;
    }
    uint32_t p[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t a = c + 2 * i < C ? (uint32_t)__builtin_bit_cast(uint16_t, src[c + 2 * i]) : 0u;
      const uint32_t b = c + 2 * i + 1 < C ? (uint32_t)__builtin_bit_cast(uint16_t, src[c + 2 * i + 1]) : 0u;
      p[i] = a | b << 16;
    }
    out[0] = make_uint4(p[0], p[1], p[2], p[3]);
  } else {
    float f[8];
    uint32_t p[4][3];
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = c + e < C ? src[c + e] : 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) split_bf16<3>(f[2 * i], f[2 * i + 1], p[i]);
#pragma unroll
    for (int q = 0; q < 3; ++q) out[q] = make_uint4(p[0][q], p[1][q], p[2][q], p[3][q]);
  }
}

// x as operands, for rows that do not fit the LDS: [block][word][piece][tile of 16 rows of x][lane], 16 bytes each.
template <class D>
__global__ __launch_bounds__(256) void w4_x_kernel(const typename D::T* x, int64_t ldx, int M, int C, int words, int vectors, int NT,
                                                   uint4* out) {
  const int at = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (at >= words * NT) return;
  const int lane = threadIdx.x & 63, m = at % NT * 16 + (lane & 15), word = at / NT;
  uint4 p[Q4Type<D>::PIECES];
  x_pieces<D>(x + (int64_t)min(m, M - 1) * ldx, word * 32 + 8 * (lane >> 4), C, vectors, p);
#pragma unroll
  for (int q = 0; q < Q4Type<D>::PIECES; ++q) out[((size_t)(word * Q4Type<D>::PIECES + q) * NT + at % NT) * 64 + lane] = p[q];
}

__device__ __forceinline__ float load_as(const void* p, int64_t i, int dtype) {
  if (dtype == CI_F32) return reinterpret_cast<const float*>(p)[i];
  if (dtype == CI_F16) return (float)reinterpret_cast<const _Float16*>(p)[i];
  return to_float<BF16>(reinterpret_cast<const uint16_t*>(p)[i]);
}
__device__ __forceinline__ void store_as(void* p, int64_t i, float v, int dtype) {
  if (dtype == CI_F32) reinterpret_cast<float*>(p)[i] = v;
  else if (dtype == CI_F16) reinterpret_cast<_Float16*>(p)[i] = (_Float16)v;
  else reinterpret_cast<uint16_t*>(p)[i] = from_float<BF16>(v);
}
__device__ __forceinline__ void store4_as(void* p, int64_t i, const float (&v)[4], int dtype) {
  if (dtype == CI_F32) {
    *reinterpret_cast<float4*>(reinterpret_cast<float*>(p) + i) = make_float4(v[0], v[1], v[2], v[3]);
    return;
  }
  uint2 u;
  if (dtype == CI_F16) {
    half2_t a, b;
    a[0] = (_Float16)v[0]; a[1] = (_Float16)v[1]; b[0] = (_Float16)v[2]; b[1] = (_Float16)v[3];
    u = make_uint2(__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b));
  } else {
    u = make_uint2(pk_bf16(v[0], v[1]), pk_bf16(v[2], v[3]));
  }
  *reinterpret_cast<uint2*>(reinterpret_cast<uint16_t*>(p) + i) = u;
}

// A workgroup multiplies RT tiles of 16 weight rows (pairs of up and gate tiles where DUAL) with NT tiles of 16 rows of x; its waves take
// the blocks of columns by turns and their sums are added at the end in the order of the waves.  XLDS: x is in the LDS, as operands of
// the M rows that there are ([word][piece][column octet g][row]).
template <class D, int G, int RT, int NT, bool DUAL, bool XLDS>
__global__ __launch_bounds__(XLDS ? (D::VEC == 8 ? 1024 : 512) : 256) void gemm_q4_rows_kernel(RowsArgs a) {
  constexpr int OP = Q4Type<D>::OP, PIECES = Q4Type<D>::PIECES;
  constexpr int J = G / 32, NG = 4 / J;   // words of a group, groups of a block
  constexpr int PF = 2;
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;

  const uint32_t* code[RT];
  const uint32_t* scale[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    const int tile = min(DUAL ? (int)blockIdx.x * (RT / 2) + t / 2 : (int)blockIdx.x * RT + t, a.tiles - 1);
    const uint32_t* w = a.w[DUAL ? t & 1 : 0];
    code[t] = w + (size_t)tile * a.nb * (kBlockBytes / 4) + lane * 4;
    scale[t] = w + a.scales + (size_t)tile * a.nb * (NG * 16) + g * 4;
  }
  struct Stage {
    uint4 code[RT], scale[RT][NG];
  } st[PF];
  auto load = [&](Stage& s, int b) {
    b = min(b, a.nb - 1);
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      s.code[t] = ld16(code[t] + (size_t)b * (kBlockBytes / 4));
#pragma unroll
      for (int i = 0; i < NG; ++i) s.scale[t][i] = ld16(scale[t] + (size_t)b * (NG * 16) + i * 16);
    }
  };
#pragma unroll
  for (int i = 0; i < PF; ++i) load(st[i], wave + i * waves);

  if constexpr (XLDS) {
    const int chunks = a.nb * 16;   // of eight columns
    for (int i = threadIdx.x; i < chunks * a.M; i += blockDim.x) {
      const int m = i / chunks, c = i % chunks;
      uint4 p[PIECES];
      x_pieces<D>(reinterpret_cast<const typename D::T*>(a.x) + m * a.ldx, c * 8, a.C, a.x_vectors, p);
#pragma unroll
      for (int q = 0; q < PIECES; ++q)
        reinterpret_cast<uint4*>(smem)[((c / 4 * PIECES + q) * 4 + c % 4) * a.M + m] = p[q];
    }
    __syncthreads();
  }
  const int xrow = min(n, a.M - 1);   // XLDS: columns of the product past the last row of x repeat it
  auto x_at = [&](int word, int q, int nt) {
    if constexpr (XLDS) return reinterpret_cast<const uint4*>(smem)[((word * PIECES + q) * 4 + g) * a.M + xrow];
    else return ld16(reinterpret_cast<const uint4*>(a.x) + ((size_t)(word * PIECES + q) * NT + nt) * 64 + lane);
  };

  const Q4Magic magic = q4_magic<OP>();
  const uint4 ones = make_uint4(kOnes<OP>, kOnes<OP>, kOnes<OP>, kOnes<OP>);
  f32x4q sum[RT][NT];
#pragma unroll
  for (int t = 0; t < RT; ++t)
#pragma unroll
    for (int u = 0; u < NT; ++u) sum[t][u] = f32x4q{0.0f, 0.0f, 0.0f, 0.0f};

  for (int b0 = wave; b0 < a.nb; b0 += PF * waves) {
#pragma unroll
    for (int i = 0; i < PF; ++i) {
      const int b = b0 + i * waves;
      if (b < a.nb) {
#pragma unroll
        for (int s = 0; s < NG; ++s) {
          f32x4q acc[RT][NT], sx[NT];
#pragma unroll
          for (int u = 0; u < NT; ++u) {
            sx[u] = f32x4q{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int t = 0; t < RT; ++t) acc[t][u] = sx[u];
          }
#pragma unroll
          for (int j = s * J; j < s * J + J; ++j) {
            uint4 w[RT];
#pragma unroll
            for (int t = 0; t < RT; ++t) {
              const uint32_t words[4] = {st[i].code[t].x, st[i].code[t].y, st[i].code[t].z, st[i].code[t].w};
              w[t] = q4_operand<OP>(words[j], magic);
            }
#pragma unroll
            for (int u = 0; u < NT; ++u)
#pragma unroll
              for (int q = 0; q < PIECES; ++q) {
                const uint4 x = x_at(b * 4 + j, q, u);
                sx[u] = mfma_q4<OP>(ones, x, sx[u]);
#pragma unroll
                for (int t = 0; t < RT; ++t) acc[t][u] = mfma_q4<OP>(w[t], x, acc[t][u]);
              }
          }
#pragma unroll
          for (int t = 0; t < RT; ++t) {
            const uint32_t sc[4] = {st[i].scale[t][s].x, st[i].scale[t][s].y, st[i].scale[t][s].z, st[i].scale[t][s].w};
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const float rest = __builtin_fmaf(half_lo(sc[r]), -kOffset<OP>, half_hi(sc[r]));
#pragma unroll
              for (int u = 0; u < NT; ++u)
                sum[t][u][r] = __builtin_fmaf(half_lo(sc[r]), acc[t][u][r], __builtin_fmaf(rest, sx[u][r], sum[t][u][r]));
            }
          }
        }
      }
      load(st[i], b + PF * waves);
    }
  }

  // the waves' sums, lane by lane
  __syncthreads();
  float4* part = reinterpret_cast<float4*>(smem);
#pragma unroll
  for (int t = 0; t < RT; ++t)
#pragma unroll
    for (int u = 0; u < NT; ++u)
      part[((t * NT + u) * waves + wave) * 64 + lane] = make_float4(sum[t][u][0], sum[t][u][1], sum[t][u][2], sum[t][u][3]);
  __syncthreads();
  constexpr int OUT = (DUAL ? RT / 2 : RT) * NT;
  for (int i = threadIdx.x; i < OUT * 64; i += blockDim.x) {
    const int l = i & 63, u = (i >> 6) % NT, t = (i >> 6) / NT;
    auto total = [&](int tile, float (&v)[4]) {
      float4 f = part[(tile * NT + u) * waves * 64 + l];
      for (int w = 1; w < waves; ++w) {
        const float4 h = part[((tile * NT + u) * waves + w) * 64 + l];
        f.x += h.x; f.y += h.y; f.z += h.z; f.w += h.w;
      }
      v[0] = f.x; v[1] = f.y; v[2] = f.z; v[3] = f.w;
    };
    const int m = u * 16 + (l & 15), row = ((int)blockIdx.x * (DUAL ? RT / 2 : RT) + t) * 16 + (l >> 4) * 4;
    if (m >= a.M || row >= a.R) continue;
    float v[4];
    total(DUAL ? 2 * t : t, v);
    if constexpr (DUAL) {
      float z[4];
      total(2 * t + 1, z);
#pragma unroll
      for (int r = 0; r < 4; ++r) v[r] *= silu(z[r]);
    } else {
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        if (a.bias && row + r < a.R) v[r] += load_as(a.bias, row + r, a.bias_dtype);
        if (a.act == CI_ACT_RELU) v[r] = v[r] < 0.0f ? 0.0f : v[r];   // keeps a NaN
      }
    }
    const int64_t at = (int64_t)m * a.ldy + row;
    if (a.y_vectors && row + 4 <= a.R) store4_as(a.y, at, v, a.y_dtype);
    else
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (row + r < a.R) store_as(a.y, at + r, v[r], a.y_dtype);
  }
}

constexpr size_t kXLds = 65536;   // x beside it leaves room for a second workgroup

size_t x_bytes(int64_t rows, int64_t C, int dtype) { return (size_t)rows * col_blocks(C) * kBlockCols * 2 * (dtype == CI_F32 ? 3 : 1); }
bool x_in_lds(int64_t M, int64_t C, int dtype) { return M <= 16 && x_bytes(M, C, dtype) <= kXLds; }

template <class D, int G, int RT, int NT, bool DUAL, bool XLDS>
int launch_rows(const RowsArgs& a, int waves, hipStream_t s) {
  const int per = DUAL ? RT / 2 : RT;
  size_t lds = (size_t)waves * RT * NT * 1024;
  if (XLDS) lds = std::max(lds, x_bytes(a.M, a.C, D::VEC == 8 ? CI_F16 : CI_F32));
  hipLaunchKernelGGL((gemm_q4_rows_kernel<D, G, RT, NT, DUAL, XLDS>), dim3((a.tiles + per - 1) / per), dim3(waves * 64), lds, s, a);
  CI_HIP_CHECK_LAUNCH();
  return CI_OK;
}

template <class D, int G, bool DUAL>
int launch_shape(const RowsArgs& a, bool x_lds, hipStream_t s) {
  if (x_lds) {
    // waves for two a SIMD on the whole chip, and no more than there are blocks
    int waves = 4;
    while (waves < (D::VEC == 8 ? 16 : 8) && (int64_t)a.tiles * waves < 4096 && waves * 2 <= a.nb) waves *= 2;
    if constexpr (DUAL) return launch_rows<D, G, 2, 1, true, true>(a, waves, s);
    else if (a.tiles >= 1024) return launch_rows<D, G, 2, 1, false, true>(a, waves, s);
    else return launch_rows<D, G, 1, 1, false, true>(a, waves, s);
  }
  if (a.M <= 16) return launch_rows<D, G, 2, 1, DUAL, false>(a, 4, s);
  if (a.M <= 32) return launch_rows<D, G, 2, 2, DUAL, false>(a, 4, s);
  return launch_rows<D, G, 2, 4, DUAL, false>(a, 4, s);
}

template <class D>
int launch_type(const RowsArgs& a, int group, bool x_lds, hipStream_t s) {
  const bool dual = a.act == CI_ACT_SWIGLU;
  switch (group) {
    case 32: return dual ? launch_shape<D, 32, true>(a, x_lds, s) : launch_shape<D, 32, false>(a, x_lds, s);
    case 64: return dual ? launch_shape<D, 64, true>(a, x_lds, s) : launch_shape<D, 64, false>(a, x_lds, s);
    default: return dual ? launch_shape<D, 128, true>(a, x_lds, s) : launch_shape<D, 128, false>(a, x_lds, s);
  }
}

template <class D>
int quantize_type(const void* w, int64_t R, int64_t C, int64_t ld, int group, uint32_t* codes, uint32_t* scales, hipStream_t s) {
  const int64_t nb = col_blocks(C), blocks = row_tiles(R) * nb;
  const int vectors = aligned16(w) && ld * D::BYTES % 16 == 0;
  auto* kernel = group == 32 ? w4_quantize_kernel<D, 32> : group == 64 ? w4_quantize_kernel<D, 64> : w4_quantize_kernel<D, 128>;
  hipLaunchKernelGGL(kernel, dim3((uint32_t)((blocks + 3) / 4)), dim3(256), 0, s, reinterpret_cast<const typename D::T*>(w), ld, (int)R,
                     (int)C, (int)nb, blocks, codes, scales, vectors);
  CI_HIP_CHECK_LAUNCH();
  return CI_OK;
}

template <class D>
int read_type(const uint32_t* packed, size_t at, int64_t R, int64_t C, int group, void* w, int64_t ld, hipStream_t s) {
  const int64_t nb = col_blocks(C), blocks = row_tiles(R) * nb;
  hipLaunchKernelGGL(w4_read_kernel<D>, dim3((uint32_t)((blocks + 3) / 4)), dim3(256), 0, s, packed, packed + at, group / 32, (int)R,
                     (int)C, (int)nb, blocks, reinterpret_cast<typename D::T*>(w), ld);
  CI_HIP_CHECK_LAUNCH();
  return CI_OK;
}

size_t code_words(int64_t R, int64_t C) { return (size_t)row_tiles(R) * col_blocks(C) * (kBlockBytes / 4); }

}  // namespace

size_t w4_bytes(int64_t R, int64_t C, int group) {
  return (size_t)row_tiles(R) * col_blocks(C) * (kBlockBytes + (size_t)(kBlockCols / group) * 64);
}
size_t w4_matvec_ws_bytes(int64_t M, int64_t C, int dtype) {
  if (x_in_lds(M, C, dtype)) return 0;
  return x_bytes(M <= 16 ? 16 : M <= 32 ? 32 : 64, C, dtype);
}

int launch_w4_quantize(const void* w, int64_t R, int64_t C, int64_t ld, int dtype, int group, void* packed, hipStream_t s) {
  uint32_t* codes = reinterpret_cast<uint32_t*>(packed);
  uint32_t* scales = codes + code_words(R, C);
  switch (dtype) {
    case CI_F32: return quantize_type<F32>(w, R, C, ld, group, codes, scales, s);
    case CI_F16: return quantize_type<F16>(w, R, C, ld, group, codes, scales, s);
    default: return quantize_type<BF16>(w, R, C, ld, group, codes, scales, s);
  }
}

int launch_w4_read(const void* packed, int64_t R, int64_t C, int group, void* w, int64_t ld, int dtype, hipStream_t s) {
  const uint32_t* p = reinterpret_cast<const uint32_t*>(packed);
  switch (dtype) {
    case CI_F32: return read_type<F32>(p, code_words(R, C), R, C, group, w, ld, s);
    case CI_F16: return read_type<F16>(p, code_words(R, C), R, C, group, w, ld, s);
    default: return read_type<BF16>(p, code_words(R, C), R, C, group, w, ld, s);
  }
}

int launch_w4_matvec(const void* x, int64_t M, int64_t ldx, int x_dtype, const void* w, const void* gate, const void* bias,
                     int bias_dtype, int act, int64_t R, int64_t C, int group, void* y, int64_t ldy, int y_dtype, void* ws,
                     hipStream_t s) {
  RowsArgs a;
  a.x = x;
  a.ldx = ldx;
  a.w[0] = reinterpret_cast<const uint32_t*>(w);
  a.w[1] = reinterpret_cast<const uint32_t*>(gate);
  a.scales = code_words(R, C);
  a.bias = bias;
  a.bias_dtype = bias_dtype;
  a.y = y;
  a.ldy = ldy;
  a.y_dtype = y_dtype;
  a.act = act;
  a.M = (int)M;
  a.R = (int)R;
  a.C = (int)C;
  a.nb = (int)col_blocks(C);
  a.tiles = (int)row_tiles(R);
  a.x_vectors = aligned16(x) && ldx * elem_bytes(x_dtype) % 16 == 0;
  a.y_vectors = reinterpret_cast<uintptr_t>(y) % (4 * elem_bytes(y_dtype)) == 0 && ldy % 4 == 0;
  const bool x_lds = x_in_lds(M, C, x_dtype);
  if (!x_lds) {
    const int NT = M <= 16 ? 1 : M <= 32 ? 2 : 4, words = a.nb * 4;
    const dim3 grid((words * NT + 3) / 4);
    uint4* out = reinterpret_cast<uint4*>(ws);
    if (x_dtype == CI_F32)
      hipLaunchKernelGGL(w4_x_kernel<F32>, grid, dim3(256), 0, s, reinterpret_cast<const float*>(x), ldx, a.M, a.C, words, a.x_vectors, NT, out);
    else if (x_dtype == CI_F16)
      hipLaunchKernelGGL(w4_x_kernel<F16>, grid, dim3(256), 0, s, reinterpret_cast<const _Float16*>(x), ldx, a.M, a.C, words, a.x_vectors, NT, out);
    else
      hipLaunchKernelGGL(w4_x_kernel<BF16>, grid, dim3(256), 0, s, reinterpret_cast<const uint16_t*>(x), ldx, a.M, a.C, words, a.x_vectors, NT, out);
    CI_HIP_CHECK_LAUNCH();
    a.x = ws;
  }
  switch (x_dtype) {
    case CI_F32: return launch_type<F32>(a, group, x_lds, s);
    case CI_F16: return launch_type<F16>(a, group, x_lds, s);
    default: return launch_type<BF16>(a, group, x_lds, s);
  }
}

}  // namespace ci
