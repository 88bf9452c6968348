// Products of one to 64 rows with 4-bit weights (q4.hpp): y = act(W x + b), or SiLU(G x) * (U x).  The projections of a decode step and the
// up, gate and down matrices of deployed core neurons; a token reads 0.28 of the bytes of 16-bit weights (groups of 64).
//
// Bound by those bytes where there are enough of them: a gated 13824 x 5120 product of one row, 80 MB, 15.2 us with two sets of weights by turns
// (5.2 TB/s, a large copy's rate; the memory-side cache has a part), 16.1 with three; 14746 x 9216 of eight rows, 77 MB, 17.4 us.  Small ones
// are bound by latency: 4096 x 6554 (14 MB) 7.2 us, 1024 x 256 4.2 us.  Above 16 rows by what is read of x from the L2, all of it in every
// workgroup: 64 rows of the gated product 64 us.
//
// Layout.  Rows by 16 and columns by 128 make a block of 1 KB, which a wave loads with one instruction: lane 16 g + n holds row n, word j
// the columns 32 j + 8 g .. + 7, so that the word is the matrix cores' operand (16 rows, 32 columns) once its codes are unpacked and
// a group is a whole number of words.  Blocks lie along the columns; behind all of them, in the same order, the steps and lowest values of
// the 16 rows, row by row: a row's groups of a block are neighbours.  Rows and columns that fill up the last blocks hold code, step and lowest value 0.
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
      uint32_t n8[8];
      q4_codes(x[j], scale, n8);
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (row < R && c + e < C) word[j] |= n8[e] << (4 * q4_nibble(e));
    }
    if (g == s % 4) scales[(block * 16 + n) * (4 / J) + s] = scale;
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
    const uint32_t word = codes[block * (kBlockBytes / 4) + lane * 4 + j], scale = scales[(block * 16 + n) * (4 / J) + j / J];
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
  int x_vectors, x_bytes, bias_dtype, y_dtype, act;
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
// Where the kernel has x from: rows in memory as they are (16-bit, requested with the weights), the LDS as operands of the M rows that there
// are ([word][piece][column octet g][row]), or operands that w4_x_kernel has laid out.
enum { kXRows, kXLds, kXOperands };

// A workgroup multiplies RT tiles of 16 weight rows (pairs of up and gate tiles where DUAL) with NT tiles of 16 rows of x; its waves take
// the blocks of columns by turns and their sums are added at the end in the order of the waves.  A block is requested two turns ahead;
// what would lie behind the last one is out of the descriptors' range, which costs no traffic and keeps the number of loads on their way
// the same on every path.  Results come with a lane's four rows of x and one row of weights, so a group's two numbers are one load for
// that row; ROWS: how many of the four are of rows that there are: up to 4 ROWS rows of x stand ROWS to a lane, and the other places repeat them.
template <class D, int G, int RT, int NT, bool DUAL, int X, int THREADS, int ROWS>
__global__ __launch_bounds__(THREADS) void gemm_q4_rows_kernel(RowsArgs a) {
  constexpr int OP = Q4Type<D>::OP, PIECES = Q4Type<D>::PIECES;
  constexpr int J = G / 32, NG = 4 / J;   // words of a group, groups of a block
  constexpr int PF = 2;
  constexpr bool kStaged = X == kXRows || (X == kXOperands && NT * PIECES * RT <= 8);   // x is requested with the weights, registers permitting
  static_assert(X != kXRows || (NT == 1 && PIECES == 1), "rows are read for one tile of 16-bit ones");
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;

  __amdgpu_buffer_rsrc_t code[RT], scale[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    const int tile = min(DUAL ? (int)blockIdx.x * (RT / 2) + t / 2 : (int)blockIdx.x * RT + t, a.tiles - 1);
    const uint32_t* w = a.w[DUAL ? t & 1 : 0];
    code[t] = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint32_t*>(w + (size_t)tile * a.nb * (kBlockBytes / 4)), 0, a.nb * kBlockBytes, 0x00020000);
    scale[t] = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint32_t*>(w + a.scales + (size_t)tile * a.nb * (NG * 16)), 0, a.nb * NG * 64, 0x00020000);
  }
  const auto xs = __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(a.x), 0, a.x_bytes, 0x00020000);
  static_assert(NT == 1 || ROWS == 4, "tiles of x but a single one are full");
  const int xrow = min(ROWS * (n >> 2) + min(n & 3, ROWS - 1), a.M - 1);   // the row of x in place n of a single tile
  int x_off[NT];
#pragma unroll
  for (int u = 0; u < NT; ++u) x_off[u] = (int)(xrow * a.ldx * 2) + g * 16;
  struct Stage {
    uint4 code[RT], x[kStaged ? NT * 4 * PIECES : 1];
    uint32_t scale[RT][NG];   // of the lane's row
  } st[PF];
  auto load = [&](Stage& s, int b) {
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      s.code[t] = __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(code[t], b * kBlockBytes + lane * 16, 0, 0));
      const int at = b * (NG * 64) + n * (NG * 4);
      if constexpr (NG == 1) {
        s.scale[t][0] = __builtin_amdgcn_raw_buffer_load_b32(scale[t], at, 0, 0);
      } else if constexpr (NG == 2) {
        const auto two = __builtin_amdgcn_raw_buffer_load_b64(scale[t], at, 0, 0);
        s.scale[t][0] = two[0], s.scale[t][1] = two[1];
      } else {
        const auto four = __builtin_amdgcn_raw_buffer_load_b128(scale[t], at, 0, 0);
#pragma unroll
        for (int i = 0; i < 4; ++i) s.scale[t][i] = four[i];
      }
    }
    if constexpr (kStaged)
#pragma unroll
      for (int u = 0; u < NT; ++u)
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int q = 0; q < PIECES; ++q) {
            const int at = X == kXRows ? x_off[u] + b * (kBlockCols * 2) + j * 64 : (((b * 4 + j) * PIECES + q) * NT + u) * 1024 + lane * 16;
            s.x[(u * 4 + j) * PIECES + q] = __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(xs, at, 0, 0));
          }
  };
#pragma unroll
  for (int i = 0; i < PF; ++i) load(st[i], wave + i * waves);

  if constexpr (X == kXLds) {
    constexpr int AHEAD = 4;   // pieces on their way at a time
    const int chunks = a.nb * 16, all = chunks * a.M;   // of eight columns
    for (int i0 = threadIdx.x; i0 < all; i0 += AHEAD * blockDim.x) {
      uint4 p[AHEAD][PIECES];
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        const int i = min(i0 + u * (int)blockDim.x, all - 1);
        x_pieces<D>(reinterpret_cast<const typename D::T*>(a.x) + i / chunks * a.ldx, i % chunks * 8, a.C, a.x_vectors, p[u]);
      }
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        const int i = i0 + u * (int)blockDim.x, m = i / chunks, c = i % chunks;
        if (i < all)
#pragma unroll
          for (int q = 0; q < PIECES; ++q) reinterpret_cast<uint4*>(smem)[((c / 4 * PIECES + q) * 4 + c % 4) * a.M + m] = p[u][q];
      }
    }
    __syncthreads();
  }
  auto x_at = [&](const Stage& s, int b, int j, int q, int nt) {
    if constexpr (X == kXRows) {
      uint4 x = s.x[nt * 4 + j];
      const int have = a.C - (b * kBlockCols + 32 * j + 8 * g);
      if (b == a.nb - 1 && have < 8) {   // what follows the row is something else
        uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = 2 * e < have ? w[e] : 0u;
        x = make_uint4(w[0], w[1], w[2], w[3]);
      }
      return x;
    } else if constexpr (X == kXLds) {
      return reinterpret_cast<const uint4*>(smem)[(((b * 4 + j) * PIECES + q) * 4 + g) * a.M + xrow];
    } else if constexpr (kStaged) {
      return s.x[(nt * 4 + j) * PIECES + q];
    } else {
      return ld16(reinterpret_cast<const uint4*>(a.x) + ((size_t)((b * 4 + j) * PIECES + q) * NT + nt) * 64 + lane);
    }
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
                const uint4 x = x_at(st[i], b, j, q, u);
                sx[u] = mfma_q4<OP>(x, ones, sx[u]);
#pragma unroll
                for (int t = 0; t < RT; ++t) acc[t][u] = mfma_q4<OP>(x, w[t], acc[t][u]);
              }
          }
#pragma unroll
          for (int t = 0; t < RT; ++t) {
            const uint32_t sc = st[i].scale[t][s];
            const float rest = __builtin_fmaf(half_lo(sc), -kOffset<OP>, half_hi(sc));
#pragma unroll
            for (int u = 0; u < NT; ++u)
#pragma unroll
              for (int r = 0; r < ROWS; ++r)
                sum[t][u][r] = __builtin_fmaf(half_lo(sc), acc[t][u][r], __builtin_fmaf(rest, sx[u][r], sum[t][u][r]));
          }
        }
      }
      load(st[i], b + PF * waves);
    }
  }

  // the waves' sums, lane by lane
  __syncthreads();
  float* part = reinterpret_cast<float*>(smem);   // [tile][tile of x][wave][row of x of the four][lane]
#pragma unroll
  for (int t = 0; t < RT; ++t)
#pragma unroll
    for (int u = 0; u < NT; ++u)
#pragma unroll
      for (int r = 0; r < ROWS; ++r) part[(((t * NT + u) * waves + wave) * ROWS + r) * 64 + lane] = sum[t][u][r];
  __syncthreads();
  constexpr int TILES = DUAL ? RT / 2 : RT;   // of results
  // neighbouring threads have neighbouring rows of weights, and so neighbouring results
  for (int i = threadIdx.x; i < TILES * NT * ROWS * 64; i += blockDim.x) {
    const int col = i & 15, t = (i >> 4) % TILES, rest = (i >> 4) / TILES, gr = rest % 4, r = rest / 4 % ROWS, u = rest / 4 / ROWS;
    const int m = u * 16 + ROWS * gr + r, row = ((int)blockIdx.x * TILES + t) * 16 + col;
    if (m >= a.M || row >= a.R) continue;
    auto total = [&](int tile) {
      float v = 0.0f;
      for (int w = 0; w < waves; ++w) v += part[(((tile * NT + u) * waves + w) * ROWS + r) * 64 + 16 * gr + col];
      return v;
    };
    float v = total(DUAL ? 2 * t : t);
    if constexpr (DUAL) {
      v *= silu(total(2 * t + 1));
    } else {
      if (a.bias) v += load_as(a.bias, row, a.bias_dtype);
      if (a.act == CI_ACT_RELU) v = v < 0.0f ? 0.0f : v;   // keeps a NaN
    }
    store_as(a.y, (int64_t)m * a.ldy + row, v, a.y_dtype);
  }
}

constexpr size_t kXInLds = 65536;   // what a launch may have unasked, and room for a second workgroup

size_t x_bytes(int64_t rows, int64_t C, int dtype) { return (size_t)rows * col_blocks(C) * kBlockCols * 2 * (dtype == CI_F32 ? 3 : 1); }
int64_t x_span(int64_t M, int64_t C, int64_t ldx) { return ((M - 1) * ldx + C) * 2; }
// Rows as they are: 16-bit, whole words at whole words, within a descriptor's reach.
bool x_rows(const void* x, int64_t M, int64_t C, int64_t ldx, int dtype) {
  return dtype != CI_F32 && M <= 16 && (reinterpret_cast<uintptr_t>(x) & 3u) == 0 && C % 2 == 0 && (M == 1 || ldx % 2 == 0) &&
         ldx <= ((int64_t)1 << 26) &&
         x_span(M, C, ldx) < ((int64_t)1 << 30);
}
bool x_in_lds(int64_t M, int64_t C, int dtype) { return M <= 16 && x_bytes(M, C, dtype) <= kXInLds; }

template <class D, int G, int RT, int NT, bool DUAL, int X, int THREADS, int ROWS>
int launch_rows(const RowsArgs& a, int waves, hipStream_t s) {
  const int per = DUAL ? RT / 2 : RT;
  size_t lds = (size_t)waves * RT * NT * 1024;
  if (X == kXLds) lds = std::max(lds, x_bytes(a.M, a.C, D::VEC == 8 ? CI_F16 : CI_F32));
  hipLaunchKernelGGL((gemm_q4_rows_kernel<D, G, RT, NT, DUAL, X, THREADS, ROWS>), dim3((a.tiles + per - 1) / per), dim3(waves * 64), lds, s, a);
  CI_HIP_CHECK_LAUNCH();
  return CI_OK;
}

template <class D, int G, bool DUAL, int X, int ROWS>
int launch_few(const RowsArgs& a, hipStream_t s) {
  // Eight waves to a compute unit, if there are as many blocks, and no more to a workgroup than registers leave room for (groups of 32, fp32).
  // Pairs of tiles share what is read of x, where there are enough of them for the chip, fours where that comes from memory (14746 x 9216, eight
  // rows: 20.0 us in pairs, 18.2 in fours).
  constexpr int MOST = D::VEC == 8 && G > 32 && X == kXLds ? 16 : 8;
  const int RT = DUAL || a.tiles >= 900 ? 2 : 1, groups = DUAL ? a.tiles : (a.tiles + RT - 1) / RT;
  int waves = 4;
  while (waves < MOST && groups * waves < 2000 && waves * 2 <= a.nb) waves *= 2;
  if constexpr (DUAL) {
    return waves == 4 ? launch_rows<D, G, 2, 1, true, X, 256, ROWS>(a, waves, s) : launch_rows<D, G, 2, 1, true, X, MOST * 64, ROWS>(a, waves, s);
  } else if (RT == 2) {
    if constexpr (X == kXRows) return launch_rows<D, G, 4, 1, false, X, 512, ROWS>(a, 8, s);   // rows this long are more than eight blocks
    else return launch_rows<D, G, 2, 1, false, X, 512, ROWS>(a, waves, s);   // never more than eight waves
  } else {
    return waves == 4 ? launch_rows<D, G, 1, 1, false, X, 256, ROWS>(a, waves, s) : launch_rows<D, G, 1, 1, false, X, MOST * 64, ROWS>(a, waves, s);
  }
}
template <class D, int G, bool DUAL, int X>
int launch_by_rows(const RowsArgs& a, hipStream_t s) {
  if (a.M <= 4) return launch_few<D, G, DUAL, X, 1>(a, s);
  return a.M <= 8 ? launch_few<D, G, DUAL, X, 2>(a, s) : launch_few<D, G, DUAL, X, 4>(a, s);
}

template <class D, int G, bool DUAL>
int launch_shape(const RowsArgs& a, int x, hipStream_t s) {
  if (x == kXLds) return launch_by_rows<D, G, DUAL, kXLds>(a, s);
  if constexpr (D::VEC == 8)
    if (x == kXRows) return launch_by_rows<D, G, DUAL, kXRows>(a, s);
  if (a.M <= 16) return launch_rows<D, G, 2, 1, DUAL, kXOperands, 256, 4>(a, 4, s);
  if (a.M <= 32) return launch_rows<D, G, 2, 2, DUAL, kXOperands, 256, 4>(a, 4, s);
  return launch_rows<D, G, 2, 4, DUAL, kXOperands, 256, 4>(a, 4, s);
}

template <class D>
int launch_type(const RowsArgs& a, int group, int x, hipStream_t s) {
  const bool dual = a.act == CI_ACT_SWIGLU;
  switch (group) {
    case 32: return dual ? launch_shape<D, 32, true>(a, x, s) : launch_shape<D, 32, false>(a, x, s);
    case 64: return dual ? launch_shape<D, 64, true>(a, x, s) : launch_shape<D, 64, false>(a, x, s);
    default: return dual ? launch_shape<D, 128, true>(a, x, s) : launch_shape<D, 128, false>(a, x, s);
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
  const int where = x_in_lds(M, C, x_dtype) ? kXLds : x_rows(x, M, C, ldx, x_dtype) ? kXRows : kXOperands;
  a.x_bytes = where == kXRows ? (int)x_span(M, C, ldx) : where == kXOperands ? (int)w4_matvec_ws_bytes(M, C, x_dtype) : 0;
  if (where == kXOperands) {
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
    case CI_F32: return launch_type<F32>(a, group, where, s);
    case CI_F16: return launch_type<F16>(a, group, where, s);
    default: return launch_type<BF16>(a, group, where, s);
  }
}

}  // namespace ci
