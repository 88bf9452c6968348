// A layer's keys and values in 4 bits (q4.hpp; ci_kv4 in coreinfer.h): where everything lies, and what the kernels are given.
//
// Layouts follow from how the matrix cores take their operands, so that what a wave loads (1 KB of 16 slots' keys, or of 16 slots'
// values, with one instruction) needs no exchange between lanes and no LDS.  n = 0 .. 15, g = 0 .. 3, D = 64 or 128 channels.
//   keys    [B, H, cap] rows of D / 8 words; word (D / 32) g + j holds the channels 32 j + 8 g .. + 7 in the order of q4_nibble: lane 16 g + n
//           reads row n's words of g and has its eighth of each product over 32 channels, and a group is whole products.
//   values  [B, H, cap / 4] quads of four slots, 16 n's of D / 32 words: the channels n, 16 + n, 32 + n, ...  Half-word s of word 2 p + f
//           (p = 0, 1; D = 64: word p) holds the channels 64 f + 16 i + n, i = 0 .. 3, of slot 2 p + s of the quad, a nibble each: masked
//           and shifted by 4 i, a word is two neighbouring slots' values of a channel, as the product over slots wants them, and a
//           product's 16 channels are of one group.  One slot's values are half-words of their own.
//   scales  [B, H, D / group, cap] words, step and lowest value.
#pragma once

#include "q4.hpp"

namespace ci {

struct Kv4 {
  uint32_t *k, *v, *ks, *vs;
  float* weight;
  int32_t* pos;
  int B, H, cap;
};

constexpr int kMaxSplits = 64;  // of a call over the slots: the lanes of the join keep a factor of each

struct Kv4Attend {
  Kv4 c;
  const void* q;
  int64_t q_b, q_s, q_h;  // strides in elements
  void* out;
  float* lse;
  float* weight_out;
  const int32_t* lens;
  int S, G, R, max_len;   // R = S G rows of a head of the cache
  uint32_t inverse_G;     // 2^32 / G, rounded up
  float scale;            // of the logits, with log2(e)
  int q_vectors;
  // Work of the launch: `blocks` workgroups (times those along the rows) share the slots of all sentences; see Shares.  wanted 0: one workgroup a head.
  int blocks, wanted, least;
  int row_tiles, token_waves;      // tiles of 16 rows; waves of a workgroup along the slots (4 or 1: then along the tiles)
  int weights;                     // 0 none, 1 from stored logits, 2 from logits computed again
  int2* place;  // [B]: a sentence's first piece and how many it has
  // partial results [blocks, row_tiles 16] twice and [blocks, row_tiles 16, D]; log-sums [B H, R]; logits [B H, R, whole steps of slots]
  float *m, *l, *o, *z, *logits;
};

template <class D> int launch_kv4_attend_type(const Kv4Attend& a, int head_dim, int group, hipStream_t s);

}  // namespace ci
