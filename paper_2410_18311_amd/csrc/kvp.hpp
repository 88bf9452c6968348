// A cache in pages and packed batches (ci_kvp in coreinfer.h): what the kernels are given and how a row finds its sentence.
#pragma once

#include "common.hpp"

namespace ci {

struct Kvp {
  void *k, *v;
  const int32_t* table;
  int64_t most;
  uint32_t pages;
  int B, H, shift;   // page = 1 << shift slots
};

inline Kvp make_kvp(const ci_kvp& c) {
  return Kvp{c.k, c.v, c.table, c.most, (uint32_t)c.pages, (int)c.B, c.H, __builtin_ctz((unsigned)c.page)};
}

// The sentence of a packed row: the last one that does not begin behind it.  The lanes of a wave look at 64 beginnings at once, so that up to
// 64 sentences take one load.  `first` need not ascend for the result to be a sentence.
__device__ __forceinline__ int sentence_of(const int32_t* __restrict__ first, int B, int row) {
  const int lane = threadIdx.x & 63;
  int lo = 0, n = B;
  while (n > 1) {
    const int step = (n + 63) / 64, at = lane * step;
    const bool before = lane == 0 || (at < n && first[lo + at] <= row);
    const int last = __popcll(__ballot(before)) - 1;
    lo += last * step;
    n = min(step, n - last * step);
  }
  return __builtin_amdgcn_readfirstlane(lo);
}

// Sums (of integers) or maxima (of those from 0 on) over the lanes up to each, by moves between lanes instead of through the LDS.
__device__ __forceinline__ int scan_add(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);   // one, two, four, eight lanes on within 16
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);   // the last of 16 to the next 16, of 32 to the next 32
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);
  return v;
}
__device__ __forceinline__ int scan_max(int v) {
  v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false));
  v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false));
  v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false));
  v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false));
  v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false));
  v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false));
  return v;
}

// The packed rows of a sentence, as the calls' limits take them.
__device__ __forceinline__ int clamp_row(int at, int T) { return min(max(at, 0), T); }

}  // namespace ci
