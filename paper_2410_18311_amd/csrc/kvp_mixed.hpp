// Attention of prompts and single tokens together over a cache in pages (kvp_attend.hpp): one launch of both kinds of workgroups, so that those that
// wait for the cache's bytes run beside those that keep the matrix cores busy, and one that joins the pieces of both.  777 rows and
// six single tokens of 32 heads over up to 8192 slots: 97 to 101 us; with the two kinds in launches of their own 122, with the single tokens spread among
// the tiles 120, because tiles that start late end late.
#pragma once

#include "kvp_rows.hpp"
#include "kvp_tiles.hpp"

namespace ci {
namespace {

template <class E, int D, int WAVES, bool LSE>
__global__ __launch_bounds__(64 * WAVES, 2) void gemm_kvp_mixed_kernel(KvpAttend a) {
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  static_assert(sizeof(RowsLds<D>) <= 4 * kTileStep * 2 * D);
  const int all = a.tiles * a.c.H, piece = (int)blockIdx.x / all;
  if (piece < a.pieces)
    tile_block<E, D, WAVES, LSE>(a, (int)blockIdx.x - piece * all, piece);
  else
    rows_block<E, D>(a, (int)blockIdx.x - a.pieces * all, 0, 1, *reinterpret_cast<RowsLds<D>*>(smem));
}

template <class E, int D>
__global__ __launch_bounds__(256) void kvp_join_mixed_kernel(KvpAttend a, unsigned tiles) {
  if (blockIdx.x < tiles) join_tiles<E, D>(a, blockIdx.x, tiles);
  else join_rows<E, D>(a, blockIdx.x - tiles, gridDim.x - tiles);
}

template <class E, int D, int WAVES>
int launch_mixed(const KvpAttend& a, hipStream_t s) {
  const size_t lds = 4 * kTileStep * 2 * D;
  auto launch = [&](auto kernel, std::atomic<uint64_t>& seen) -> int {
    const int rc = allow_dynamic_lds(seen, reinterpret_cast<const void*>(kernel), lds);
    if (rc != CI_OK) return rc;
    hipLaunchKernelGGL(kernel, dim3((unsigned)(a.tiles * a.c.H * a.pieces + a.blocks)), dim3(64 * WAVES), lds, s, a);
    CI_HIP_CHECK_LAUNCH();
    return CI_OK;
  };
  static std::atomic<uint64_t> with{0}, without{0};
  const int rc = a.lse ? launch(gemm_kvp_mixed_kernel<E, D, WAVES, true>, with) : launch(gemm_kvp_mixed_kernel<E, D, WAVES, false>, without);
  if (rc != CI_OK) return rc;
  const unsigned tiles = a.pieces > 1 ? join_tiles_blocks<D>(a) : 0, rows = a.wanted ? join_rows_blocks(a) : 0;
  if (tiles + rows > 0) {
    hipLaunchKernelGGL((kvp_join_mixed_kernel<E, D>), dim3(tiles + rows), dim3(256), 0, s, a, tiles);
    CI_HIP_CHECK_LAUNCH();
  }
  return CI_OK;
}

template <class E, int D>
int launch_16bit(const KvpAttend& a, bool rows, bool tiles, hipStream_t s) {
  return rows && tiles ? launch_mixed<E, D, 4>(a, s) : tiles ? launch_tiles<E, D, 4>(a, s) : launch_rows<E, D>(a, s);
}

}  // namespace
}  // namespace ci
