// Attention over a cache in pages: how a call is split over the chip (the kernels are in kvp_rows.hpp, kvp_tiles.hpp and
// kvp_mixed.hpp).
#include <algorithm>

#include "kvp_attend.hpp"

namespace ci {
namespace {

constexpr int kCus = 256;   // of an MI355X; a workspace query knows no device
constexpr double kLog2e = 1.4426950408889634;

struct AttendPlan {
  bool rows, in_tiles;   // which kernels run
  int few, row_tiles, blocks, wanted, least;
  int tiles, pieces;
  size_t place, m, l, o, tile_m, tile_l, tile_exact, tile_o, bytes;   // places in the workspace
};

constexpr int kTileRows = 128;

// Most steps of `step` slots that the rows of a sentence see something of.
int64_t most_steps(int64_t step, int64_t rows, int64_t max_len, int64_t window, int64_t sinks) {
  const int64_t all = (max_len + step - 1) / step;
  return window == 0 || window >= max_len ? all : std::min(all, (window + rows) / step + 2 + (std::min(sinks, max_len) + step - 1) / step);
}

AttendPlan attend_plan(const ci_kvp& c, int64_t T, int64_t G, int64_t max_rows, int64_t max_len, int64_t window, int64_t sinks) {
  AttendPlan p = {};
  const int64_t heads = c.B * c.H, R = max_rows * G;
  // Rows of 16-bit types go in tiles where a head has more than 64; from 17 on where the others' rereading of the cache, once for 16 rows, is
  // 192k slots or more (32 heads, rows kernel and tiles: 64 rows over 1000 slots 22.5 and 23.4 us, over 4000 46.8 and 28.3, over 16000
  // 156 and 65; 24 rows over 1000 15.4 and 22.5, over 16000 89.6 and 60.8).  Where all sentences may be prompts the tiles take short ones too;
  // beside single tokens they leave those of up to 16 rows.
  p.in_tiles = c.dtype != CI_F32 && (R > 64 || (R > 16 && heads * ((R + 15) / 16) * max_len >= (int64_t)192 << 10));
  p.rows = !p.in_tiles || T < c.B * max_rows;
  p.few = !p.in_tiles ? 1 << 30 : p.rows ? 16 : 0;
  auto take = [&](size_t words) {
    const size_t at = p.bytes;
    p.bytes += (words * sizeof(float) + 255) / 256 * 256;
    return at;
  };
  if (p.rows) {
    const int64_t tiles = (std::min<int64_t>(R, p.few) + 15) / 16, steps = most_steps(32, max_rows, max_len, window, sinks);
    // Four workgroups a compute unit, of which two are at work at once and the others balance them (eight sentences to 65536 slots 178 us;
    // two 202, three 190, six 182); no piece below three steps a wave (4096 slots of 40 heads 20.5 us, two 22.7).
    const int64_t wanted = 4 * kCus;
    p.least = 12;
    // A head's slots stay together where they are few, or few for so many heads (whole and in pieces: 8 heads over 500 slots 11.0 and 14.5 us, over
    // 2000 22 and 14.5; 256 heads over 2000 48.7 and 55.7, over 12000 of one sentence and 300 of the others 111 and 24.5; 2400 heads over 4000 of one and
    // 300 of the others 89 and 125), where there would be more pieces than partial results are worth, and in fp32 prompts, whose tiles see only part
    // of the slots each.
    const bool whole = steps <= 16 || steps <= std::min<int64_t>(128, heads * tiles / 2) || heads * tiles > (tiles > 4 ? 2 : 16) * kCus;
    p.wanted = whole ? 0 : (int)(wanted / tiles);
    p.blocks = (int)heads + p.wanted;
    // Beyond 64 workgroups a compute unit one takes several tiles: only the sentences that have so many rows need them.
    p.row_tiles = (int)std::min<int64_t>({tiles, 65535, std::max<int64_t>(1, 64 * kCus / p.blocks)});
    if (p.wanted) {
      const size_t rows = (size_t)p.blocks * p.row_tiles * 16;
      p.place = take(2 * (size_t)c.B);
      p.m = take(rows);
      p.l = take(rows);
      p.o = take(rows * c.D);
    }
  }
  if (p.in_tiles) {
    p.tiles = (int)(T * G / kTileRows + c.B);   // see tile_start
    const int64_t full = (T * G + kTileRows - 1) / kTileRows * c.H, steps = most_steps(64, max_rows, max_len, window, sinks);
    // As many workgroups as fit at once (three a compute unit of 64 channels, two of 128: 512 rows over 16384 slots of 32 heads in 4 pieces 53 us,
    // in 3 56, in 5 70, in 8 65); no piece below eight steps, and no more partial results than of 8 kCus tiles, however many sentences
    // there may be.
    p.pieces = (int)std::max<int64_t>(1, std::min<int64_t>({(c.D == 64 ? 3 : 2) * kCus / full, steps / 8, kMaxPieces, 8 * kCus / (p.tiles * c.H)}));
    if (p.pieces > 1) {
      const size_t rows = (size_t)p.tiles * c.H * p.pieces * kTileRows;
      p.tile_m = take(rows);
      p.tile_l = take(rows);
      p.tile_exact = take(rows);
      p.tile_o = take(rows * c.D);
    }
  }
  return p;
}

}  // namespace

size_t kvp_attend_ws_bytes(const ci_kvp& c, int64_t T, int64_t G, int64_t max_rows, int64_t max_len, int64_t window, int64_t sinks) {
  return attend_plan(c, T, G, max_rows, max_len, window, sinks).bytes;
}

int launch_kvp_attend(const ci_kvp& c, const void* q, int64_t G, const int64_t (&stride)[2], int64_t T, const int32_t* first,
                      const int32_t* lens, int64_t max_rows, int64_t max_len, int64_t window, int64_t sinks, float scale, void* out,
                      float* lse, void* ws, hipStream_t s) {
  const AttendPlan p = attend_plan(c, T, G, max_rows, max_len, window, sinks);
  KvpAttend a = {};
  a.c = make_kvp(c);
  a.q = q;
  a.q_t = stride[0];
  a.q_h = stride[1];
  a.out = out;
  a.lse = lse;
  a.first = first;
  a.lens = lens;
  a.T = (int)T;
  a.G = (int)G;
  a.max_rows = (int)max_rows;
  a.max_len = (int)max_len;
  a.window = window >= max_len ? 0 : (int)window;   // everything is inside it
  a.sinks = (int)std::min(sinks, max_len);
  a.scale = (float)(scale * kLog2e);
  const int e = elem_bytes(c.dtype);
  a.q_vectors = aligned16(q) && stride[0] * e % 16 == 0 && stride[1] * e % 16 == 0;
  char* base = reinterpret_cast<char*>(ws);
  a.place = reinterpret_cast<int2*>(base + p.place);
  a.m = reinterpret_cast<float*>(base + p.m);
  a.l = reinterpret_cast<float*>(base + p.l);
  a.o = reinterpret_cast<float*>(base + p.o);
  a.few = p.few;
  a.row_tiles = p.row_tiles;
  a.blocks = p.blocks;
  a.wanted = p.wanted;
  a.least = p.least;
  a.join_rows = (int)std::max<int64_t>(1, std::min<int64_t>(max_rows, p.few / G));
  a.tiles = p.tiles;
  a.tile_rows = kTileRows;
  a.pieces = p.pieces;
  a.tile_m = reinterpret_cast<float*>(base + p.tile_m);
  a.tile_l = reinterpret_cast<float*>(base + p.tile_l);
  a.tile_exact = reinterpret_cast<float*>(base + p.tile_exact);
  a.tile_o = reinterpret_cast<float*>(base + p.tile_o);
  switch (c.dtype) {
    case CI_F32: return launch_kvp_attend_type<F32>(a, c.D, p.rows, p.in_tiles, s);
    case CI_F16: return launch_kvp_attend_type<F16>(a, c.D, p.rows, p.in_tiles, s);
    default: return launch_kvp_attend_type<BF16>(a, c.D, p.rows, p.in_tiles, s);
  }
}

}  // namespace ci
