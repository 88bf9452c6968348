// Attention over a cache in 4 bits: how a call is split over the chip (the kernels are in kv4_attend.hpp).
#include <algorithm>

#include "kv4.hpp"

namespace ci {
namespace {

constexpr int kCus = 256;   // of an MI355X; a workspace query knows no device
constexpr double kLog2e = 1.4426950408889634;

struct AttendPlan {
  int R, row_tiles, token_waves, blocks, wanted, least, weights;
  size_t place, m, l, o, z, logits, bytes;   // places in the workspace
};

AttendPlan attend_plan(int64_t heads, int D, int64_t S, int64_t G, int64_t max_len, bool weights) {
  AttendPlan p;
  p.R = (int)(S * G);
  p.row_tiles = (p.R + 15) / 16;
  p.weights = !weights ? 0 : p.R <= 16 ? 1 : 2;
  p.token_waves = p.row_tiles >= 4 ? 1 : 4;
  const int64_t row_blocks = p.token_waves == 4 ? p.row_tiles : (p.row_tiles + 3) / 4;
  const int64_t steps = (max_len + 31) / 32, blocks = heads * row_blocks;
  // Three workgroups a compute unit (what the registers leave room for), two where waves share the rows (whose partial results are many); no
  // piece below two steps a wave, respectively 16 steps.
  const int64_t wanted = (p.token_waves == 4 ? 3 : 2) * kCus;
  p.least = p.token_waves == 4 ? 8 : 16;
  p.wanted = blocks * 2 > wanted || steps <= p.least ? 0 : (int)(wanted / row_blocks);
  p.blocks = (int)heads + p.wanted;
  auto take = [&](size_t floats) {
    const size_t at = p.bytes;
    p.bytes += (floats * sizeof(float) + 255) / 256 * 256;
    return at;
  };
  p.bytes = 0;
  const size_t rows = p.wanted ? (size_t)p.blocks * p.row_tiles * 16 : 0;
  p.place = take(p.wanted ? 2 * (size_t)heads : 0);   // as many sentences at most
  p.m = take(rows);
  p.l = take(rows);
  p.o = take(rows * D);
  p.z = take(p.weights ? (size_t)heads * p.R : 0);
  p.logits = take(p.weights == 1 ? (size_t)heads * p.R * steps * 32 : 0);
  p.bytes += 256;
  return p;
}

}  // namespace

size_t kv4_attend_ws_bytes(int64_t heads, int D, int64_t S, int64_t G, int64_t max_len, bool weights) {
  return attend_plan(heads, D, S, G, max_len, weights).bytes;
}

int launch_kv4_attend(const ci_kv4& c, const void* q, int64_t S, int64_t G, const int64_t (&stride)[3], int dtype, float scale,
                      const int32_t* lens, int64_t max_len, void* out, float* lse, float* weight_out, void* ws, hipStream_t s) {
  const AttendPlan p = attend_plan(c.B * c.H, c.D, S, G, max_len, weight_out != nullptr);
  Kv4Attend a;
  a.c = Kv4{reinterpret_cast<uint32_t*>(c.k), reinterpret_cast<uint32_t*>(c.v), c.k_scale, c.v_scale, c.weight, c.pos,
            (int)c.B, (int)c.H, (int)c.cap};
  a.q = q;
  a.q_b = stride[0];
  a.q_s = stride[1];
  a.q_h = stride[2];
  a.out = out;
  a.lse = lse;
  a.weight_out = weight_out;
  a.lens = lens;
  a.S = (int)S;
  a.G = (int)G;
  a.inverse_G = (uint32_t)((((uint64_t)1 << 32) + G - 1) / G);
  a.R = p.R;
  a.max_len = (int)max_len;
  a.scale = (float)(scale * kLog2e);
  const int e = elem_bytes(dtype);
  a.q_vectors = aligned16(q) && stride[0] * e % 16 == 0 && stride[1] * e % 16 == 0 && stride[2] * e % 16 == 0;
  char* base = reinterpret_cast<char*>(ws);
  a.place = reinterpret_cast<int2*>(base + p.place);
  a.m = reinterpret_cast<float*>(base + p.m);
  a.l = reinterpret_cast<float*>(base + p.l);
  a.o = reinterpret_cast<float*>(base + p.o);
  a.z = reinterpret_cast<float*>(base + p.z);
  a.logits = reinterpret_cast<float*>(base + p.logits);
  a.blocks = p.blocks;
  a.wanted = p.wanted;
  a.least = p.least;
  a.row_tiles = p.row_tiles;
  a.token_waves = p.token_waves;
  a.weights = p.weights;
  switch (dtype) {
    case CI_F32: return launch_kv4_attend_type<F32>(a, c.D, c.group, s);
    case CI_F16: return launch_kv4_attend_type<F16>(a, c.D, c.group, s);
    default: return launch_kv4_attend_type<BF16>(a, c.D, c.group, s);
  }
}

}  // namespace ci
