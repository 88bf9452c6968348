// C ABI of rotary positions and the cache in pages: argument validation (host only, before any HIP call) and dispatch, in the manner of api.hip.
#include <math.h>

#include <algorithm>

#include "common.hpp"

namespace ci {
namespace {

bool type_ok(int dt) { return dt == CI_F32 || dt == CI_F16 || dt == CI_BF16; }
bool elem_aligned(const void* p, int dtype) { return reinterpret_cast<uintptr_t>(p) % elem_bytes(dtype) == 0; }
bool word_aligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }
// Strides in elements that stay within 2^40, so that no offset of a call leaves 64 bits.
bool strides_ok(const int64_t* stride) {
  for (int i = 0; i < 2; ++i)
    if (stride[i] < 0 || stride[i] > ((int64_t)1 << 40)) return false;
  return true;
}
// Whether two of a, b rows that are stride[0], stride[1] apart, D elements each, share an element (or lie in one another).
bool rows_overlap(const int64_t* stride, int64_t a, int64_t b, int64_t D) {
  const bool swap = stride[0] < stride[1];
  const int64_t inner = swap ? stride[0] : stride[1], outer = swap ? stride[1] : stride[0], n = swap ? a : b, m = swap ? b : a;
  return (n > 1 && inner < D) || (m > 1 && outer < (n > 1 ? (n - 1) * inner : 0) + D);
}
// Whether one of the T x H rows of `bytes` that begin stride[0], stride[1] bytes apart from p on has a byte in the block from .. from + size.
bool rows_touch(const void* p, const int64_t (&stride)[2], int64_t T, int64_t H, int64_t bytes, const void* from, int64_t size) {
  const int64_t at = (int64_t)reinterpret_cast<uintptr_t>(p), begin = (int64_t)reinterpret_cast<uintptr_t>(from), end = begin + size;
  const bool swap = stride[0] < stride[1];
  const int64_t inner = swap ? stride[0] : stride[1], outer = swap ? stride[1] : stride[0], n = swap ? T : H, m = swap ? H : T;
  const int64_t extent = (n - 1) * inner + bytes;   // of the rows that are `inner` apart
  if (end <= at || begin >= at + (m - 1) * outer + extent) return false;
  // the first index from which on rows `step` apart from `a` on reach past `begin`
  auto past = [&](int64_t a, int64_t length, int64_t step) { return a + length > begin || step == 0 ? 0 : (begin - a - length) / step + 1; };
  for (int64_t i = past(at, extent, outer); i < m && at + i * outer < end; ++i) {
    const int64_t a = at + i * outer, j = past(a, bytes, inner);
    if (j < n && a + j * inner < end && a + j * inner + bytes > begin) return true;
    if (outer == 0) break;
  }
  return false;
}
// Whether rows of D elements share a byte with the T H D elements from `out` on.
bool touches(const void* p, const int64_t* stride, int64_t T, int64_t H, int64_t D, int dtype, const void* out) {
  const int64_t e = elem_bytes(dtype);
  return rows_touch(p, {stride[0] * e, stride[1] * e}, T, H, D * e, out, T * H * D * e);
}
// The same of two sets of rows with the same strides, or of which one is a block; others are not looked at.
bool rope_overlap(const void* x, const int64_t* stride, int64_t T, int64_t H, int64_t D, int dtype, const void* y, const int64_t* y_stride, bool same) {
  auto block = [&](const int64_t* s) { return (T == 1 || s[0] == H * D) && (H == 1 || s[1] == D); };
  if (block(y_stride)) return touches(x, stride, T, H, D, dtype, y);
  if (block(stride)) return touches(y, y_stride, T, H, D, dtype, x);
  if (!same) return false;
  // a row of one set on a row of the other: their distance on one of the differences between two rows of a set
  const int64_t e = elem_bytes(dtype), back = ((T - 1) * stride[0] + (H - 1) * stride[1]) * e;
  return rows_touch(reinterpret_cast<const void*>((uintptr_t)((int64_t)(uintptr_t)x - back)), {stride[0] * e, stride[1] * e}, 2 * T - 1, 2 * H - 1, D * e,
                    y, D * e);
}

int rope_status(const ci_rope* r, int64_t D) {
  if (!r) return CI_OK;
  if (r->style != CI_ROPE_HALF && r->style != CI_ROPE_INTERLEAVED) return CI_ERR_BAD_DTYPE;
  if (r->rot < 0 || r->rot > D || r->rot % 2 != 0 || !isfinite(r->scale) || (r->rot > 0 && !r->turns)) return CI_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(r->turns) % 8 != 0) return CI_ERR_BAD_LAYOUT;
  return CI_OK;
}
int cache_status(const ci_kvp* c) {
  if (!c) return CI_ERR_INVALID_ARG;
  if (!type_ok(c->dtype)) return CI_ERR_BAD_DTYPE;
  if (c->B < 1 || c->H < 1 || c->B > 65535 || c->H > 65535 || c->B * c->H > 65535 || c->pages < 1 || c->pages > INT32_MAX || c->most < 1 ||
      c->most > CI_MAX_CACHE_SLOTS)
    return CI_ERR_INVALID_ARG;
  if ((c->D != 64 && c->D != 128) || c->page < 16 || c->page > 256 || (c->page & (c->page - 1)) != 0) return CI_ERR_UNSUPPORTED;
  if (c->most * c->page > CI_MAX_CACHE_SLOTS || !c->k || !c->v || !c->table) return CI_ERR_INVALID_ARG;
  if (!aligned16(c->k) || !aligned16(c->v) || !word_aligned(c->table)) return CI_ERR_BAD_LAYOUT;
  return CI_OK;
}
bool eps_ok(const void* norm, float eps) { return !norm || (eps >= 0.0f && isfinite(eps)); }

}  // namespace
}  // namespace ci

using namespace ci;

extern "C" {

int coreinfer_rope_turns(int64_t rot, double base, int scaling, double factor, double original, double fast, double slow,
                         uint64_t* turns) {
  if (scaling < CI_ROPE_PLAIN || scaling > CI_ROPE_PARTS) return CI_ERR_BAD_DTYPE;
  if (!turns || rot < 2 || rot > CI_MAX_ROPE_CHANNELS || rot % 2 != 0 || !(base > 0.0) || !isfinite(base)) return CI_ERR_INVALID_ARG;
  if (scaling != CI_ROPE_PLAIN && (!(factor > 0.0) || !isfinite(factor))) return CI_ERR_INVALID_ARG;
  if (scaling == CI_ROPE_PARTS && (!(original > 0.0) || !isfinite(original) || !(fast > slow) || !isfinite(fast) || !isfinite(slow)))
    return CI_ERR_INVALID_ARG;
  const double two_pi = 6.283185307179586476925;
  if (scaling == CI_ROPE_BASE && rot > 2) base *= pow(factor, (double)rot / (double)(rot - 2));
  for (int64_t i = 0; i < rot / 2; ++i) {
    double f = pow(base, -2.0 * (double)i / (double)rot);
    if (scaling == CI_ROPE_LINEAR) f /= factor;
    if (scaling == CI_ROPE_PARTS) {
      const double g = std::min(1.0, std::max(0.0, (original * f / two_pi - slow) / (fast - slow)));
      f *= g + (1.0 - g) / factor;
    }
    if (!isfinite(f)) return CI_ERR_INVALID_ARG;
    const double turn = f / two_pi;
    turns[i] = (uint64_t)ldexp(turn - floor(turn), 64);   // below 1, so below 2^64
  }
  return CI_OK;
}

int coreinfer_rope(const void* x, const int64_t* stride, int64_t T, int64_t H, int64_t D, int dtype, const void* norm, float eps,
                   const ci_rope* rope, const int32_t* pos, int backward, void* y, const int64_t* y_stride, void* stream) {
  if (!type_ok(dtype)) return CI_ERR_BAD_DTYPE;
  if (T < 0 || T > CI_MAX_PACKED_ROWS || H < 1 || H > 65535 || D < 1 || D > CI_MAX_ROPE_CHANNELS) return CI_ERR_INVALID_ARG;
  const int rc = rope_status(rope, D);
  if (rc != CI_OK) return rc;
  if ((backward && norm) || !eps_ok(norm, eps)) return CI_ERR_INVALID_ARG;
  if (T == 0) return CI_OK;
  if (!x || !y || !stride || !y_stride || (rope && rope->rot > 0 && !pos)) return CI_ERR_INVALID_ARG;
  if (!strides_ok(stride) || !strides_ok(y_stride) || !elem_aligned(x, dtype) || !elem_aligned(y, dtype) || !elem_aligned(norm, dtype) ||
      !word_aligned(pos))
    return CI_ERR_BAD_LAYOUT;
  if (rows_overlap(y_stride, T, H, D)) return CI_ERR_BAD_LAYOUT;
  // strides of lengths of one say nothing
  const bool same = (T == 1 || stride[0] == y_stride[0]) && (H == 1 || stride[1] == y_stride[1]);
  if (x == y ? !same : rope_overlap(x, stride, T, H, D, dtype, y, y_stride, same)) return CI_ERR_BAD_LAYOUT;
  return launch_rope(x, {stride[0], stride[1]}, T, H, D, dtype, norm, eps, rope, pos, backward != 0, y, {y_stride[0], y_stride[1]},
                     (hipStream_t)stream);
}

int coreinfer_kvp_append(const ci_kvp* cache, const void* k, const void* v, const int64_t* stride, int64_t T, const int32_t* first,
                         const int32_t* lens, const int32_t* pos, const ci_rope* rope, const void* k_norm, float eps, const void* q,
                         int64_t Hq, const int64_t* q_stride, const void* q_norm, void* q_out, void* stream) {
  int rc = cache_status(cache);
  if (rc != CI_OK) return rc;
  const int dtype = cache->dtype;
  if (T < 0 || T > CI_MAX_PACKED_ROWS || Hq < 0 || Hq > 65535) return CI_ERR_INVALID_ARG;
  rc = rope_status(rope, cache->D);
  if (rc != CI_OK) return rc;
  if (!eps_ok(k_norm, eps) || !eps_ok(q_norm, eps)) return CI_ERR_INVALID_ARG;
  if (T == 0) return CI_OK;
  if (!k || !v || !stride || !first || !lens) return CI_ERR_INVALID_ARG;
  if ((Hq > 0) != (q != nullptr) || (Hq > 0) != (q_out != nullptr) || (q && !q_stride) || (!q && q_norm)) return CI_ERR_INVALID_ARG;
  if (!strides_ok(stride) || (q && !strides_ok(q_stride)) || !elem_aligned(k, dtype) || !elem_aligned(v, dtype) ||
      !elem_aligned(q, dtype) || !elem_aligned(k_norm, dtype) || !elem_aligned(q_norm, dtype) || !aligned16(q_out) || !word_aligned(first) ||
      !word_aligned(lens) || !word_aligned(pos))
    return CI_ERR_BAD_LAYOUT;
  if (q && touches(q, q_stride, T, Hq, cache->D, dtype, q_out)) return CI_ERR_BAD_LAYOUT;
  const int64_t none[2] = {0, 0};
  const int64_t* qs = q ? q_stride : none;
  return launch_kvp_append(*cache, k, v, {stride[0], stride[1]}, T, first, lens, pos, rope, k_norm, eps, q, Hq, {qs[0], qs[1]}, q_norm,
                           q_out, (hipStream_t)stream);
}

int coreinfer_kvp_attend_workspace_size(const ci_kvp* cache, int64_t T, int64_t Hq, int64_t max_rows, int64_t max_len, int64_t window,
                                        int64_t sinks, size_t* bytes) {
  const int rc = cache_status(cache);
  if (rc != CI_OK) return rc;
  if (!bytes || T < 0 || T > CI_MAX_PACKED_ROWS || Hq < cache->H || Hq % cache->H != 0 || Hq / cache->H > 4096 ||
      T * Hq > ((int64_t)1 << 30) || max_rows < 1 || max_rows > CI_MAX_PACKED_ROWS || max_len < 1 ||
      max_len > cache->most * cache->page || window < 0 || sinks < 0 || window > INT64_MAX / 2 || sinks > INT64_MAX / 2)
    return CI_ERR_INVALID_ARG;
  *bytes = T == 0 ? 0 : kvp_attend_ws_bytes(*cache, T, Hq / cache->H, std::min(max_rows, T), max_len, window, sinks);
  return CI_OK;
}

int coreinfer_kvp_attend(const ci_kvp* cache, const void* q, int64_t Hq, const int64_t* stride, int64_t T, const int32_t* first,
                         const int32_t* lens, int64_t max_rows, int64_t max_len, int64_t window, int64_t sinks, float scale, void* out,
                         float* lse, void* ws, size_t ws_bytes, void* stream) {
  size_t need = 0;
  const int rc = coreinfer_kvp_attend_workspace_size(cache, T, Hq, max_rows, max_len, window, sinks, &need);
  if (rc != CI_OK) return rc;
  if (!(scale > 0.0f) || !isfinite(scale * 1.442695041f)) return CI_ERR_INVALID_ARG;   // the kernels multiply by scale log2(e)
  if (T == 0) return CI_OK;
  if (!q || !stride || !first || !lens || !out) return CI_ERR_INVALID_ARG;
  if (!strides_ok(stride) || !elem_aligned(q, cache->dtype) || !aligned16(out) || !word_aligned(first) || !word_aligned(lens) ||
      !word_aligned(lse))
    return CI_ERR_BAD_LAYOUT;
  if (need && (!ws || ws_bytes < need)) return CI_ERR_WORKSPACE;
  if (need && !aligned16(ws)) return CI_ERR_BAD_LAYOUT;
  if (touches(q, stride, T, Hq, cache->D, cache->dtype, out)) return CI_ERR_BAD_LAYOUT;
  return launch_kvp_attend(*cache, q, Hq / cache->H, {stride[0], stride[1]}, T, first, lens, std::min(max_rows, T), max_len, window, sinks,
                           scale, out, lse, ws, (hipStream_t)stream);
}

}  // extern "C"
