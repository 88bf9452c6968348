// C ABI of the 4-bit operators: argument validation (host only, before any HIP call) and dispatch, in the manner of api.hip.
#include <math.h>

#include "common.hpp"

namespace ci {
namespace {

bool type_ok(int dt) { return dt == CI_F32 || dt == CI_F16 || dt == CI_BF16; }
bool group_ok(int group) { return group == 32 || group == 64 || group == 128; }
bool size_ok(int64_t n) { return n >= 1 && n <= CI_MAX_NEURONS; }
bool elem_aligned(const void* p, int dtype) { return reinterpret_cast<uintptr_t>(p) % elem_bytes(dtype) == 0; }
bool word_aligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

int shape_status(int64_t B, int64_t H, int64_t cap, int D, int group) {
  if (B < 1 || H < 1 || B > 65535 || H > 65535 || B * H > 65535 || cap < 1 || cap > CI_MAX_CACHE_SLOTS) return CI_ERR_INVALID_ARG;
  if (cap % 32 != 0) return CI_ERR_BAD_LAYOUT;
  if ((D != 64 && D != 128) || !group_ok(group) || group > D) return CI_ERR_UNSUPPORTED;
  return CI_OK;
}
int cache_status(const ci_kv4* c) {
  if (!c) return CI_ERR_INVALID_ARG;
  const int rc = shape_status(c->B, c->H, c->cap, c->D, c->group);
  if (rc != CI_OK) return rc;
  if (!c->k || !c->v || !c->k_scale || !c->v_scale) return CI_ERR_INVALID_ARG;
  if (!aligned16(c->k) || !aligned16(c->v) || !aligned16(c->k_scale) || !aligned16(c->v_scale) || !word_aligned(c->weight) ||
      !word_aligned(c->pos))
    return CI_ERR_BAD_LAYOUT;
  return CI_OK;
}
// Strides in elements that stay within 2^40, so that no offset of a call leaves 64 bits.
bool strides_ok(const int64_t* stride) {
  for (int i = 0; i < 3; ++i)
    if (stride[i] < 0 || stride[i] > ((int64_t)1 << 40)) return false;
  return true;
}

}  // namespace
}  // namespace ci

using namespace ci;

extern "C" {

int coreinfer_w4_size(int64_t R, int64_t C, int group, size_t* bytes) {
  if (!bytes || !size_ok(R) || !size_ok(C)) return CI_ERR_INVALID_ARG;
  if (!group_ok(group)) return CI_ERR_UNSUPPORTED;
  *bytes = w4_bytes(R, C, group);
  return CI_OK;
}

int coreinfer_w4_quantize(const void* w, int64_t R, int64_t C, int64_t ld, int dtype, int group, void* packed, void* stream) {
  if (!type_ok(dtype)) return CI_ERR_BAD_DTYPE;
  if (!w || !packed || !size_ok(R) || !size_ok(C)) return CI_ERR_INVALID_ARG;
  if (!group_ok(group)) return CI_ERR_UNSUPPORTED;
  if (ld < C || ld > ((int64_t)1 << 40) || !elem_aligned(w, dtype) || !aligned16(packed)) return CI_ERR_BAD_LAYOUT;
  return launch_w4_quantize(w, R, C, ld, dtype, group, packed, (hipStream_t)stream);
}

int coreinfer_w4_read(const void* packed, int64_t R, int64_t C, int group, void* w, int64_t ld, int dtype, void* stream) {
  if (!type_ok(dtype)) return CI_ERR_BAD_DTYPE;
  if (!w || !packed || !size_ok(R) || !size_ok(C)) return CI_ERR_INVALID_ARG;
  if (!group_ok(group)) return CI_ERR_UNSUPPORTED;
  if (ld < C || ld > ((int64_t)1 << 40) || !elem_aligned(w, dtype) || !aligned16(packed)) return CI_ERR_BAD_LAYOUT;
  return launch_w4_read(packed, R, C, group, w, ld, dtype, (hipStream_t)stream);
}

int coreinfer_w4_matvec_workspace_size(int64_t M, int64_t C, int x_dtype, size_t* bytes) {
  if (!type_ok(x_dtype)) return CI_ERR_BAD_DTYPE;
  if (!bytes || M < 1 || M > CI_MAX_W4_ROWS || !size_ok(C)) return CI_ERR_INVALID_ARG;
  *bytes = w4_matvec_ws_bytes(M, C, x_dtype);
  return CI_OK;
}

int coreinfer_w4_matvec(const void* x, int64_t M, int64_t ldx, int x_dtype, const void* w, const void* gate, const void* bias,
                        int bias_dtype, int act, int64_t R, int64_t C, int group, void* y, int64_t ldy, int y_dtype, void* ws,
                        size_t ws_bytes, void* stream) {
  if (!type_ok(x_dtype) || !type_ok(y_dtype) || (bias && !type_ok(bias_dtype)) ||
      (act != CI_ACT_NONE && act != CI_ACT_RELU && act != CI_ACT_SWIGLU))
    return CI_ERR_BAD_DTYPE;
  size_t need = 0;
  const int rc = coreinfer_w4_matvec_workspace_size(M, C, x_dtype, &need);
  if (rc != CI_OK) return rc;
  if (!x || !w || !y || !size_ok(R)) return CI_ERR_INVALID_ARG;
  if ((act == CI_ACT_SWIGLU) != (gate != nullptr) || (act == CI_ACT_SWIGLU && bias)) return CI_ERR_INVALID_ARG;
  if (!group_ok(group)) return CI_ERR_UNSUPPORTED;
  if (ldx < C || ldy < R || ldx > ((int64_t)1 << 40) || ldy > ((int64_t)1 << 40)) return CI_ERR_BAD_LAYOUT;
  if (!elem_aligned(x, x_dtype) || !elem_aligned(y, y_dtype) || (bias && !elem_aligned(bias, bias_dtype)) || !aligned16(w) ||
      !aligned16(gate))
    return CI_ERR_BAD_LAYOUT;
  if (need && (!ws || ws_bytes < need)) return CI_ERR_WORKSPACE;
  if (need && !aligned16(ws)) return CI_ERR_BAD_LAYOUT;
  return launch_w4_matvec(x, M, ldx, x_dtype, w, gate, bias, bias_dtype, act, R, C, group, y, ldy, y_dtype, ws, (hipStream_t)stream);
}

int coreinfer_kv4_sizes(int64_t B, int64_t H, int64_t cap, int D, int group, size_t* codes_bytes, size_t* scale_bytes) {
  const int rc = shape_status(B, H, cap, D, group);
  if (rc != CI_OK) return rc;
  if (!codes_bytes || !scale_bytes) return CI_ERR_INVALID_ARG;
  *codes_bytes = (size_t)(B * H) * (size_t)cap * (size_t)(D / 2);
  *scale_bytes = (size_t)(B * H) * (size_t)cap * (size_t)(D / group) * sizeof(uint32_t);
  return CI_OK;
}

int coreinfer_kv4_append(const ci_kv4* cache, const void* k, const void* v, int64_t S, const int64_t* stride, int dtype,
                         const int32_t* start, const int32_t* lens, const int32_t* next, void* stream) {
  if (!type_ok(dtype)) return CI_ERR_BAD_DTYPE;
  const int rc = cache_status(cache);
  if (rc != CI_OK) return rc;
  if (!k || !v || !stride || !lens || S < 1 || S > (1 << 19)) return CI_ERR_INVALID_ARG;
  if (!strides_ok(stride) || !elem_aligned(k, dtype) || !elem_aligned(v, dtype) || !word_aligned(start) || !word_aligned(lens) ||
      !word_aligned(next))
    return CI_ERR_BAD_LAYOUT;
  return launch_kv4_append(*cache, k, v, S, {stride[0], stride[1], stride[2]}, dtype, start, lens, next, (hipStream_t)stream);
}

int coreinfer_kv4_read(const ci_kv4* cache, const int32_t* lens, int64_t first, int64_t count, void* k, void* v, int dtype,
                       void* stream) {
  if (!type_ok(dtype)) return CI_ERR_BAD_DTYPE;
  const int rc = cache_status(cache);
  if (rc != CI_OK) return rc;
  if (!lens || !k || !v || first < 0 || count < 1 || count > cache->cap || first > cache->cap - count) return CI_ERR_INVALID_ARG;
  if (!word_aligned(lens) || !aligned16(k) || !aligned16(v)) return CI_ERR_BAD_LAYOUT;
  return launch_kv4_read(*cache, lens, first, count, k, v, dtype, (hipStream_t)stream);
}

int coreinfer_kv4_attend_workspace_size(int64_t B, int64_t H, int D, int64_t S, int64_t Hq, int64_t max_len, int weights,
                                        size_t* bytes) {
  const int rc = shape_status(B, H, 32, D, 32);
  if (rc != CI_OK) return rc;
  if (!bytes || S < 1 || S > (1 << 20) || Hq < H || Hq > ((int64_t)1 << 32) || Hq % H != 0 || Hq / H > 4096 ||
      S * (Hq / H) > (1 << 20) || max_len < 1 ||
      max_len > CI_MAX_CACHE_SLOTS)
    return CI_ERR_INVALID_ARG;
  *bytes = kv4_attend_ws_bytes(B * H, D, S, Hq / H, max_len, weights != 0);
  return CI_OK;
}

int coreinfer_kv4_attend(const ci_kv4* cache, const void* q, int64_t S, int64_t Hq, const int64_t* stride, int dtype, float scale,
                         const int32_t* lens, int64_t max_len, void* out, float* lse, float* weight_out, void* ws,
                         size_t ws_bytes, void* stream) {
  if (!type_ok(dtype)) return CI_ERR_BAD_DTYPE;
  int rc = cache_status(cache);
  if (rc != CI_OK) return rc;
  size_t need = 0;
  rc = coreinfer_kv4_attend_workspace_size(cache->B, cache->H, cache->D, S, Hq, max_len, weight_out != nullptr, &need);
  if (rc != CI_OK) return rc;
  if (!q || !stride || !lens || !out || max_len > cache->cap || (weight_out && !cache->weight)) return CI_ERR_INVALID_ARG;
  if (!(scale > 0.0f) || !isfinite(scale * 1.442695041f)) return CI_ERR_INVALID_ARG;   // the kernels multiply by scale log2(e)
  if (!strides_ok(stride) || !elem_aligned(q, dtype) || !aligned16(out) || !word_aligned(lens) || !word_aligned(lse) ||
      !word_aligned(weight_out))
    return CI_ERR_BAD_LAYOUT;
  if (!ws || ws_bytes < need) return CI_ERR_WORKSPACE;
  if (!aligned16(ws)) return CI_ERR_BAD_LAYOUT;
  return launch_kv4_attend(*cache, q, S, Hq / cache->H, {stride[0], stride[1], stride[2]}, dtype, scale, lens, max_len, out, lse,
                           weight_out, ws, (hipStream_t)stream);
}

int coreinfer_kv4_evict_workspace_size(int64_t B, int64_t H, int64_t max_len, int64_t budget, size_t* bytes) {
  if (!bytes || B < 1 || H < 1 || B > 65535 || H > 65535 || B * H > 65535 || max_len < 1 || max_len > CI_MAX_CACHE_SLOTS ||
      budget < 1 || budget > CI_MAX_CACHE_SLOTS)
    return CI_ERR_INVALID_ARG;
  *bytes = kv4_evict_ws_bytes(B * H, max_len, budget);
  return CI_OK;
}

int coreinfer_kv4_evict(const ci_kv4* cache, const int32_t* lens, const int32_t* next, int64_t max_len, int64_t budget,
                        int64_t recent, float* weight_out, int32_t* pos_out, int32_t* lens_out, void* ws, size_t ws_bytes,
                        void* stream) {
  int rc = cache_status(cache);
  if (rc != CI_OK) return rc;
  size_t need = 0;
  rc = coreinfer_kv4_evict_workspace_size(cache->B, cache->H, max_len, budget, &need);
  if (rc != CI_OK) return rc;
  if (!cache->weight || !cache->pos || !lens || !next || !weight_out || !pos_out || max_len > cache->cap || recent < 0 ||
      recent > budget)
    return CI_ERR_INVALID_ARG;
  if (!word_aligned(lens) || !word_aligned(next) || !word_aligned(weight_out) || !word_aligned(pos_out) || !word_aligned(lens_out))
    return CI_ERR_BAD_LAYOUT;
  if (!ws || ws_bytes < need) return CI_ERR_WORKSPACE;
  if (!aligned16(ws)) return CI_ERR_BAD_LAYOUT;
  return launch_kv4_evict(*cache, lens, next, max_len, budget, recent, weight_out, pos_out, lens_out, ws, (hipStream_t)stream);
}

}  // extern "C"
