// Attention over a cache in pages: the f32 kernels (kvp_rows.hpp).
#include "kvp_rows.hpp"

namespace ci {
template <> int launch_kvp_attend_type<F32>(const KvpAttend& a, int D, bool, bool, hipStream_t s) {
  return D == 64 ? launch_rows<F32, 64>(a, s) : launch_rows<F32, 128>(a, s);
}
}  // namespace ci
