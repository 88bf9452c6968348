// Attention over a cache in pages: the f16 kernels.
#include "kvp_mixed.hpp"

namespace ci {
template <> int launch_kvp_attend_type<F16>(const KvpAttend& a, int D, bool rows, bool tiles, hipStream_t s) {
  return D == 64 ? launch_16bit<F16, 64>(a, rows, tiles, s) : launch_16bit<F16, 128>(a, rows, tiles, s);
}
}  // namespace ci
