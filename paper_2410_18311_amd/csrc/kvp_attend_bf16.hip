// Attention over a cache in pages: the bf16 kernels.
#include "kvp_mixed.hpp"

namespace ci {
template <> int launch_kvp_attend_type<BF16>(const KvpAttend& a, int D, bool rows, bool tiles, hipStream_t s) {
  return D == 64 ? launch_16bit<BF16, 64>(a, rows, tiles, s) : launch_16bit<BF16, 128>(a, rows, tiles, s);
}
}  // namespace ci
