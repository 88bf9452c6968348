// Attention over a cache in pages: the f16 kernels (kvp_rows.hpp, kvp_tiles.hpp).
#include "kvp_rows.hpp"
#include "kvp_tiles.hpp"

namespace ci {
template <> int launch_kvp_attend_type<F16>(const KvpAttend& a, int D, bool rows, bool tiles, hipStream_t s) {
  int rc = CI_OK;
  if (tiles) rc = D == 64 ? launch_tiles<F16, 64, 4>(a, s) : launch_tiles<F16, 128, 4>(a, s);
  if (rows && rc == CI_OK) rc = D == 64 ? launch_rows<F16, 64>(a, s) : launch_rows<F16, 128>(a, s);
  return rc;
}
}  // namespace ci
