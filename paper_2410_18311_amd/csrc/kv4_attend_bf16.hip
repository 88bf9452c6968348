// Attention over a cache in 4 bits: the bf16 kernels (kv4_attend.hpp).
#include "kv4_attend.hpp"

namespace ci {
template int launch_kv4_attend_type<BF16>(const Kv4Attend& a, int head_dim, int group, hipStream_t s);
}  // namespace ci
