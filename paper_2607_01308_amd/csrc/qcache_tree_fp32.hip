// Tree attention (qcache_tree.h) for fp32 queries.
#include "qcache_tree.h"

namespace cm {

hipError_t launch_tree_fp32(const TreeAttention& a, int32_t d, int32_t tiles, hipStream_t stream) {
  return launch_tree<3>(a, d, tiles, stream);
}

}  // namespace cm
