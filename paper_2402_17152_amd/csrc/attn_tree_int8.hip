// Attention of drafted tokens over a cache of int8 rows.
#include "attn_tree.h"

namespace hstu {
namespace tree {

hipError_t launch_int8(const TreeArgs& a, const TreeSplit& sp, hipStream_t s) {
  return launch<kCacheInt8>(a, sp, s);
}

}  // namespace tree
}  // namespace hstu
