// Attention of drafted tokens over a cache of e4m3 rows.
#include "attn_tree.h"

namespace hstu {
namespace tree {

hipError_t launch_e4m3(const TreeArgs& a, const TreeSplit& sp, hipStream_t s) {
  return launch<kCacheE4m3>(a, sp, s);
}

}  // namespace tree
}  // namespace hstu
