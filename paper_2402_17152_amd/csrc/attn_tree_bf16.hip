// Attention of drafted tokens over a cache of bf16 rows.
#include "attn_tree.h"

namespace hstu {
namespace tree {

hipError_t launch_bf16(const TreeArgs& a, const TreeSplit& sp, hipStream_t s) {
  return launch<kCacheBf16>(a, sp, s);
}

}  // namespace tree
}  // namespace hstu
