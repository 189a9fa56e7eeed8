// dsa_tree_attention over fp8 caches.
#include "tree_attn.h"

namespace dsa {

hipError_t launch_tree_fp8(const Derived& d, const TreeLaunch& l, const TreeArgs& a, bool f32,
                           hipStream_t st) {
  return launch_tree<true>(d, l, a, f32, st);
}

}  // namespace dsa
