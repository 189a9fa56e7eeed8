// dsa_tree_attention over bf16 caches.
#include "tree_attn.h"

namespace dsa {

hipError_t launch_tree_bf16(const Derived& d, const TreeLaunch& l, const TreeArgs& a, bool f32,
                            hipStream_t st) {
  return launch_tree<false>(d, l, a, f32, st);
}

}  // namespace dsa
