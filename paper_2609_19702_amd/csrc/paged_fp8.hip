#include "paged_attn.h"

namespace dsa {

hipError_t launch_paged_fp8(const Derived& d, const PagedLaunch& l, const PagedArgs& a,
                             hipStream_t st) {
  return d.D == 64 ? launch_paged<true, 64>(l, a, st) : launch_paged<true, 128>(l, a, st);
}

}  // namespace dsa
