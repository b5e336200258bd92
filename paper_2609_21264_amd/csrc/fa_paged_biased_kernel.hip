// Attention of many new tokens per sequence over the paged cache with scores biased by distance (and capped, windows, prefixes).
#include "fa_paged_forms_many.h"

namespace fa {

hipError_t launch_paged_many_biased(const PagedParams& p, const PagedMany& m, int d_qk, bool e4m3, hipStream_t stream) {
  return launch_form<kFormBiased>(p, m, d_qk, e4m3, stream);
}

}  // namespace fa
