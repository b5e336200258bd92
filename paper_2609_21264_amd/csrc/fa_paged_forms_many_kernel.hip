// Attention of many new tokens per sequence over the paged cache with forms: scores capped or biased by distance, windows,
// prefixes and trees of drafted tokens. Instances of the kernel in fa_paged_many.h.
#include <hip/hip_runtime.h>

#include "fa_paged_many.h"

namespace fa {

namespace {
template <int DQK, int DV, bool E4M3>
hipError_t launch_dims(const PagedParams& p, const PagedMany& m, hipStream_t stream) {
  constexpr bool SHORT = !E4M3 && DQK != 192;  // as paged_many has it
  return m.split ? launch_many<typename PagedInstance<DQK, DV, E4M3, SHORT, true, true>::C>(p, m.blocks, stream)
                 : launch_many<typename PagedInstance<DQK, DV, E4M3, SHORT, false, true>::C>(p, m.blocks, stream);
}
}  // namespace

hipError_t launch_paged_many_forms(PagedParams p, const PagedMany& m, int d_qk, bool e4m3, hipStream_t stream) {
  many_constants(p);
  if (d_qk == 64) return e4m3 ? launch_dims<64, 64, true>(p, m, stream) : launch_dims<64, 64, false>(p, m, stream);
  if (d_qk == 128) return e4m3 ? launch_dims<128, 128, true>(p, m, stream) : launch_dims<128, 128, false>(p, m, stream);
  return e4m3 ? launch_dims<192, 128, true>(p, m, stream) : launch_dims<192, 128, false>(p, m, stream);
}

}  // namespace fa
