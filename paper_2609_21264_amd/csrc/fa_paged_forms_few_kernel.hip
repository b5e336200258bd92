// Attention of few new tokens per sequence over the paged cache with forms: scores capped or biased by distance, windows,
// prefixes and trees of drafted tokens. Instances of the kernel in fa_paged_few.h.
#include <hip/hip_runtime.h>

#include "fa_paged_few.h"

namespace fa {

namespace {
template <int QB>
hipError_t launch_dims(const PagedParams& p, int d_qk, bool fp8, hipStream_t stream) {
  if (d_qk == 64)
    return fp8 ? launch_few<typename FewInstance<64, 64, true, QB, QB == 1, true>::C>(p, stream)
               : launch_few<typename FewInstance<64, 64, false, QB, QB == 1, true>::C>(p, stream);
  if (d_qk == 128)
    return fp8 ? launch_few<typename FewInstance<128, 128, true, QB, QB == 1, true>::C>(p, stream)
               : launch_few<typename FewInstance<128, 128, false, QB, QB == 1, true>::C>(p, stream);
  return fp8 ? launch_few<typename FewInstance<192, 128, true, QB, QB == 1, true>::C>(p, stream)
             : launch_few<typename FewInstance<192, 128, false, QB, QB == 1, true>::C>(p, stream);
}
}  // namespace

// Items of 64 row-heads, of which a sequence mostly has several, go through the caches; items of 32 past them. Through the caches
// against past them, us: two items a sequence and head, 16 trees of 26 tokens over 4 000 keys, 32/8 heads, d = 128 89.7 : 92.6, 24 x 24
// capped tokens over 2 000 keys 89.8 : 90.6 (e4m3 84.3 : 82.8, 86.8 : 87.0); where there is one, past them would be faster: 32 trees of 12
// over 3 000 keys 86.9 : 73.6 (e4m3 68.0 : 63.1), 8 of 16 over 9 000 70.4 : 63.2 (57.9 : 57.5), 40 of 33, 16/16 heads, d = 64, 65.8 : 60.6.
hipError_t launch_paged_few_forms(PagedParams p, int d_qk, bool fp8, int col_blocks, hipStream_t stream) {
  few_constants(p);
  return col_blocks == 1 ? launch_dims<1>(p, d_qk, fp8, stream) : launch_dims<2>(p, d_qk, fp8, stream);
}

}  // namespace fa
