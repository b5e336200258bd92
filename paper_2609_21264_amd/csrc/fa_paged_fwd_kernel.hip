// Attention of many new tokens per sequence over a paged key/value cache (gfx950): the instances of the kernel in
// fa_paged_many.h, the choice between them, and their launches.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "fa_paged_many.h"

namespace fa {
namespace {

// Where there is a short instance, the long one runs only grids that fill the chip (paged_many): it is never split.
template <int DQK, int DV, bool E4M3, bool SHORT>
hipError_t launch_many_split(const PagedParams& p, const PagedMany& m, hipStream_t stream) {
  if constexpr (SHORT || E4M3 || DQK == 192) {
    if (m.split) return launch_many<typename PagedInstance<DQK, DV, E4M3, SHORT, true>::C>(p, m.blocks, stream);
  }
  return launch_many<typename PagedInstance<DQK, DV, E4M3, SHORT, false>::C>(p, m.blocks, stream);
}

}  // namespace

PagedMany paged_many(int n_seq, int n_tokens, int max_keys, int hkv, int group, int max_q, int few_cols, int d_qk, bool e4m3,
                     bool forms) {
  PagedMany m{};
  const int64_t rows = (int64_t)n_tokens * group;
  int64_t seqs = rows / (few_cols + 1);
  if (seqs > n_seq) seqs = n_seq;
  // Short blocks where sequences have no more, and where long ones would not fill the chip twice (d = 128; at d = 64, with
  // two long workgroups per CU, as often). Long against short, a block per workgroup, one box: d = 128 32/8 heads 512 x 512
  // 22.3 : 17.1 us, 2048 x 2048 (256 long blocks) 56.6 : 51.2, 4096 x 4096 (512) 133 : 143, 2048 x 8192 219 : 228; d = 64 16/16
  // 2048 x 2048 48.0 : 28.4, 4096 x 4096 87.1 : 55.8, 3 x 4096 x 4096 (768) 155 : 144.
  const int64_t fill = d_qk == 64 ? 1024 : 512;
  // With forms always: masks and changed scores are computed beside the matrix instructions of the other wave of a SIMD.
  m.is_short = !e4m3 && d_qk != 192 && (forms || (int64_t)max_q * group <= 128 || (rows / 256 + seqs) * hkv < fill);
  m.cols = m.is_short ? 128 : 256;
  m.n_wg = m.is_short || (d_qk == 64 && !e4m3) ? 512 : 256;
  // The most blocks that the packed tokens can make: whole ones, and a last one for each sequence of this kernel.
  m.blocks = rows / m.cols + seqs;
  // Never with long blocks where there are short ones: fill is n_wg at least. Every sequence that may have rows here counts as a
  // block, single tokens too, so a chunk is no longer split beside many of them: 32/8 heads, d = 128, 1 024 tokens over
  // 9 000 keys beside 24 over 2 000 194 us, beside 31 217; e4m3 beside 4 166, beside 15 236; 32/32 heads, d_qk = 192, 512 over
  // 4 500 beside 4 over 1 000 96, beside 5 146. The line of work is counted in 32 bits: where the table has pages for more
  // units than that (128 blocks over 2^30 keys each) no block is split.
  const int64_t units = kBlockCost + (static_cast<int64_t>(max_keys) + kSplitTile - 1) / kSplitTile;  // of a block, at most
  m.split = m.blocks * hkv < m.n_wg && m.blocks * hkv * units <= INT32_MAX;
  return m;
}

hipError_t launch_paged_many(const PagedParams& args, const PagedMany& m, int d_qk, bool e4m3, hipStream_t stream) {
  PagedParams p = args;
  many_constants(p);
  if (e4m3) {
    if (d_qk == 64) return launch_many_split<64, 64, true, false>(p, m, stream);
    if (d_qk == 128) return launch_many_split<128, 128, true, false>(p, m, stream);
    return launch_many_split<192, 128, true, false>(p, m, stream);
  }
  if (d_qk == 64)
    return m.is_short ? launch_many_split<64, 64, false, true>(p, m, stream)
                      : launch_many_split<64, 64, false, false>(p, m, stream);
  if (d_qk == 128)
    return m.is_short ? launch_many_split<128, 128, false, true>(p, m, stream)
                      : launch_many_split<128, 128, false, false>(p, m, stream);
  return launch_many_split<192, 128, false, false>(p, m, stream);
}

}  // namespace fa
