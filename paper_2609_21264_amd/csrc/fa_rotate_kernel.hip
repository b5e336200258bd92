// Position rotation of queries or keys [B, H, S, d] that are in no cache (gfx950), and the way back, which is also the
// rotation's gradient: a turn by the negative angle.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "fa_fastdiv.h"
#include "fa_turn.h"

namespace fa {
namespace {

// A workgroup takes 256 / tasks tokens of one batch (tasks: the threads of a head's row, fa_turn.h) and some of the heads, a
// thread the same chunk of every head, so that the angles stay in registers and a pair is read, turned and
// written by one thread (Y may be X). What bounds it: the bytes of X and Y.
constexpr int kRotateThreads = 256;
// Heads of a workgroup, fewer where that leaves too few workgroups: 2 x 9 999 tokens of 16 heads, d = 64, three axes, there and
// back 34.6 us with 8 (4.7 TB/s read and written; 36.2 on a slower box), 39.3 with all 16, 35.5 with 4, 38.3 with 2, 49.0 with one.
constexpr int kRotateHeads = 8, kRotateWorkgroups = 512;

template <bool AT>
__global__ __launch_bounds__(kRotateThreads) void fa_rotate_kernel(RotateParams p) {
  const TurnTasks w(p.d, p.rot, p.begin, p.inter);
  const int lanes = kRotateThreads / w.tasks;
  const int j = threadIdx.x % w.tasks, row = threadIdx.x / w.tasks;
  if (row >= lanes) return;
  const bool turn = j < w.turned, pair = turn && !p.inter;
  if (!turn && p.in_place) return;
  const int ch = w.chunk(j);
  const int h0 = (int)blockIdx.y * p.heads, h1 = min(h0 + p.heads, p.h);
  // Unsigned: a step past the last block may lead behind 2^31.
  for (uint32_t blk = blockIdx.x; blk < (uint32_t)p.n_blocks; blk += gridDim.x) {
    const int b = (int)fast_div(blk, p.m_per, p.sh_per);
    const int64_t s = (int64_t)((int)blk - b * p.per) * lanes + row;
    if (s >= p.s) continue;
    F8 cs{}, sn{};
    if (turn) {
      const int* pos = AT ? p.pos.positions + b * p.pos.batch + s * p.pos.token : nullptr;
      const float* table = p.cos_sin;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        if (i > 0 && p.inter) break;
        const int four = p.inter ? j : 2 * j + i;
        if constexpr (AT)
          angles_at(cs, sn, i, p.pos, pos, table, p.rot, four);
        else
          angles_of_row(cs, sn, i, table + s * p.rot, p.rot, four);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) sn.x[e] *= p.sign;
    }
    const uint16_t* src = p.x + b * p.x_b + s * p.x_s + 8 * ch;
    uint16_t* dst = p.y + b * p.y_b + s * p.y_s + 8 * ch;
    for (int h = h0; h < h1; ++h) {
      F8 x = unpack8(*reinterpret_cast<const u32x4*>(src + h * p.x_h));
      if (pair) {
        F8 y = unpack8(*reinterpret_cast<const u32x4*>(src + h * p.x_h + 8 * w.half));
        turn_halves(x, y, cs, sn);
        *reinterpret_cast<u32x4*>(dst + h * p.y_h + 8 * w.half) = pack8(y);
      } else if (turn) {
        turn_neighbours(x, cs, sn);
      }
      *reinterpret_cast<u32x4*>(dst + h * p.y_h) = pack8(x);
    }
  }
}

}  // namespace

hipError_t launch_rotate(RotateParams p, hipStream_t stream) {
  const int half = p.inter ? 0 : p.rot / 16, lanes = kRotateThreads / (p.d / 8 - half);
  p.per = (int)(((int64_t)p.s + lanes - 1) / lanes);
  p.n_blocks = p.batch * p.per;  // below 2^31: batch * s is
  const FastDiv f = make_fastdiv((uint32_t)p.per);
  p.m_per = f.m, p.sh_per = f.sh;
  p.heads = p.h < kRotateHeads ? p.h : kRotateHeads;
  while (p.heads > 1 && (int64_t)p.n_blocks * ((p.h + p.heads - 1) / p.heads) < kRotateWorkgroups) p.heads = (p.heads + 1) / 2;
  if ((p.h - 1) / p.heads >= 65535) p.heads = (p.h - 1) / 65535 + 1;  // as many workgroups as the grid's second dimension holds
  constexpr int kMost = 1 << 20;
  const dim3 grid((unsigned)(p.n_blocks < kMost ? p.n_blocks : kMost), (unsigned)((p.h + p.heads - 1) / p.heads));
  void* args[] = {&p};
  return hipLaunchKernel(p.pos.positions != nullptr ? reinterpret_cast<const void*>(&fa_rotate_kernel<true>)
                                                    : reinterpret_cast<const void*>(&fa_rotate_kernel<false>),
                         grid, dim3(kRotateThreads), args, 0, stream);
}

}  // namespace fa
