// Paged key/value cache for gfx950: appending new tokens with their position rotation, the launches of the
// attention of few new tokens per sequence (fa_paged_few.h), and the join of what either attention kernel splits.
//
// The cache holds keys and values in pages of `page_size` tokens; a block table names the pages of a
// sequence in order. What a sequence holds (kv_lens), which of the packed tokens are its new ones
// (q_starts) and its pages (block_table) are device arrays, so the host never sees them: every index
// that comes from them is checked or clamped here before it reaches an address.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <type_traits>

#include "fa_device.h"
#include "fa_e4m3.h"
#include "fa_fastdiv.h"
#include "fa_internal.h"
#include "fa_paged_device.h"
#include "fa_paged_few.h"
#include "fa_turn.h"

namespace fa {
namespace {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// ---- append ------------------------------------------------------------------------------------------
//
// One workgroup per packed token. A thread owns 16 bytes of a head, and with them the 16 bytes of their
// partners where dim c turns with dim c + rot / 2, so that a pair is read, turned in fp32 and written by one
// thread (Q may be rotated in place), and takes every so many-th head: the cos and sin of its dims stay in
// registers. What bounds it: the bytes of Q, K and V and the latency of the chain token -> sequence ->
// page -> load -> store. 12 290 tokens of 32/8 heads, d = 128, bf16: 53 us in the kernel, 5.8 TB/s read and written; 777 of 16/16
// heads, d_qk = 192: 8 us; one token: 3.4 us. By positions, 8 970 tokens of 32/8 heads with three axes 46 us (4.8 TB/s), 26
// tokens 5.

// Sequence of packed token t: the last b with q_starts[b] <= t, by 64 probes at a time (one step up to 63
// sequences, two up to 4 095). -1 if t comes before the first sequence; n_seq if behind the last.
__device__ __forceinline__ int sequence_of(const int* q_starts, int n_seq, int t, int lane) {
  int lo = 0, len = n_seq + 1;
  while (true) {
    const int step = (len + 63) / 64, at = lane * step;
    const bool below = at < len && q_starts[lo + at] <= t;
    const int n = __builtin_popcountll(__builtin_amdgcn_ballot_w64(below));
    if (n == 0) return lo - 1;
    lo += (n - 1) * step;
    if (step == 1) return lo;
    len = min(step, len - (n - 1) * step);
  }
}

// x / scale in e4m3, rounded to nearest even; what passes the largest finite value (448) becomes it, NaN
// stays NaN.
__device__ __forceinline__ u32x2 pack8_e4m3(const F8& f, float scale) {
  float y[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float x = f.x[i] / scale;
    y[i] = x > 448.f ? 448.f : x < -448.f ? -448.f : x;
  }
  int lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
  lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], lo, true);
  int hi = __builtin_amdgcn_cvt_pk_fp8_f32(y[4], y[5], 0, false);
  hi = __builtin_amdgcn_cvt_pk_fp8_f32(y[6], y[7], hi, true);
  return u32x2{(uint32_t)lo, (uint32_t)hi};
}

constexpr int kAppendThreads = 256;
// Tokens of a row of the grid: a dimension of it holds fewer than 2^32 threads, so 2^24 tokens and more need a second one.
constexpr int kAppendRowLog = 22;

// AT: the rows of the table go by p.pos, not by the keys' places.
template <bool FP8, bool AT>
__global__ __launch_bounds__(kAppendThreads) void fa_append_kernel(AppendParams p) {
  const int t = (int)(blockIdx.y << kAppendRowLog | blockIdx.x), tid = threadIdx.x, lane = tid & 63;  // below 2^31
  if (t >= p.bt.n_tokens) return;
  const int b = __builtin_amdgcn_readfirstlane(sequence_of(p.bt.q_starts, p.bt.n_seq, t, lane));
  if (b < 0 || b >= p.bt.n_seq) return;
  const PagedSeq s = load_seq(p.bt, b);
  const int64_t pos = (int64_t)s.kv - s.q_end + t;
  if (t >= s.q_end || pos < 0) return;
  // A token whose page number is none of the cache's leaves the cache alone; its query is rotated.
  const int page = scalar_load(p.bt.block_table + b * p.bt.table_stride + (pos >> p.c.page_shift));
  const bool held = page >= 0 && page < p.c.n_pages;
  const int64_t slot = pos & ((1 << p.c.page_shift) - 1);

  // Q and K: thread (h0, j) takes task j of every `lanes`-th head.
  const TurnTasks w(p.c.d_qk, p.rot, p.begin, p.inter);
  const int half = w.half, lanes = kAppendThreads / w.tasks;
  const int j = tid % w.tasks, h0 = tid / w.tasks;
  if (h0 < lanes) {
    const bool turn = j < w.turned;
    const int ch = w.chunk(j);
    const bool pair = turn && !p.inter;
    const int heads = p.hq + (held ? p.c.hkv : 0);
    // (Pointers and strides in registers of their own: of a choice between fields of p the compiler makes a load from the chosen
    // one's address, and then loads no argument before its use: one token 4.2 us against 3.4, 777 tokens 9.5 against 8.6.)
    const uint16_t* const q = p.q + t * p.q_token + 8 * ch;
    const uint16_t* const k = p.k + t * p.k_token + 8 * ch;
    const int64_t q_head = p.q_head, k_head = p.k_head;
    F8 cs{}, sn{};
    if (turn) {
      // Half-split: cos and sin of 8 pairs; neighbouring pairs: of the chunk's 4.
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        if (i > 0 && p.inter) break;
        const int four = p.inter ? j : 2 * j + i;
        if constexpr (AT)
          angles_at(cs, sn, i, p.pos, p.pos.positions + t * p.pos.token, p.cos_sin, p.rot, four);
        else
          angles_of_row(cs, sn, i, p.cos_sin + pos * p.rot, p.rot, four);
      }
    }
    for (int h = h0; h < heads; h += lanes) {
      const bool is_q = h < p.hq;
      const int g = h - p.hq;
      const uint16_t* src = is_q ? q + h * q_head : k + g * k_head;
      // Both words of a pair are loaded before either is used (threads that copy load theirs twice, from L1: a branch would wait
      // in between): 12 290 tokens 51.8 us against 53.2, 8 970 by three axes 45.7 against 50.7; loaded a head ahead 53.0 and 47.1.
      const u32x4 wx = *reinterpret_cast<const u32x4*>(src);
      u32x4 wy;
      if (!p.inter) wy = *reinterpret_cast<const u32x4*>(src + (pair ? 8 * half : 0));
      F8 x = unpack8(wx), y;
      if (pair) {
        y = unpack8(wy);
        turn_halves(x, y, cs, sn);
      } else if (turn) {
        turn_neighbours(x, cs, sn);
      }
      if (is_q) {
        uint16_t* dst = p.q_out + t * p.qo_token + h * p.qo_head + 8 * ch;
        *reinterpret_cast<u32x4*>(dst) = pack8(x);
        if (pair) *reinterpret_cast<u32x4*>(dst + 8 * half) = pack8(y);
      } else {
        const int64_t at = page * p.c.k_page + g * p.c.k_head + slot * p.c.k_slot + 8 * ch;
        if constexpr (FP8) {
          const float sc = p.c.k_scale != nullptr ? p.c.k_scale[g] : 1.f;
          uint8_t* dst = static_cast<uint8_t*>(p.c.k) + at;
          *reinterpret_cast<u32x2*>(dst) = pack8_e4m3(x, sc);
          if (pair) *reinterpret_cast<u32x2*>(dst + 8 * half) = pack8_e4m3(y, sc);
        } else {
          uint16_t* dst = static_cast<uint16_t*>(p.c.k) + at;
          *reinterpret_cast<u32x4*>(dst) = pack8(x);
          if (pair) *reinterpret_cast<u32x4*>(dst + 8 * half) = pack8(y);
        }
      }
    }
  }
  if (!held) return;
  const int vch = p.c.d_v / 8;
  for (int i = tid; i < p.c.hkv * vch; i += kAppendThreads) {
    const int g = i / vch, ch = i % vch;
    const u32x4 w = *reinterpret_cast<const u32x4*>(p.v + t * p.v_token + g * p.v_head + 8 * ch);
    const int64_t at = page * p.c.v_page + g * p.c.v_head + slot * p.c.v_slot + 8 * ch;
    if constexpr (FP8)
      *reinterpret_cast<u32x2*>(static_cast<uint8_t*>(p.c.v) + at) =
          pack8_e4m3(unpack8(w), p.c.v_scale != nullptr ? p.c.v_scale[g] : 1.f);
    else
      *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(p.c.v) + at) = w;
  }
}

// What a join reads: the items of one attention kernel, a workgroup (of the grid's first dimension) for each of its
// workgroups times cols (columns that an item is expected to have).
struct JoinSource {
  const PagedItem* desc;  // [n]
  const float* o_part;
  const float* lse_part;
  int part_cols, n, cols;
};

// Join of the parts of an item (none: n_parts 0): O = sum_k w_k O_k / sum_k w_k with w_k = exp(LSE_k - max
// LSE). DV / 4 threads (4 output dims each) by pg part groups take a column, group j
// the parts j, j + pg, ... with a running maximum, up to six at a time whose loads are in flight together (exactly as many
// as there are: their latency, and for blocks of the kernel for many rows their bytes, are the kernel's time); the groups'
// sums are added in their order through LDS. pg is the smallest power of two that leaves a group at most six parts, at most
// 1024 / DV; the workgroup's other groups take other columns. BOTH: one launch joins the items of both attention kernels (a second one would take 4 us more, this
// form costs 1 us where there is one): the first a.n * a.cols workgroups take those of `a`, the rest those of `b`. Else
// the grid is a.n by a.cols. Bound by latency: 4.4 us where few items are split, 14 for 64 blocks of 256 row-heads in four
// parts (34 MB of fp32, 2.4 TB/s).
template <int DV>
struct JoinLds {
  float m[1024 / DV], den[1024 / DV];
  f32x4 acc[1024 / DV][DV / 4];
};
// Place of the k-th part of an item whose first part is workgroup `first`'s.
__device__ __forceinline__ int64_t part_place(int first, int k) { return 2 * ((int64_t)first + k) + (k == 0 ? 1 : 0); }

template <int DV, bool BOTH>
__global__ __attribute__((amdgpu_flat_work_group_size(256, 256), amdgpu_waves_per_eu(8))) void fa_paged_join_kernel(PagedParams p, JoinSource a, JoinSource b) {
  __shared__ JoinLds<DV> lds;
  JoinSource src = a;
  int item = (int)blockIdx.x, share = (int)blockIdx.y;
  if constexpr (BOTH) {
    const int n_a = a.n * a.cols;
    if (item >= n_a) src = b, item -= n_a;
    share = (int)((uint32_t)item / (uint32_t)src.n);
    item -= share * src.n;
  }
  const PagedItem it = src.desc[item];
  if (it.n_parts <= 1) return;
  const int first = it.first, part_cols = src.part_cols;
  const float* const o_part = src.o_part;
  const float* const lse_part = src.lse_part;
  int pg = 1;
  while (6 * pg < it.n_parts && pg < 1024 / DV) pg *= 2;
  constexpr int TD = DV / 4, NG = 256 / TD;  // threads per column, groups
  const int q = threadIdx.x % TD, grp = threadIdx.x / TD;
  const int j = grp & (pg - 1), at_once = NG / pg;
  for (int c0 = share * at_once; c0 < it.n_cols; c0 += src.cols * at_once) {
    const int col = c0 + grp / pg;
    const bool live = col < it.n_cols;
    float m = -INFINITY, den = 0.f;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    // N parts of each group, base + j + pg * i (the last group's last may lie behind the item's last part).
    auto batch = [&](auto n, int base) {
      constexpr int N = decltype(n)::value;
      float l[N], top = m;
      f32x4 v[N];
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int64_t at = part_place(first, min(base + j + pg * i, it.n_parts - 1)) * part_cols + (live ? col : 0);
        l[i] = lse_part[at];
        v[i] = *reinterpret_cast<const f32x4*>(o_part + at * DV + 4 * q);
      }
#pragma unroll
      for (int i = 0; i < N; ++i) {
        l[i] = base + j + pg * i < it.n_parts ? l[i] : -INFINITY;
        top = fmaxf(top, l[i]);
      }
      const float ref = top == -INFINITY ? 0.f : top, a = expf(m - ref);
      den *= a;
      acc *= a;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const float w = expf(l[i] - ref);
        den += w;
        acc += w * v[i];
      }
      m = top;
    };
    for (int base = 0; base < it.n_parts; base += 6 * pg) {
      switch ((it.n_parts - base + pg - 1) / pg) {  // for the whole workgroup the same
        case 1: batch(std::integral_constant<int, 1>{}, base); break;
        case 2: batch(std::integral_constant<int, 2>{}, base); break;
        case 3: batch(std::integral_constant<int, 3>{}, base); break;
        case 4: batch(std::integral_constant<int, 4>{}, base); break;
        case 5: batch(std::integral_constant<int, 5>{}, base); break;
        default: batch(std::integral_constant<int, 6>{}, base);
      }
    }
    if (pg > 1) {
      __syncthreads();  // the last columns' sums have been read
      lds.acc[grp][q] = acc;
      if (q == 0) lds.m[grp] = m, lds.den[grp] = den;
      __syncthreads();
    }
    if (live && j == 0) {
      if (pg > 1) {
        for (int k = 1; k < pg; ++k) m = fmaxf(m, lds.m[grp + k]);
        const float ref = m == -INFINITY ? 0.f : m;
        den = 0.f, acc = f32x4{0.f, 0.f, 0.f, 0.f};
        for (int k = 0; k < pg; ++k) {
          const float w = expf(lds.m[grp + k] - ref);
          den += w * lds.den[grp + k];
          acc += w * lds.acc[grp + k][q];
        }
      }
      const bool some = den > 0.f;  // else no part with a visible key, or one whose sum is no number
      acc = some ? acc * (1.f / den) : f32x4{0.f, 0.f, 0.f, 0.f};
      const int c = it.c0 + col, row = c / p.group, head = it.g * p.group + c - row * p.group;
      const int64_t tok = it.q0 + row;
      *reinterpret_cast<u32x2*>(p.o + tok * p.o_token + (int64_t)head * p.o_head + 4 * q) =
          u32x2{pack_bf16x2(acc.x, acc.y), pack_bf16x2(acc.z, acc.w)};
      if (q == 0 && p.lse != nullptr) p.lse[tok * p.hq + head] = some ? m + logf(den) : -INFINITY;
    }
  }
}

}  // namespace

hipError_t launch_append(AppendParams p, bool fp8, hipStream_t stream) {
  void* args[] = {&p};
  constexpr unsigned kRow = 1u << kAppendRowLog;
  const unsigned n = (unsigned)p.bt.n_tokens;
  const dim3 grid(n < kRow ? n : kRow, (n + kRow - 1) / kRow);
  const bool at = p.pos.positions != nullptr && p.rot > 0;
  const void* k = fp8 ? (at ? reinterpret_cast<const void*>(&fa_append_kernel<true, true>)
                            : reinterpret_cast<const void*>(&fa_append_kernel<true, false>))
                      : (at ? reinterpret_cast<const void*>(&fa_append_kernel<false, true>)
                            : reinterpret_cast<const void*>(&fa_append_kernel<false, false>));
  return hipLaunchKernel(k, grid, dim3(kAppendThreads), args, 0, stream);
}

int paged_workgroups(int d_qk, bool fp8, int col_blocks) {
  if (d_qk == 64) return 512;
  return fp8 && col_blocks == 1 ? 512 : 256;
}
static_assert(FewInstance<64, 64, false, 2, true>::kWorkgroups == 512 && FewInstance<64, 64, true, 2, true>::kWorkgroups == 512 &&
                  FewInstance<64, 64, false, 1, true>::kWorkgroups == 512 && FewInstance<64, 64, true, 1, true>::kWorkgroups == 512 &&
                  FewInstance<128, 128, true, 1, true>::kWorkgroups == 512 && FewInstance<192, 128, true, 1, true>::kWorkgroups == 512 &&
                  FewInstance<128, 128, false, 1, true>::kWorkgroups == 256 && FewInstance<128, 128, true, 2, true>::kWorkgroups == 256,
              "paged_workgroups");

template <int QB, bool STREAM>
hipError_t launch_few_dims(PagedParams p, int d_qk, bool fp8, hipStream_t stream) {
  if (d_qk == 64)
    return fp8 ? launch_few<typename FewInstance<64, 64, true, QB, STREAM>::C>(p, stream)
               : launch_few<typename FewInstance<64, 64, false, QB, STREAM>::C>(p, stream);
  if (d_qk == 128)
    return fp8 ? launch_few<typename FewInstance<128, 128, true, QB, STREAM>::C>(p, stream)
               : launch_few<typename FewInstance<128, 128, false, QB, STREAM>::C>(p, stream);
  return fp8 ? launch_few<typename FewInstance<192, 128, true, QB, STREAM>::C>(p, stream)
             : launch_few<typename FewInstance<192, 128, false, QB, STREAM>::C>(p, stream);
}

hipError_t launch_paged_few(PagedParams p, int d_qk, bool fp8, int col_blocks, bool stream_kv, hipStream_t stream) {
  few_constants(p);
  if (col_blocks == 1) return launch_few_dims<1, true>(p, d_qk, fp8, stream);
  return stream_kv ? launch_few_dims<2, true>(p, d_qk, fp8, stream) : launch_few_dims<2, false>(p, d_qk, fp8, stream);
}

hipError_t launch_paged_join(PagedParams p, int d_v, int few_cols, int many_cols, hipStream_t stream) {
  auto clamped = [](int cols) { return cols < 1 ? 1 : cols > 32 ? 32 : cols; };
  many_cols = many_cols * d_v / 1024;  // blocks have few parts each, so a workgroup takes 1024 / d_v columns at once
  JoinSource few{p.desc, p.o_part, p.lse_part, p.part_cols, p.n_wg, clamped(few_cols)};
  JoinSource many{p.many_desc, p.many_o, p.many_lse, many_place_cols(p.many_cols), p.many_wg, clamped(many_cols)};
  const bool both = few_cols > 0 && many_cols > 0;
  JoinSource* first = few_cols > 0 ? &few : &many;
  void* args[] = {&p, first, &many};
  const dim3 grid = both ? dim3((unsigned)(few.n * few.cols + many.n * many.cols)) : dim3(first->n, first->cols);
  const void* k = both ? (d_v == 64 ? reinterpret_cast<const void*>(&fa_paged_join_kernel<64, true>)
                                    : reinterpret_cast<const void*>(&fa_paged_join_kernel<128, true>))
                       : (d_v == 64 ? reinterpret_cast<const void*>(&fa_paged_join_kernel<64, false>)
                                    : reinterpret_cast<const void*>(&fa_paged_join_kernel<128, false>));
  return hipLaunchKernel(k, grid, dim3(256), args, 0, stream);
}

}  // namespace fa
