// Attention of many new tokens per sequence over a paged key/value cache (gfx950): prompts and chunks of them.
// The pipelined step of the fused forward (fa_fwd_attn.h) with another source of keys and another arrangement of
// rows and work:
//  * A block is 256 consecutive row-heads (128 in the short instances) of one (sequence, key/value head): column c of the block's item is
//    token c / group of the sequence's new ones and query head c % group of the group, so all heads of a group share
//    every K/V tile whatever the group's size, and a short chunk pads at most once. Each lane keeps the
//    last key its columns see; the mask is the same with and without causal masking.
//  * A wave brings BN / 4 (16 or 8) consecutive keys of a tile, which lie in one page (pages have 16 slots at
//    least): the page's number makes the buffer descriptor, one per wave and tile. A register holds the page numbers
//    of the wave's next 64 tiles, one per lane; a step reads its own with a lane read, so no step waits for the table.
//  * Pages that are not there are rare: each item looks for one first, and only then masks every tile by pages.
//  * Where there are blocks enough, a workgroup takes one block, a sequence's last (longest) blocks first.
//    Otherwise (SPLIT) the lengths decide: where the longest block is much longer than an even share of the work (a chunk of
//    a prompt against a long cache), the blocks lie on one line of work, kBlockCost + tiles units each, that the
//    workgroups share evenly, and parts of a block that several share are joined as those of the kernel for few
//    rows are; else a workgroup takes one block here too.
// What bounds it: MFMA and the softmax between them, as in the fused forward. 32/8 heads, d = 128, prompts of 4 096 and 3 001
// tokens 200-215 us by box (985-1 055 TFLOP/s; over an e4m3 cache 218, 969), a chunk of 1 024 over 9 000 keys, split, 140 (1 000) and its
// part of the join; 32/32 heads, d_qk = 192, 512 tokens over 4 500 keys, split, 64 (700) and 13 for the join. Over contiguous keys the fused forward takes 1/1.03 to 1/1.06 of its time from 8 192 tokens
// on, 1/1.10 at 2 048 (d = 128), 1/1.26 at 4 096 of 16/16 heads with d = 64.
#include <float.h>
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "fa_device.h"
#include "fa_fwd_attn.h"
#include "fa_internal.h"
#include "fa_paged_device.h"

namespace fa {
namespace {

constexpr int kBlockCost = 4;  // fixed cost of a block in tiles
constexpr int kSplitTile = 64;  // keys of a tile where blocks are split
// Splitting costs a second block's start, writing and reading the parts and the join, 20-40 us in all, so it pays where the
// longest block has 32 units more than an even share, and 1.9 times as many. Measured, a block per workgroup against
// split, 128-row-head blocks, one box: d = 128 32/8 heads 1024 x 1024 26 us against 42, 256 x 4096 (8 times the share) 73 : 42,
// 512 x 4096 (4 times) 74 : 56, 3 x 512 x 4096 (1.4) 112 : 123, 1024 x 8192 (2.0) 148 : 145; d = 64 16/16 2048 x 2048 (26 units
// more) 28 : 36, 256 x 4096 47 : 28, 3 x 1024 x 8192 (1.3) 145 : 135; blocks of 256, d = 128: 2048 x 2048 57 : 79, 1024 x 8192
// (2.0) 176 : 137, 3 x 512 x 4096 101 : 119.
constexpr int kSplitUnits = 32;

// This wave's share of the loads of one K or V tile: BN / NWAVES rows of CH 16-byte chunks, all in one page; E bytes per
// element.
template <int NWAVES, int BN, int CH, int E>
struct PagedLoader {
  static constexpr int R = BN / NWAVES, NI = BN * CH / 64 / NWAVES;
  static_assert(R * CH == NI * 64 && R <= 16 && 16 % R == 0, "a wave's rows are whole loads inside one page");
  uint64_t base;        // head, in page 0
  int64_t page_bytes;
  uint32_t slot_bytes;
  uint32_t voff[NI];    // bytes from the wave's first row
  template <class Swz>
  __device__ __forceinline__ void init(const unsigned char* head, int64_t page_stride, int64_t slot_stride, int wave, int lane,
                                       Swz swz) {
    base = reinterpret_cast<uint64_t>(head);
    page_bytes = page_stride * E;
    slot_bytes = (uint32_t)(slot_stride * E);
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int x = i * 64 + lane, row = x / CH;
      voff[i] = (uint32_t)row * slot_bytes + (uint32_t)((x % CH) ^ swz(wave * R + row)) * 16u;
    }
  }
  // Buffer of the rows from key `key` on that lie before `lim`, in page `page`: none if that is none of the cache's.
  __device__ __forceinline__ u32x4 rsrc(int page, int n_pages, int key, int smask, int lim) const {
    const bool ok = page >= 0 && page < n_pages;
    const uint64_t a = base + (uint64_t)((int64_t)(ok ? page : 0) * page_bytes + (int64_t)(key & smask) * slot_bytes);
    const int rows = ok ? max(0, min(R, lim - key)) : 0;
    return u32x4{(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)a),
                 (uint32_t)__builtin_amdgcn_readfirstlane((int)((uint32_t)(a >> 32) & 0xffffu)),
                 (uint32_t)__builtin_amdgcn_readfirstlane(rows * (int)slot_bytes), 0x00020000u};
  }
  __device__ __forceinline__ void issue_one(const u32x4& r, uint32_t l, int i) const {
    dma16_buffer(r, voff[i], l + i * 1024);
  }
  __device__ __forceinline__ void issue(const u32x4& r, uint32_t l) const {
#pragma unroll
    for (int i = 0; i < NI; ++i) issue_one(r, l, i);
  }
};

// A block's place: which keys its columns see.
template <int BN, int BC>
struct Block {
  int cols, c0, row0, row1;  // row-heads of the item, the block's first, its first and last row
  int kv_end, plain;         // keys visible to its last row; leading tiles that need no mask for any row
  __device__ __forceinline__ Block(const PagedSeq& s, int cb, const PagedParams& p) {
    cols = s.n_q * p.group;
    c0 = cb * BC;
    row0 = (int)fast_div((uint32_t)c0, p.m_group, p.sh_group);
    row1 = (int)fast_div((uint32_t)min(c0 + BC, cols) - 1u, p.m_group, p.sh_group);
    kv_end = p.causal ? max(0, s.kv - s.n_q + row1 + 1) : s.kv;
    plain = (p.causal ? max(0, s.kv - s.n_q + row0 + 1) : s.kv) / BN;
  }
  __device__ __forceinline__ int tiles() const { return (kv_end + BN - 1) / BN; }
};
template <int BC>
__device__ __forceinline__ int n_blocks(const PagedSeq& s, const PagedParams& p) {
  const int64_t cols = (int64_t)s.n_q * p.group;
  return cols > p.few_cols ? (int)((cols + BC - 1) / BC) : 0;
}
template <int BN, int BC>
__device__ __forceinline__ int head_units(const PagedSeq& s, int n_cb, const PagedParams& p, int lane) {
  uint32_t sum = 0;
  for (int c = lane; c < n_cb; c += 64) sum += (uint32_t)(kBlockCost + Block<BN, BC>(s, c, p).tiles());
  return (int)wave_sum(sum);
}
template <class C>
__global__ __attribute__((amdgpu_flat_work_group_size(C::NT, C::NT), amdgpu_waves_per_eu(C::WPE, C::WPE)))
void fa_paged_fwd_kernel(PagedParams p) {
  using A = Attn<C>;
  constexpr int DQK = C::DQK, DV = C::DV, BN = C::BN, QB = C::QB;
  constexpr int BC = C::NWAVES * 32 * QB;  // row-heads per block
  constexpr int R = BN / C::NWAVES;        // keys that a wave brings of a tile
  constexpr int E = C::E;
  static_assert(C::KSPLIT == 1 && C::KA - C::VA <= 1, "a V tile is loaded with its K tile or one step later");
  static_assert(!C::SPLIT || BN == kSplitTile, "the host counts the line's units");

  __shared__ __attribute__((aligned(1024))) unsigned char smem[C::LDS_BYTES];
  const int tid = threadIdx.x;
  int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  A st;
  st.qw = st.diag = 0;
  st.page_stride = p.c.k_page;
  st.slot_stride = p.c.k_slot;
  st.page_shift = p.c.page_shift;
  st.n_pages = p.c.n_pages;
  const int smask = (1 << p.c.page_shift) - 1;

  // ---- this workgroup's work ----
  int b = 0, g = 0, cb = 0, n_cb = 0;
  int me = 0, start = 0, r = 0, r1 = 0, per = 1, total = 0;  // split: place on the line, the block's first unit, units [r, r1)
  bool split = false;
  PagedSeq s{};
  if constexpr (C::SPLIT) {
    if (tid == 0) p.many_desc[blockIdx.x].n_parts = 0;
  }
  // The first 64 sequences stay in registers, one per lane; those behind them are read again for each use.
  PagedSeq first{};
  if (lane < p.bt.n_seq) first = load_seq_lane(p.bt, lane);
  auto seqs_from = [&](int c) {
    PagedSeq x{};
    if (c == 0)
      x = first;
    else if (c + lane < p.bt.n_seq)
      x = load_seq_lane(p.bt, c + lane);
    return x;
  };
  if (p.few_cols != 0 && big_work(p, first, lane) < p.many_work) return;  // all sequences run in the kernel for few rows
  if constexpr (C::SPLIT) {
    uint32_t sum = 0;
    int longest = 0;
    for (int c = 0; c < p.bt.n_seq; c += 64) {
      const PagedSeq sl = seqs_from(c);
      uint64_t left = __builtin_amdgcn_ballot_w64(n_blocks<BC>(sl, p) > 0);
      while (left != 0) {
        const PagedSeq x = seq_of_lane(sl, __builtin_ctzll(left));
        left &= left - 1;
        const int n = n_blocks<BC>(x, p);
        sum = add_sat(sum, (uint32_t)min((int64_t)head_units<BN, BC>(x, n, p, lane) * p.c.hkv, (int64_t)UINT32_MAX));
        longest = max(longest, kBlockCost + Block<BN, BC>(x, n - 1, p).tiles());
      }
    }
    total = uniform((int)min(sum, (uint32_t)INT32_MAX));
    longest = uniform(longest);
    per = max(p.many_min_units, (int)((uint32_t)(total - 1) >> p.many_log) + 1);
    split = longest - per > kSplitUnits && 10ll * longest >= 19ll * per;  // else there are workgroups for all blocks (paged_many)
    if (split) {
      // Consecutive workgroups run on different XCDs, so the line is dealt to the XCDs in eighths: what shares a
      // key/value head mostly shares an L2.
      const int active = (int)((uint32_t)(total + per - 1) / (uint32_t)per), eighth = (active + kNumXcd - 1) / kNumXcd;
      const int slot = (int)(blockIdx.x / kNumXcd);
      me = uniform((int)(blockIdx.x % kNumXcd) * eighth + slot);
      if (slot >= eighth || (int64_t)me * per >= total) return;
      r = me * per;
      r1 = min(total - r, per) + r;
    }
  }
  if (C::SPLIT && split) {
    // The sequence, head and block that hold unit r.
    bool found = false;
    for (int c = 0; c < p.bt.n_seq && !found; c += 64) {
      const PagedSeq sl = seqs_from(c);
      uint64_t left = __builtin_amdgcn_ballot_w64(n_blocks<BC>(sl, p) > 0);
      while (left != 0 && !found) {
        const int l = __builtin_ctzll(left);
        left &= left - 1;
        s = seq_of_lane(sl, l);
        n_cb = n_blocks<BC>(s, p);
        const int units = head_units<BN, BC>(s, n_cb, p, lane);
        if ((int64_t)r < start + (int64_t)units * p.c.hkv) {
          b = c + l;
          g = uniform((int)((uint32_t)(r - start) / (uint32_t)units));
          start += g * units;
          found = true;
        } else {
          start += units * p.c.hkv;
        }
      }
    }
    if (!found) return;  // not reached: r < total
    for (int c = 0; c < n_cb; c += 64) {
      const uint32_t u = c + lane < n_cb ? (uint32_t)(kBlockCost + Block<BN, BC>(s, c + lane, p).tiles()) : 0u;
      const uint32_t incl = wave_scan(u);
      const uint64_t above = __builtin_amdgcn_ballot_w64(incl > (uint32_t)(r - start));
      if (above != 0) {
        const int l = __builtin_ctzll(above);
        cb = c + l;
        start += (int)lane_of(incl - u, l);
        break;
      }
      start += (int)lane_of(incl, 63);
    }
  } else {
    g = (int)(blockIdx.x % (uint32_t)p.c.hkv);
    int idx = (int)(blockIdx.x / (uint32_t)p.c.hkv);
    bool found = false;
    for (int c = 0; c < p.bt.n_seq && !found; c += 64) {
      const PagedSeq sl = seqs_from(c);
      const uint32_t n = (uint32_t)n_blocks<BC>(sl, p), incl = wave_scan(n);
      const uint64_t above = __builtin_amdgcn_ballot_w64(incl > (uint32_t)idx);
      if (above != 0) {
        const int l = __builtin_ctzll(above);
        b = c + l;
        s = seq_of_lane(sl, l);
        n_cb = (int)lane_of(n, l);
        cb = (int)lane_of(incl, l) - 1 - idx;  // the last block, with the most keys, first
        found = true;
      } else {
        idx -= (int)lane_of(incl, 63);
      }
    }
    if (!found) return;  // the grid is sized for the most blocks there can be
  }

  while (true) {
    const Block<BN, BC> blk(s, cb, p);
    const int tiles = blk.tiles();
    int t0 = 0, nt = tiles, n_parts = 1, first_wg = me;
    bool skip = false;
    if (C::SPLIT && split) {
      const int cost = kBlockCost + tiles, end = min(r1 - start, cost) + start;
      t0 = max(0, r - start - kBlockCost);
      nt = max(0, end - start - kBlockCost - t0);
      // The block belongs to the workgroups that have tiles of it (one without a tile: to that of its first unit).
      skip = tiles == 0 ? start < r : nt == 0;
      if (tiles != 0) {
        first_wg = uniform((int)((uint32_t)(start + kBlockCost) / (uint32_t)per));
        // (The line ends inside a block only if q_starts decreases and so many sequences share tokens that it was cut.)
        n_parts = uniform((int)((min((uint32_t)start + (uint32_t)cost, (uint32_t)total) - 1u) / (uint32_t)per)) - first_wg + 1;
      }
      r = end;
    }
    if (!skip) {
      // What follows from the lane is computed for each block anew (and again for its output): kept over the loop,
      // the addresses would not fit in the registers beside the step.
      if constexpr (C::SPLIT) asm volatile("" : "+v"(lane));
      st.i32 = lane & 31;
      st.h = lane >> 5;
      st.v_key = 8 * (lane >> 5) + ((lane & 15) >> (C::E4M3 ? 1 : 2));
      st.v_t = C::E4M3 ? (((lane >> 4) & 1) ^ v8_swizzle<C::VCH>(st.v_key))
                       : ((2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ v_swizzle<DV>(st.v_key));
      st.v_half = (lane & 1) * 8;
      const int kb0 = t0 * BN, t1 = t0 + nt;
      const int kv_lim = min(blk.kv_end, t1 * BN);  // keys loaded; behind it the tile loads read zeros
      st.sk = s.kv;
      st.table = p.bt.block_table + (int64_t)b * p.bt.table_stride;
      st.cs = p.cs;
      if constexpr (C::E4M3) {
        if (p.c.k_scale != nullptr) {  // a masked score has to stay infinite
          const float c = p.cs * scalar_load(p.c.k_scale + g);
          st.cs = fabsf(c) < FLT_MIN ? copysignf(FLT_MIN, c) : c;
        }
      }
      st.mask_val = st.cs < 0.f ? INFINITY : -INFINITY;

      // Q of this wave's columns, straight into registers; columns behind the last repeat it and are not stored.
#pragma unroll
      for (int qb = 0; qb < QB; ++qb) {
        const uint32_t c = (uint32_t)min(blk.c0 + wave * 32 * QB + qb * 32 + st.i32, blk.cols - 1);
        const int qi = (int)fast_div(c, p.m_group, p.sh_group), member = (int)c - qi * p.group;
        st.last_key[qb] = p.causal ? s.kv - s.n_q + qi : s.kv - 1;
        const uint16_t* qp = p.q + (int64_t)(s.q0 + qi) * p.q_token + (int64_t)(g * p.group + member) * p.q_head;
#pragma unroll
        for (int ks = 0; ks < A::KS; ++ks)
          load_q<A::AG>(st.qf[qb][ks], qp + (C::E4M3 ? 32 * (ks / 2) + 16 * st.h + 8 * (ks & 1) : 16 * ks + 8 * st.h));
      }

      // The pages of this wave's keys of tiles w0 .. w0 + 63, one per lane (behind the last key: the last one's).
      int entries = 0;
      auto window = [&](int w0) {
        const int key = min((w0 + lane) * BN + wave * R, kv_lim - 1);
        entries = key >= 0 ? st.table[key >> p.c.page_shift] : -1;
        asm volatile("" : "+v"(entries));  // waited for here, not at every use
      };
      // Whether a page of the range is not there. (The first 64 are read beside the window, so that both are waited for
      // once.)
      const int e0 = (kb0 >> p.c.page_shift) + lane, e1 = (kv_lim + smask) >> p.c.page_shift;
      int page0 = 0;
      if (e0 < e1) page0 = st.table[e0];
      window(t0);
      bool hole = e0 < e1 && (page0 < 0 || page0 >= p.c.n_pages);
      for (int e = e0 + 64; e < e1; e += 64) {
        const int page = st.table[e];
        hole = hole || page < 0 || page >= p.c.n_pages;
      }
      st.holes = __builtin_amdgcn_ballot_w64(hole) != 0;
      int n_plain = st.holes ? 0 : min(max(blk.plain - t0, 0), nt);

      const unsigned char* kh = static_cast<const unsigned char*>(p.c.k) + (int64_t)g * p.c.k_head * E;
      const unsigned char* vh = static_cast<const unsigned char*>(p.c.v) + (int64_t)g * p.c.v_head * E;
      st.kg = reinterpret_cast<const uint16_t*>(kh);
      PagedLoader<C::NWAVES, BN, C::KCH, E> kload;
      PagedLoader<C::NWAVES, BN, C::VCH, E> vload;
      kload.init(kh, p.c.k_page, p.c.k_slot, wave, lane,
                 [](int row) { return C::E4M3 ? k8_swizzle<C::KCH>(row & 15) : k_swizzle<DQK>(row); });
      vload.init(vh, p.c.v_page, p.c.v_slot, wave, lane,
                 [](int row) { return C::E4M3 ? v8_swizzle<C::VCH>(row & 15) : v_swizzle<DV>(row); });
      unsigned char* const vring = smem + C::NKR * C::K_BYTES;
      auto kslot = [&](int t) { return smem + ((unsigned)t % C::NKR) * C::K_BYTES; };
      auto vslot = [&](int t) { return vring + ((unsigned)t % C::NVR) * C::V_BYTES; };
      auto lds_of = [&](const unsigned char* slot, int ni) {
        return (uint32_t)__builtin_amdgcn_readfirstlane((int)(lds_offset(slot) + wave * ni * 1024));
      };
      // Descriptors of the K and V tile to be loaded next. A V tile is loaded with its K tile or a step later, with the
      // page found for that.
      u32x4 gk, gv;
      uint32_t gkl = 0, gvl = 0;
      int v_page = 0;
      auto aim_k = [&](int j) {
        const int page = __builtin_amdgcn_readlane(entries, j & 63);
        gk = kload.rsrc(page, p.c.n_pages, kb0 + j * BN + wave * R, smask, kv_lim);
        return page;
      };
      auto aim_v = [&](int j, int page) { gv = vload.rsrc(page, p.c.n_pages, kb0 + j * BN + wave * R, smask, kv_lim); };
      // The prologue's groups j = -KA .. -1, as in the fused forward: K(j + KA) and V(j + VA), and in front of group 1 - KA
      // zeros in the slot of the V tile before the first, which step 0 multiplies by P = 0.
#pragma unroll
      for (int j = -C::KA; j < 0; ++j) {
        if (j == 1 - C::KA) vload.issue(u32x4{0u, 0u, 0u, 0x00020000u}, lds_of(vslot(C::NVR - 1), C::V_LOADS));
        const int page = aim_k(j + C::KA);
        kload.issue(gk, lds_of(kslot(j + C::KA), C::K_LOADS));
        if (j + C::VA >= 0) {
          aim_v(j + C::VA, C::VA == C::KA ? page : v_page);
          vload.issue(gv, lds_of(vslot(j + C::VA), C::V_LOADS));
        }
        v_page = page;
      }
      // Q and K0: behind K0 are V0 when VA = KA, the zeros and the groups after.
      wait_vmcnt<C::V_LOADS + (C::VA == C::KA ? C::V_LOADS : 0) + (C::KA - 1) * (C::K_LOADS + C::V_LOADS)>();
#pragma unroll
      for (int qb = 0; qb < QB; ++qb)
#pragma unroll
        for (int ks = 0; ks < A::KS; ++ks) q_ready<A::AG>(st.qf[qb][ks]);
#pragma unroll
      for (int qb = 0; qb < QB; ++qb) {
        st.m_run[qb] = -INFINITY;
        st.l_run[qb] = 0.f;
#pragma unroll
        for (int db = 0; db < A::DB; ++db) {
          st.oacc[db][qb] = f32x16{};
          agpr_fence<A::AG>(st.oacc[db][qb]);
        }
      }

      typename A::Scores sA, sB;
      typename A::Probs pA, pB;
      if (nt > 0) {
        compiler_fence();
        __builtin_amdgcn_s_barrier();
        compiler_fence();
        st.scores(sA, kslot(0));
        if (n_plain == 0) st.mask_tile(sA, kb0);
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) st.m_run[qb] = st.row_max(sA, qb);
#pragma unroll
        for (int kb = 0; kb < A::KB; ++kb)
#pragma unroll
          for (int qb = 0; qb < QB; ++qb)
#pragma unroll
            for (int e = 0; e < 8; ++e) pB[kb][qb][e] = 0u;
      }
      // Before step j: K(j+1) and V(j-1) have landed; see the fused forward, also for the rings.
      Ring<C::K_BYTES, C::NKR> kring(0);
      Ring<C::V_BYTES, C::NVR> vpos(C::NVR - 2);
      auto kread = [&](int t) { return smem + kring.at(t); };
      auto vread = [&](int t) { return vring + vpos.at(t); };
      auto sync_step = [&](int j) {
        wait_vmcnt<C::V_LOADS + (C::KA - 2) * (C::K_LOADS + C::V_LOADS)>();
        compiler_fence();
        __builtin_amdgcn_s_barrier();
        compiler_fence();
        if (((j + C::KA) & 63) == 0) window(t0 + j + C::KA);
        const int page = aim_k(j + C::KA);
        aim_v(j + C::VA, C::VA == C::KA ? page : v_page);
        v_page = page;
        gkl = lds_of(smem + kring.at(j + C::KA), C::K_LOADS);
        gvl = lds_of(vring + vpos.at(j + C::VA), C::V_LOADS);
        kring.next();
        vpos.next();
      };
      auto issue = [&](int k) {
        if (k < C::K_LOADS)
          kload.issue_one(gk, gkl, k);
        else
          vload.issue_one(gv, gvl, k - C::K_LOADS);
      };
      unsigned char* const vzero = vslot(C::NVR - 1);
      int j = 0;
      for (; j + 1 < nt; j += 2) {
        sync_step(j);
        st.step(sA, sB, pA, pB, kread(j + 1), j > 0 ? vread(j - 1) : vzero, j >= n_plain, kb0 + j * BN, issue);
        sync_step(j + 1);
        st.step(sB, sA, pB, pA, kread(j + 2), vread(j), j + 1 >= n_plain, kb0 + (j + 1) * BN, issue);
      }
      if (j < nt) {
        sync_step(j);
        st.step(sA, sB, pA, pB, kread(j + 1), j > 0 ? vread(j - 1) : vzero, j >= n_plain, kb0 + j * BN, issue);
      }
      if (nt > 0) {
        // P V of the last tile, on a selected copy of P (see the fused forward).
        wait_vmcnt<C::VA * (C::K_LOADS + C::V_LOADS)>();
        compiler_fence();
        __builtin_amdgcn_s_barrier();
        compiler_fence();
        typename A::Probs pl;
        const uint32_t take_a = (nt & 1) ? 0xffffffffu : 0u;
#pragma unroll
        for (int kb = 0; kb < A::KB; ++kb)
#pragma unroll
          for (int qb = 0; qb < QB; ++qb)
#pragma unroll
            for (int e = 0; e < 8; ++e) pl[kb][qb][e] = (pA[kb][qb][e] & take_a) | (pB[kb][qb][e] & ~take_a);
        vpos.next();
        st.pv_tile(pl, vread(nt - 1));
      }
      // Every load has landed and every wave is done with the last V tile: the output is staged in the rings.
      wait_vmcnt<0>();
      compiler_fence();
      __builtin_amdgcn_s_barrier();
      compiler_fence();

#pragma unroll
      for (int qb = 0; qb < QB; ++qb)
#pragma unroll
        for (int db = 0; db < A::DB; ++db) agpr_fence<A::AG>(st.oacc[db][qb]);
      if constexpr (C::SPLIT) asm volatile("" : "+v"(lane));
      st.i32 = lane & 31;
      st.h = lane >> 5;
      constexpr int WROWS = 32 * QB, RB = DV * 2;
      const int col0 = wave * WROWS;  // this wave's first column of the block
      float vs = 1.f;
      if constexpr (C::E4M3) vs = p.c.v_scale != nullptr ? scalar_load(p.c.v_scale + g) : 1.f;
      if (C::SPLIT && n_parts > 1) {
        // A part: O normalised by its own sum (fp32), and its LSE. Place 2 me: of a block that begins before.
        const int64_t place = (2 * (int64_t)me + (me == first_wg ? 1 : 0)) * many_place_cols(BC);
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) {
          const float l_tot = half_swap_sum(st.l_run[qb]);
          const float inv = l_tot > 0.f ? vs / l_tot : 0.f;
          const bool some = l_tot > 0.f;
          const int col = col0 + qb * 32 + st.i32;
          if (blk.c0 + col < blk.cols) {
            float* orow = p.many_o + (place + col) * DV;
#pragma unroll
            for (int db = 0; db < A::DB; ++db)
#pragma unroll
              for (int g4 = 0; g4 < 4; ++g4) {
                const f32x4 o = {st.oacc[db][qb][4 * g4] * inv, st.oacc[db][qb][4 * g4 + 1] * inv,
                                 st.oacc[db][qb][4 * g4 + 2] * inv, st.oacc[db][qb][4 * g4 + 3] * inv};
                *reinterpret_cast<f32x4*>(orow + db * 32 + 8 * g4 + 4 * st.h) = some ? o : f32x4{0.f, 0.f, 0.f, 0.f};
              }
            if (st.h == 0)  // a sum that is no number stays one in the join
              p.many_lse[place + col] =
                  some ? (st.m_run[qb] - C::P_LOG2 + log2f(l_tot)) * kLn2 : isnan(l_tot) ? NAN : -INFINITY;
          }
        }
        if (me == first_wg && tid == 0)
          p.many_desc[blockIdx.x] = PagedItem{n_parts, s.q0, min(BC, blk.cols - blk.c0), blk.c0, g, me};
      } else {
        // O through LDS, so that each store instruction writes whole rows (layout: see the fused forward).
        unsigned char* stage = smem + wave * WROWS * RB;
        const int osw = o_swizzle<DV>(st.i32) << 4, ohalf = (st.h ^ o_half<DV>(st.i32)) << 3;
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) {
          const float l_tot = half_swap_sum(st.l_run[qb]);
          const float inv = l_tot > 0.f ? vs / l_tot : 0.f;
          const bool some = l_tot > 0.f;  // else no visible key, or a score that is no number
          unsigned char* srow = stage + (qb * 32 + st.i32) * RB + ohalf;
#pragma unroll
          for (int db = 0; db < A::DB; ++db)
#pragma unroll
            for (int g4 = 0; g4 < 4; ++g4) {
              const uint32_t w0 = pack_bf16x2(st.oacc[db][qb][4 * g4] * inv, st.oacc[db][qb][4 * g4 + 1] * inv);
              const uint32_t w1 = pack_bf16x2(st.oacc[db][qb][4 * g4 + 2] * inv, st.oacc[db][qb][4 * g4 + 3] * inv);
              *reinterpret_cast<uint2*>(srow + (((4 * db + g4) << 4) ^ osw)) = some ? make_uint2(w0, w1) : make_uint2(0u, 0u);
            }
          const uint32_t c = (uint32_t)(blk.c0 + col0 + qb * 32 + st.i32);
          if (p.lse != nullptr && st.h == 0 && (int)c < blk.cols) {
            const int qi = (int)fast_div(c, p.m_group, p.sh_group);
            p.lse[(int64_t)(s.q0 + qi) * p.hq + g * p.group + ((int)c - qi * p.group)] =
                some ? (st.m_run[qb] - C::P_LOG2 + log2f(l_tot)) * kLn2 : -INFINITY;
          }
        }
        // Each wave reads back only its own rows, so no barrier. A lane's next column is RPI further on: its address
        // moves by that many heads, and to the next token where the group ends (products of 64 bits for every row
        // would take longer than the stores).
        constexpr int CPR = RB / 16, RPI = 64 / CPR, NIT = WROWS / RPI;
        const int ch = lane % CPR;
        const int rows_on = (int)fast_div(RPI, p.m_group, p.sh_group), heads_on = RPI - rows_on * p.group;
        const int64_t step = rows_on * p.o_token + heads_on * p.o_head, wrap = p.o_token - p.group * p.o_head;
        int c = blk.c0 + col0 + lane / CPR;
        const int qi = (int)fast_div((uint32_t)c, p.m_group, p.sh_group);
        int member = c - qi * p.group;
        uint16_t* dst = p.o + (int64_t)(s.q0 + qi) * p.o_token + (int64_t)(g * p.group + member) * p.o_head + ch * 8;
        u32x4 ov[NIT];
#pragma unroll
        for (int it = 0; it < NIT; ++it) {
          const int row = it * RPI + lane / CPR;
          const unsigned char* chunk = stage + row * RB + ((ch ^ o_swizzle<DV>(row)) << 4);
          const int hl = o_half<DV>(row) << 3;
          const uint2 x = *reinterpret_cast<const uint2*>(chunk + hl);
          const uint2 y = *reinterpret_cast<const uint2*>(chunk + (hl ^ 8));
          ov[it] = u32x4{x.x, x.y, y.x, y.y};
        }
#pragma unroll
        for (int it = 0; it < NIT; ++it) asm volatile("" : "+v"(ov[it]));
#pragma unroll
        for (int it = 0; it < NIT; ++it) {
          if (c < blk.cols) *reinterpret_cast<u32x4*>(dst) = ov[it];
          c += RPI;
          dst += step;
          member += heads_on;
          const bool over = member >= p.group;
          member -= over ? p.group : 0;
          dst += over ? wrap : 0;
        }
      }
    }
    if constexpr (!C::SPLIT) {
      break;
    } else {
      if (!split || r >= r1) break;
      // The next block: of this head, of the next, of the next sequence with any.
      start += kBlockCost + tiles;
      if (++cb == n_cb) {
        cb = 0;
        if (++g == p.c.hkv) {
          g = 0;
          do {
            if (++b >= p.bt.n_seq) return;  // not reached: r < total
            s = load_seq(p.bt, b);
            n_cb = n_blocks<BC>(s, p);
          } while (n_cb == 0);
        }
      }
      __syncthreads();  // the next block's loads overwrite what the stores above were read from
    }
  }
}

// Instances. Long: those of the fused forward (64 query columns per wave; d = 64: 32-key tiles, two workgroups per CU), but
// 64-key tiles at d = 64 over e4m3, whose 32-key tiles would be half a load per wave. Short: 32 columns per wave, two
// workgroups per CU, where sequences have at most 128 row-heads or long blocks would not fill the chip (paged_many; bf16, d_qk 64
// and 128: in 64-key tiles two waves per SIMD do not fit at d_qk = 192).
template <int DQK, int DV, bool E4M3, bool SHORT, bool SPLIT>
struct PagedInstance {
  using C = Cfg<DQK, DV, 64, 4, 2, true, SPLIT, 1, 2, 6, 2, 4, 1, true, E4M3>;
};
template <bool SPLIT>
struct PagedInstance<64, 64, false, false, SPLIT> {
  using C = Cfg<64, 64, 32, 4, 2, true, SPLIT, 2, 2, 4, 2, 4, 1, true>;
};
template <int DQK, int DV, bool SPLIT>
struct PagedInstance<DQK, DV, false, true, SPLIT> {
  using C = Cfg<DQK, DV, 64, 4, 1, true, SPLIT, 2, DQK >= 128 ? 1 : 2, DQK >= 128 ? 2 : 6, 2, DQK >= 128 ? 3 : 4, 1, true>;
};

template <class C>
hipError_t launch_many(PagedParams p, int64_t blocks, hipStream_t stream) {
  void* args[] = {&p};
  const dim3 grid((unsigned)(C::SPLIT ? p.many_wg : blocks * p.c.hkv));
  return hipLaunchKernel(reinterpret_cast<const void*>(&fa_paged_fwd_kernel<C>), grid, dim3(C::NT), args, 0, stream);
}
// Where there is a short instance, the long one runs only grids that fill the chip (paged_many): it is never split.
template <int DQK, int DV, bool E4M3, bool SHORT>
hipError_t launch_many_split(const PagedParams& p, const PagedMany& m, hipStream_t stream) {
  if constexpr (SHORT || E4M3 || DQK == 192) {
    if (m.split) return launch_many<typename PagedInstance<DQK, DV, E4M3, SHORT, true>::C>(p, m.blocks, stream);
  }
  return launch_many<typename PagedInstance<DQK, DV, E4M3, SHORT, false>::C>(p, m.blocks, stream);
}

}  // namespace

PagedMany paged_many(int n_seq, int n_tokens, int max_keys, int hkv, int group, int max_q, int few_cols, int d_qk, bool e4m3) {
  PagedMany m{};
  const int64_t rows = (int64_t)n_tokens * group;
  int64_t seqs = rows / (few_cols + 1);
  if (seqs > n_seq) seqs = n_seq;
  // Short blocks where sequences have no more, and where long ones would not fill the chip twice (d = 128; at d = 64, with
  // two long workgroups per CU, as often). Long against short, a block per workgroup, one box: d = 128 32/8 heads 512 x 512
  // 22.3 : 17.1 us, 2048 x 2048 (256 long blocks) 56.6 : 51.2, 4096 x 4096 (512) 133 : 143, 2048 x 8192 219 : 228; d = 64 16/16
  // 2048 x 2048 48.0 : 28.4, 4096 x 4096 87.1 : 55.8, 3 x 4096 x 4096 (768) 155 : 144.
  const int64_t fill = d_qk == 64 ? 1024 : 512;
  m.is_short = !e4m3 && d_qk != 192 && ((int64_t)max_q * group <= 128 || (rows / 256 + seqs) * hkv < fill);
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

hipError_t launch_paged_many(PagedParams p, const PagedMany& m, int d_qk, bool e4m3, hipStream_t stream) {
  const FastDiv fg = make_fastdiv(p.group);
  p.m_group = fg.m;
  p.sh_group = fg.sh;
  p.many_min_units = kBlockCost + 4;
  p.many_log = 0;
  while ((1 << p.many_log) < p.many_wg) ++p.many_log;
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
