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
// tokens 200-215 us by box (985-1 055 TFLOP/s; over an e4m3 cache 218, 969), a chunk of 1 024 over 9 000 keys, split, 140
// (1 000) and its part of the join; 32/32 heads, d_qk = 192, 512 tokens over 4 500 keys, split, 64 (700) and 13 for the join. Over
// contiguous keys the fused forward takes 1/1.03 to 1/1.06 of its time from 8 192 tokens on, 1/1.10 at 2 048 (d = 128), 1/1.26
// at 4 096 of 16/16 heads with d = 64.
// With forms (FormKeys below): a tile's exact maximum is computed before its step, which takes the place of redoing tiles, so that
// rows may see their first key anywhere and a bias may rise; tiles that all rows see whole are not masked; tiles between the
// prefix and the block's first window are not visited; with slopes, tiles are taken from the last to the first, so that the
// maximum comes early. Blocks of 128 row-heads, two waves on a SIMD, where there are such instances. 4 096 and 3 001
// tokens, us, plain : masks : caps : slopes : both: 32/8 heads, d = 128 204 : 215 : 265 : 230 : 289, over e4m3 217 : 242 : 368 : 273 : 376;
// 16/16 heads, d_qk = 192 132 : 145 : 204 : 165 : 221; 32/32 heads, d = 64 135 : 148 : 202 : 162 : 231. What a cap or a bias costs is
// VALU time (an exponential, a reciprocal and two operations more a score; one), beside which only another wave of the SIMD
// computes: most with one wave (e4m3, d_qk = 192).
// Internal; included by the kernel sources only.
#pragma once

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
// longest block has 32 units more than an even share, and 1.9 times as many. Measured, a block per workgroup against split,
// 128-row-head blocks, one box: d = 128 32/8 heads 1024 x 1024 26 us against 42, 256 x 4096 (8 times the share) 73 : 42, 512 x
// 4096 (4 times) 74 : 56, 3 x 512 x 4096 (1.4) 112 : 123, 1024 x 8192 (2.0) 148 : 145; d = 64 16/16 2048 x 2048 (26 units more)
// 28 : 36, 256 x 4096 47 : 28, 3 x 1024 x 8192 (1.3) 145 : 135; blocks of 256, d = 128: 2048 x 2048 57 : 79, 1024 x 8192 (2.0)
// 176 : 137, 3 x 512 x 4096 101 : 119. The rule is the same with forms, whose tiles cost more, so that splitting pays a little
// earlier (another box; caps): d = 128 32/8 256 x 4096 102 : 46, 512 x 4096 103 : 64, 1024 x 1024 36 : 37, 3 x 512 x 4096 144 :
// 149, 1024 x 8192 192 : 180 (masks 152 : 150, slopes 168 : 156), trees of 60 of 16 sequences over 9 000 to 1 200 keys 183 :
// 122, over e4m3 268 : 115; e4m3 1024 x 8192 366 : 223; d_qk = 192 32/32 512 x 4500 223 : 99. Off at d = 64 16/16, where it
// does not split: 2048 x 2048 47 : 36, 3 x 1024 x 8192 229 : 189.
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

// The kernel's parameters read anew from where they were passed: what few tiles need is not kept in scalar registers over the
// loop, of which the step and the loads leave none.
__device__ __forceinline__ const __attribute__((address_space(4))) PagedParams& fresh_params() {
  auto p = (const __attribute__((address_space(4))) PagedParams*)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));
  return *p;
}
template <bool FORM>
__device__ __forceinline__ std::conditional_t<FORM, PagedParams, const PagedParams&> reread(const PagedParams& p) {
  if constexpr (FORM) {
    PagedParams q;
    __builtin_memcpy(&q, (const void*)&fresh_params(), sizeof(q));
    return q;
  } else {
    return p;
  }
}
__device__ __forceinline__ PagedForms fresh_forms() {
  const auto& f = fresh_params().f;
  return PagedForms{f.cap_a, f.cap_r, f.slopes, f.prefix_lens, f.mask, f.mask_stride, f.mask_words, f.window, f.causal};
}

// The lane's number without a register that holds it meanwhile.
__device__ __forceinline__ int lane_anew() {
  uint32_t all = ~0u;
  asm volatile("" : "+s"(all));
  return (int)__builtin_amdgcn_mbcnt_hi(all, __builtin_amdgcn_mbcnt_lo(all, 0u));
}

// The state of a wave with forms. Before a step, values() turns a tile's raw scores s into what the step makes exponents of, mul * s
// + add (in units of log2; hidden keys -inf), with as few operations per score as the form allows:
//   masked   nothing: mul = cs
//   capped   s = 1 / (1 + 2^(b s)): mul = -2 a, add = a (capped() in fa_paged_device.h)
//   biased   in a tile before all rows' positions s -= slope / cs * (the lane's last key - key), one operation, and add
//            takes the distance of that last key off (so that both are no more than the whole distance, and near keys lose
//            nothing to far ones); else s -= slope / cs * |p - key|; the final score where it
//            is capped too, where cs is next to 0, and where a bias may reach 2^20: maximum, reference and exponents are
//            rounded apart, by up to 2^-22 of them, and of the final score alone they are the same
template <class C>
struct FormKeys {
  static constexpr int BN = C::WBN, QB = C::QB, KB = BN / 32;
  PagedSeq seq;
  int row[QB];          // of the sequence's new tokens
  int whole0, whole1;   // every row of the block sees the keys from whole0 to before whole1
  float cap_a, cap_b;   // capped; biased: cap_a 0 for none
  float slope[QB];      // biased: times log2(e), over cs unless `final`
  bool final;
  int pos0;             // biased: position of the block's first row
  __device__ __forceinline__ void init_row(const PagedParams& p, int qb, int r, int head) {
    row[qb] = r;
    if constexpr (C::FORM == kFormBiased) slope[qb] = bounded_slope(p.f.slopes[head] * kLog2e);
  }
  __device__ __forceinline__ void init_block(const PagedParams& p, const PagedSeq& s, int row0, int row1, float cs) {
    SeenRow first, last;
    first.init(p.f, s, row0);
    last.init(p.f, s, row1);
    whole0 = last.first, whole1 = first.last + 1;
    seq = s;
    if constexpr (C::FORM != kFormMasked) {
      cap_a = p.f.cap_a;
      cap_b = uniform(cap_factor(p.f, cs));
    }
    if constexpr (C::FORM == kFormBiased) {
      pos0 = first.pos;
      bool steep = false;
#pragma unroll
      for (int qb = 0; qb < QB; ++qb) steep = steep || fabsf(slope[qb]) * (float)max(s.kv, s.n_q) >= 0x1p20f;
      final = cap_a != 0.f || fabsf(cs) < 0x1p-60f || __builtin_amdgcn_ballot_w64(steep) != 0;
#pragma unroll
      for (int qb = 0; qb < QB; ++qb) slope[qb] = final ? slope[qb] : slope[qb] / cs;
    }
  }
  // Whether the tile at key n0 hides a key from some row.
  __device__ __forceinline__ bool hides(int n0) const {
    return !((n0 >= whole0 && n0 + BN <= whole1) || n0 + BN <= seq.pre);
  }
  // Keys of the 32 from n0 on that the column sees, in pages that are there.
  __device__ __forceinline__ uint32_t bits(const PagedForms& f, int qb, int n0, const PagedKeys<true, QB>& pages) const {
    SeenRow r;
    r.init(f, seq, row[qb]);
    uint32_t v = seen_bits(f, seq, r, n0);
    if (pages.holes) {
#pragma unroll
      for (int u = 0; u < 2; ++u) {  // 16 keys lie in one page
        const int key = n0 + 16 * u, page = key < seq.kv ? pages.page_of(key) : 0;
        if (page < 0 || page >= pages.n_pages) v &= u == 0 ? 0xffff0000u : 0x0000ffffu;
      }
    }
    return v;
  }
  static constexpr int key_of(int kb, int r) { return 32 * kb + 16 * (r >> 3) + (r & 7); }  // from the lane's first key on
  static constexpr int kLast = key_of(KB - 1, 15);
  // h: the half of the wave.
  template <class Scores>
  __device__ __forceinline__ float values(Scores& s, float (&add)[QB], int n0, bool masked, float cs, int h,
                                          const PagedKeys<true, QB>& pages) const {
    float mul = cs;
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) add[qb] = 0.f;
    auto each = [&](auto f) {
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int qb = 0; qb < QB; ++qb)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            float x = f(s[kb][qb][r], qb, key_of(kb, r));
            asm volatile("" : "+v"(x));  // in place: products for a branch not taken would move all scores
            s[kb][qb][r] = x;
          }
    };
    if (C::FORM == kFormCapped || (C::FORM == kFormBiased && cap_a != 0.f)) {
      each([&](float x, int, int) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(cap_b * x)); });
      mul = -2.f * cap_a;
#pragma unroll
      for (int qb = 0; qb < QB; ++qb) add[qb] = cap_a;
    }
    if constexpr (C::FORM == kFormBiased) {
      float far[QB];  // the row's position less the lane's first key
#pragma unroll
      for (int qb = 0; qb < QB; ++qb) far[qb] = (float)(seq.kv - seq.n_q + row[qb] - n0 - 8 * h);
      if (!final && n0 + BN <= pos0 + 1) {
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) add[qb] = -(slope[qb] * (far[qb] - (float)kLast)) * cs;
        each([&](float x, int qb, int key) { return fmaf(slope[qb], (float)(key - kLast), x); });
      } else {
        if (final) {
          each([&](float x, int qb, int) { return fmaf(mul, x, add[qb]); });
          mul = 1.f;
#pragma unroll
          for (int qb = 0; qb < QB; ++qb) add[qb] = 0.f;
        }
        each([&](float x, int qb, int key) { return fmaf(-slope[qb], fabsf(far[qb] - (float)key), x); });
      }
    }
    if (masked) {
      const PagedForms f = fresh_forms();
      const uint32_t hidden = mul < 0.f ? 0x7f800000u : 0xff800000u;
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) {
          const uint32_t v = bits(f, qb, n0 + 32 * kb, pages) >> (8 * h);
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            uint32_t m;  // (The builtin becomes an and, a compare and a select.)
            asm("v_bfe_i32 %0, %1, %2, 1" : "=v"(m) : "v"(v), "i"(16 * (r >> 3) + (r & 7)));
            float x = __uint_as_float((__float_as_uint(s[kb][qb][r]) & m) | (hidden & ~m));
            asm volatile("" : "+v"(x));
            s[kb][qb][r] = x;
          }
        }
    }
    return mul;
  }
};

// A block's place: which keys its columns see.
template <int BN, int BC, bool FORM>
struct Block {
  int cols, c0, row0, row1;  // row-heads of the item, the block's first, its first and last row
  int kv_end;                // keys visible to its last row
  int plain;                 // without forms: leading tiles that need no mask for any row
  int pre, gap;              // with forms: its tiles (SeenTiles)
  __device__ __forceinline__ Block(const PagedSeq& s, int cb, const PagedParams& p) {
    cols = s.n_q * p.group;
    c0 = cb * BC;
    row0 = (int)fast_div((uint32_t)c0, p.m_group, p.sh_group);
    row1 = (int)fast_div((uint32_t)min(c0 + BC, cols) - 1u, p.m_group, p.sh_group);
    plain = pre = gap = 0;
    if constexpr (FORM) {
      const SeenTiles<BN> seen(p.f, s, row0, row1);
      kv_end = seen.end, pre = seen.pre, gap = seen.gap;
    } else {
      kv_end = p.causal ? max(0, s.kv - s.n_q + row1 + 1) : s.kv;
      plain = (p.causal ? max(0, s.kv - s.n_q + row0 + 1) : s.kv) / BN;
    }
  }
  __device__ __forceinline__ int tiles() const { return (kv_end + BN - 1) / BN - (FORM ? gap : 0); }
};
template <int BC>
__device__ __forceinline__ int n_blocks(const PagedSeq& s, const PagedParams& p) {
  const int64_t cols = (int64_t)s.n_q * p.group;
  return cols > p.few_cols ? (int)((cols + BC - 1) / BC) : 0;
}
template <int BN, int BC, bool FORM>
__device__ __forceinline__ int head_units(const PagedSeq& s, int n_cb, const PagedParams& p, int lane) {
  uint32_t sum = 0;
  for (int c = lane; c < n_cb; c += 64) sum += (uint32_t)(kBlockCost + Block<BN, BC, FORM>(s, c, p).tiles());
  return (int)wave_sum(sum);
}
template <class C>
__global__ __attribute__((amdgpu_flat_work_group_size(C::NT, C::NT), amdgpu_waves_per_eu(C::WPE, C::WPE)))
void fa_paged_fwd_kernel(PagedParams args) {
  const PagedParams& p = args;
  using A = Attn<C>;
  constexpr int DQK = C::DQK, DV = C::DV, BN = C::BN, QB = C::QB;
  constexpr int BC = C::NWAVES * 32 * QB;  // row-heads per block
  constexpr int R = BN / C::NWAVES;        // keys that a wave brings of a tile
  constexpr int E = C::E;
  constexpr bool FORM = C::FORM != kFormNone;
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
  if (lane < p.bt.n_seq) first = load_seq_lane<FORM>(p, lane);
  auto seqs_from = [&](int c) {
    PagedSeq x{};
    if (c == 0)
      x = first;
    else if (c + lane < p.bt.n_seq)
      x = load_seq_lane<FORM>(p, c + lane);
    return x;
  };
  if (p.few_cols != 0 && big_work<FORM>(p, first, lane) < p.many_work) return;  // all sequences run in the kernel for few rows
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
        sum = add_sat(sum, (uint32_t)min((int64_t)head_units<BN, BC, FORM>(x, n, p, lane) * p.c.hkv, (int64_t)UINT32_MAX));
        longest = max(longest, kBlockCost + Block<BN, BC, FORM>(x, n - 1, p).tiles());
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
        const int units = head_units<BN, BC, FORM>(s, n_cb, p, lane);
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
      const uint32_t u = c + lane < n_cb ? (uint32_t)(kBlockCost + Block<BN, BC, FORM>(s, c + lane, p).tiles()) : 0u;
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
    decltype(auto) p = reread<FORM>(args);
    const Block<BN, BC, FORM> blk(s, cb, p);
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
      if constexpr (FORM)
        lane = lane_anew();
      else if constexpr (C::SPLIT)
        asm volatile("" : "+v"(lane));
      st.i32 = lane & 31;
      st.h = lane >> 5;
      st.v_key = 8 * (lane >> 5) + ((lane & 15) >> (C::E4M3 ? 1 : 2));
      st.v_t = C::E4M3 ? (((lane >> 4) & 1) ^ v8_swizzle<C::VCH>(st.v_key))
                       : ((2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ v_swizzle<DV>(st.v_key));
      st.v_half = (lane & 1) * 8;
      const int kb0 = t0 * BN, t1 = t0 + nt;
      // Keys loaded; behind it the tile loads read zeros. (With forms tiles are not in order: see lim_of.)
      const int kv_lim = FORM ? blk.kv_end : min(blk.kv_end, t1 * BN);
      // First key of the j-th tile from t0 on. A bias by distance takes them from the last one on, so that the maximum comes
      // early.
      auto key_of = [&](int j) {
        if constexpr (FORM) {
          const int at = C::FORM == kFormBiased ? max(tiles - 1 - t0 - j, 0) : t0 + j;
          return (at < blk.pre ? at : at + blk.gap) * BN;
        }
        return kb0 + j * BN;
      };
      auto lim_of = [&](int j) {
        if (FORM && j >= nt) return 0;
        return FORM && blk.gap > 0 && key_of(j) < blk.pre * BN ? s.pre : kv_lim;  // behind the prefix nothing is read
      };
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
        if constexpr (FORM) st.init_row(p, qb, qi, g * p.group + member);
        const uint16_t* qp = p.q + (int64_t)(s.q0 + qi) * p.q_token + (int64_t)(g * p.group + member) * p.q_head;
#pragma unroll
        for (int ks = 0; ks < A::KS; ++ks)
          load_q<A::AG>(st.qf[qb][ks], qp + (C::E4M3 ? 32 * (ks / 2) + 16 * st.h + 8 * (ks & 1) : 16 * ks + 8 * st.h));
      }

      // The pages of this wave's keys of tiles w0 .. w0 + 63, one per lane (behind the last key: the last one's).
      int entries = 0;
      auto window = [&](int w0) {
        const int key = min((FORM ? key_of(min(w0 + lane - t0, nt - 1)) : (w0 + lane) * BN) + wave * R, kv_lim - 1);
        entries = key >= 0 ? st.table[key >> p.c.page_shift] : -1;
        asm volatile("" : "+v"(entries));  // waited for here, not at every use
      };
      // Whether a page of the range is not there. (The first 64 are read beside the window, so that both are waited for
      // once.)
      const int e0 = (kb0 >> p.c.page_shift) + lane, e1 = (kv_lim + smask) >> p.c.page_shift;
      bool hole = false;
      auto look = [&](int from, int to) {
        for (int e = from; e < to; e += 64) {
          const int page = st.table[e];
          hole = hole || page < 0 || page >= p.c.n_pages;
        }
      };
      if constexpr (FORM) {  // the pages of all the block's tiles, those between prefix and window left out
        window(t0);
        const int pre_end = (blk.pre * BN + smask) >> p.c.page_shift;
        look(lane, min(pre_end, e1));
        if (blk.gap > 0) look(((blk.pre + blk.gap) * BN >> p.c.page_shift) + lane, e1);
      } else {
        int page0 = 0;
        if (e0 < e1) page0 = st.table[e0];
        window(t0);
        hole = e0 < e1 && (page0 < 0 || page0 >= p.c.n_pages);
        look(e0 + 64, e1);
      }
      st.holes = __builtin_amdgcn_ballot_w64(hole) != 0;
      const int n_plain = FORM || st.holes ? 0 : min(max(blk.plain - t0, 0), nt);
      if constexpr (FORM) st.init_block(p, s, blk.row0, blk.row1, st.cs);
      auto masked = [&](int j) {
        if constexpr (FORM)
          return st.holes || st.hides(key_of(j));
        else
          return j >= n_plain;
      };

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
        gk = kload.rsrc(page, p.c.n_pages, key_of(j) + wave * R, smask, lim_of(j));
        return page;
      };
      auto aim_v = [&](int j, int page) { gv = vload.rsrc(page, p.c.n_pages, key_of(j) + wave * R, smask, lim_of(j)); };
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
        if constexpr (!FORM) {
          if (n_plain == 0) st.mask_tile(sA, kb0);
#pragma unroll
          for (int qb = 0; qb < QB; ++qb) st.m_run[qb] = st.row_max(sA, qb);
        }
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
        st.step(sA, sB, pA, pB, kread(j + 1), j > 0 ? vread(j - 1) : vzero, masked(j), key_of(j), issue);
        sync_step(j + 1);
        st.step(sB, sA, pB, pA, kread(j + 2), vread(j), masked(j + 1), key_of(j + 1), issue);
      }
      if (j < nt) {
        sync_step(j);
        st.step(sA, sB, pA, pB, kread(j + 1), j > 0 ? vread(j - 1) : vzero, masked(j), key_of(j), issue);
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
      decltype(auto) po = reread<FORM>(args);  // for the output
      if constexpr (FORM)
        lane = lane_anew();
      else if constexpr (C::SPLIT)
        asm volatile("" : "+v"(lane));
      st.i32 = lane & 31;
      st.h = lane >> 5;
      constexpr int WROWS = 32 * QB, RB = DV * 2;
      const int col0 = wave * WROWS;  // this wave's first column of the block
      float vs = 1.f;
      if constexpr (C::E4M3) vs = po.c.v_scale != nullptr ? scalar_load(po.c.v_scale + g) : 1.f;
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
            float* orow = po.many_o + (place + col) * DV;
#pragma unroll
            for (int db = 0; db < A::DB; ++db)
#pragma unroll
              for (int g4 = 0; g4 < 4; ++g4) {
                const f32x4 o = {st.oacc[db][qb][4 * g4] * inv, st.oacc[db][qb][4 * g4 + 1] * inv,
                                 st.oacc[db][qb][4 * g4 + 2] * inv, st.oacc[db][qb][4 * g4 + 3] * inv};
                *reinterpret_cast<f32x4*>(orow + db * 32 + 8 * g4 + 4 * st.h) = some ? o : f32x4{0.f, 0.f, 0.f, 0.f};
              }
            if (st.h == 0)  // a sum that is no number stays one in the join
              po.many_lse[place + col] =
                  some ? (st.m_run[qb] - C::P_LOG2 + log2f(l_tot)) * kLn2 : isnan(l_tot) ? NAN : -INFINITY;
          }
        }
        if (me == first_wg && (FORM ? wave == 0 && lane == 0 : tid == 0))
          po.many_desc[blockIdx.x] = PagedItem{n_parts, s.q0, min(BC, blk.cols - blk.c0), blk.c0, g, me};
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
          if (po.lse != nullptr && st.h == 0 && (int)c < blk.cols) {
            const int qi = (int)fast_div(c, po.m_group, po.sh_group);
            po.lse[(int64_t)(s.q0 + qi) * po.hq + g * po.group + ((int)c - qi * po.group)] =
                some ? (st.m_run[qb] - C::P_LOG2 + log2f(l_tot)) * kLn2 : -INFINITY;
          }
        }
        // Each wave reads back only its own rows, so no barrier. A lane's next column is RPI further on: its address
        // moves by that many heads, and to the next token where the group ends (products of 64 bits for every row
        // would take longer than the stores).
        constexpr int CPR = RB / 16, RPI = 64 / CPR, NIT = WROWS / RPI;
        const int ch = lane % CPR;
        const int rows_on = (int)fast_div(RPI, po.m_group, po.sh_group), heads_on = RPI - rows_on * po.group;
        const int64_t step = rows_on * po.o_token + heads_on * po.o_head, wrap = po.o_token - po.group * po.o_head;
        int c = blk.c0 + col0 + lane / CPR;
        const int qi = (int)fast_div((uint32_t)c, po.m_group, po.sh_group);
        int member = c - qi * po.group;
        uint16_t* dst = po.o + (int64_t)(s.q0 + qi) * po.o_token + (int64_t)(g * po.group + member) * po.o_head + ch * 8;
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
          const bool over = member >= po.group;
          member -= over ? po.group : 0;
          dst += over ? wrap : 0;
        }
      }
    }
    if constexpr (!C::SPLIT) {
      break;
    } else {
      if (!split || r >= r1) break;
      decltype(auto) pn = reread<FORM>(args);
      // The next block: of this head, of the next, of the next sequence with any.
      start += kBlockCost + tiles;
      if (++cb == n_cb) {
        cb = 0;
        if (++g == pn.c.hkv) {
          g = 0;
          do {
            if (++b >= pn.bt.n_seq) return;  // not reached: r < total
            s = load_seq<FORM>(pn, b);
            n_cb = n_blocks<BC>(s, pn);
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
// and 128: in 64-key tiles two waves per SIMD do not fit at d_qk = 192). With forms, which redo no tile, there are registers for a
// second K fragment ahead at d = 128: with it and the step's priority, prompts of 4 096 and 3 001 tokens with masks 221 us -> 212, caps
// 279 -> 262, slopes 233 -> 227.
template <int DQK, int DV, bool E4M3, bool SHORT, bool SPLIT, int FORM = kFormNone>
struct PagedInstance {
  using C = Cfg<DQK, DV, 64, 4, 2, true, SPLIT, 1, 2, 6, 2, 4, 1, true, E4M3, FORM>;
};
template <bool SPLIT>
struct PagedInstance<64, 64, false, false, SPLIT, kFormNone> {
  using C = Cfg<64, 64, 32, 4, 2, true, SPLIT, 2, 2, 4, 2, 4, 1, true>;
};
template <int DQK, int DV, bool SPLIT, int FORM>
struct PagedInstance<DQK, DV, false, true, SPLIT, FORM> {
  using C = Cfg<DQK, DV, 64, 4, 1, true, SPLIT, 2, DQK >= 128 && FORM == kFormNone ? 1 : 2, DQK >= 128 ? 2 : 6, 2, DQK >= 128 ? 3 : 4, 1, true, false, FORM>;
};

template <class C>
hipError_t launch_many(PagedParams p, int64_t blocks, hipStream_t stream) {
  void* args[] = {&p};
  const dim3 grid((unsigned)(C::SPLIT ? p.many_wg : blocks * p.c.hkv));
  return hipLaunchKernel(reinterpret_cast<const void*>(&fa_paged_fwd_kernel<C>), grid, dim3(C::NT), args, 0, stream);
}
// What the launchers fill in.
inline void many_constants(PagedParams& p) {
  const FastDiv fg = make_fastdiv(p.group);
  p.m_group = fg.m;
  p.sh_group = fg.sh;
  p.many_min_units = kBlockCost + 4;
  p.many_log = 0;
  while ((1 << p.many_log) < p.many_wg) ++p.many_log;
}

}  // namespace
}  // namespace fa
