// Attention of few new tokens per sequence over the paged key/value cache (gfx950): the kernel and its instances.
// Internal; included by the kernel sources only.
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "fa_device.h"
#include "fa_e4m3.h"
#include "fa_fastdiv.h"
#include "fa_internal.h"
#include "fa_paged_device.h"

namespace fa {
namespace {

// ---- attention of few rows per sequence -------------------------------------------------------------
//
// An item is one column block of one (sequence, key/value head): up to 32 or 64 of its group * n_q row-heads
// (column c = row * group + member) as the columns of one or two 32x32 MFMAs, against the key tiles visible to them.
// The lengths are on the device, so the host cannot cut the work: all items lie on one line, kItemCost +
// tiles units each, and workgroup i takes units [i * per, (i + 1) * per) of it, `per` from the line's length.
// Every workgroup so has the same work whatever the lengths are, a long sequence is split over as many
// workgroups as it is long, and at most one item per boundary is split. An item that lies in one workgroup is
// finished there; of a split one every workgroup leaves its part (O normalised by the part's own sum, and
// the part's LSE) in its own two places of the workspace, and the join kernel adds the parts with
// their log-sum-exp weights. (A join by the workgroup that finishes last, found by marks in the workspace, saves the second
// launch's 3 us on the host, but is slower on the GPU wherever an item has more than a few parts: 8 000 keys of one
// request 20.0 us against 15.6, 131 072 94.4 against 92.4.)
//
// Inside an item: the waves take 32 keys each of a tile and stream them HBM -> LDS into a ring of their
// own (no barrier), two 16-key halves per K and V block, each half inside one page. S^T = K Q^T, the
// online softmax, O^T += V^T P^T as in the decode kernel. An e4m3 cache stays 8-bit in LDS and is
// widened (exactly) as fragments are read: K to bf16, V to fp16, so that P keeps 11 bits there; the scales
// of K and V enter with the scores' scale and with the final division. P in 16 bits is what the matrix instructions take; row
// sums and maxima keep fp32. Over bf16 caches it adds to the rounding of O: outputs are off by 2.0-2.3e-3 of their norm
// against 1.6-1.7e-3 with P in fp32; over e4m3 caches, in fp16, it does not show.
//
// What bounds it: reading K and V once. 32/8 heads, d = 128: one token over 131 072 keys 83-85 us (6.3-6.5 TB/s) and 5 for
// the join; 64 tokens over 20 000 to 130 keys each 124-128 (6.0-6.2) and 5; 16 over 16 384 and 10 001 in e4m3 71-75 (5.8-6.1) and
// 5. Short ones are bound by the chain of line, table, Q, K, V and join: one token over 1 023 keys 8 us and 3.

//
// With forms (p.f): what a column sees of a tile is a word of 32 bits, scores are capped and biased before it is applied, and
// tiles between the prefix and the first row's window are no part of an item. Still bound by K and V: 32 tokens over 8 000 to
// 700 keys with capped scores 77 us (5.8 TB/s), with slopes 79, without 77, over e4m3 48 with either (4.7); 48 tokens over
// 60 001 and 9 000 e4m3 keys with a window of 4 096 77 (5.2), without one 526.

constexpr int kItemCost = 1;  // fixed cost of an item in tiles
constexpr int kMinUnits = 2;  // least work of a workgroup: one token over 1 023 keys 12.0 us with 2, 15.6 with 4
constexpr float kRise = 8.f;  // how far (log2) a maximum may rise over its reference

template <int DQK_, int DV_, bool FP8_, int QB_, bool STREAM_, int SLOTS_, bool FORM_ = false>
struct FewCfg {
  static constexpr bool FORM = FORM_;                           // scores and masks by p.f
  static constexpr int QB = QB_, COLS = 32 * QB_;               // 32-column MFMA blocks per wave, columns of an item
  static constexpr bool STREAM = STREAM_;                       // K and V loaded past the caches
  static constexpr int DQK = DQK_, DV = DV_, NW = 4, SLOTS = SLOTS_;
  static constexpr bool FP8 = FP8_;
  static constexpr int E = FP8 ? 1 : 2;                         // bytes per element
  static constexpr float P_LOG2 = FP8 ? kE4m3PLog2 : 0.f;       // probabilities and their sums are held times 2^P_LOG2
  static constexpr int KS = DQK / 16, DB = DV / 32;
  static constexpr int KROW = DQK * E, VROW = DV * E;           // bytes per LDS row
  static constexpr int KCH = KROW / 16, VCH = VROW / 16;        // 16-byte chunks per row
  static constexpr int KL = KCH / 4, VL = VCH / 4;              // loads per 16-key half (16 rows / 64 lanes)
  static constexpr int K_BYTES = 32 * KROW, V_BYTES = 32 * VROW, WSLOT = K_BYTES + V_BYTES;
  static constexpr int RING = NW * SLOTS * WSLOT;
  static constexpr int TILE = 32 * NW;                          // keys per tile
  static constexpr int OROW = DV + 4;
  static constexpr int O_BYTES = NW * COLS * OROW * 4;
  static constexpr int JOIN_BYTES = O_BYTES + 2 * NW * COLS * 4;
  static constexpr int LDS_BYTES = RING > JOIN_BYTES ? RING : JOIN_BYTES;
  static constexpr int D = SLOTS - 1;                           // tiles loaded ahead
  static constexpr int L = 2 * (KL + VL);                       // loads per tile
  static_assert(LDS_BYTES <= 163840 && KCH % 4 == 0 && VCH % 4 == 0, "LDS budget, whole loads");
  static_assert(2 * VL + D * L < 64, "vmcnt range");
  static_assert((SLOTS & (SLOTS - 1)) == 0, "a slot's place stays a scalar");
};

__device__ __forceinline__ void load_q16(bf16x8& r, const void* ptr) {
  asm volatile("global_load_dwordx4 %0, %1, off" : "=v"(r) : "v"(ptr) : "memory");
}
__device__ __forceinline__ void q_settled(bf16x8& r) { asm volatile("" : "+v"(r)); }

// Units of a sequence on the line of work, and what they are made of. Where items are taken whole every item is one unit.
template <int TILE, int COLS, bool FORM>
struct SeqWork {
  int tiles, cost, n_cb;
  uint32_t units;  // below 2^31 by the host's check
  __device__ __forceinline__ SeqWork(const PagedSeq& s, const PagedParams& p, int few_cols) {
    const int64_t cols = (int64_t)s.n_q * p.group;
    if constexpr (FORM)
      tiles = SeenTiles<TILE>(p.f, s, 0, s.n_q - 1).n;
    else
      tiles = (s.kv + TILE - 1) / TILE;
    cost = kItemCost + (p.whole ? 0 : tiles);
    n_cb = cols > few_cols ? 0 : (int)((cols + COLS - 1) / COLS);
    units = (uint32_t)n_cb * (uint32_t)p.c.hkv * (uint32_t)cost;
  }
};

template <class C>
__global__ __attribute__((amdgpu_flat_work_group_size(C::NW * 64, C::NW * 64)))
void fa_paged_few_kernel(PagedParams p) {
  constexpr int DQK = C::DQK, DV = C::DV, KS = C::KS, DB = C::DB, NW = C::NW, TILE = C::TILE, D = C::D;
  constexpr int QB = C::QB, COLS = C::COLS;
  constexpr bool FP8 = C::FP8, FORM = C::FORM;
  __shared__ __attribute__((aligned(1024))) unsigned char smem[C::LDS_BYTES];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int i32 = lane & 31, h = lane >> 5;
  const int me = blockIdx.x;

  // The line's length, and the sequence that holds this workgroup's first unit (every wave for itself). The first 64
  // sequences stay in registers, one per lane.
  PagedSeq sl{};
  if (lane < p.bt.n_seq) sl = load_seq_lane<FORM>(p, lane);
  int few_cols = p.few_cols;
  if (few_cols != INT32_MAX && big_work<FORM>(p, sl, lane) < p.many_work) few_cols = INT32_MAX;  // all sequences run here
  uint32_t mine = SeqWork<TILE, COLS, FORM>(sl, p, few_cols).units, incl = wave_scan(mine);
  uint32_t sum = lane_of(incl, 63);
  if (p.bt.n_seq > 64) {
    uint32_t rest = 0;
    for (int c = 64 + lane; c < p.bt.n_seq; c += 64) rest = add_sat(rest, SeqWork<TILE, COLS, FORM>(load_seq_lane<FORM>(p, c), p, few_cols).units);
    sum = add_sat(sum, wave_sum(rest));
  }
  const int total = uniform((int)min(sum, (uint32_t)INT32_MAX));
  const int per = p.whole ? 1 : max(p.min_units, (int)((uint32_t)(total - 1) >> p.wg_log) + 1);
  if (!p.whole && tid == 0) p.desc[me].n_parts = 0;
  if ((int64_t)me * per >= total) return;
  const int r0 = me * per, r1 = min(total - r0, per) + r0;
  int b = 0, start = 0;
  while (true) {
    const uint64_t above = __builtin_amdgcn_ballot_w64(add_sat((uint32_t)start, incl) > (uint32_t)r0);
    if (above != 0) {
      const int l = __builtin_ctzll(above);
      start += (int)lane_of(incl - mine, l);
      sl = seq_of_lane(sl, l);
      b += l;
      break;
    }
    start += (int)lane_of(incl, 63);
    b += 64;
    if (b >= p.bt.n_seq) return;  // not reached: r0 < total
    sl = PagedSeq{};
    if (b + lane < p.bt.n_seq) sl = load_seq_lane<FORM>(p, b + lane);
    mine = SeqWork<TILE, COLS, FORM>(sl, p, few_cols).units;
    incl = wave_scan(mine);
  }

  unsigned char* const ring = smem + wave * C::SLOTS * C::WSLOT;
  const uint32_t ring_lds = __builtin_amdgcn_readfirstlane(lds_offset(ring));
  // Source offsets of this lane in a 16-key half: load i brings 16-byte chunks 64 i .. 64 i + 63, chunk x of
  // the half being chunk x % CH of its row x / CH, whose place holds logical chunk (x % CH) ^ swizzle(row).
  // The swizzles repeat every 16 rows, so both halves have the same offsets.
  uint32_t koff[C::KL], voff[C::VL];
#pragma unroll
  for (int i = 0; i < C::KL; ++i) {
    const int x = i * 64 + lane, row = x / C::KCH;
    const int sw = FP8 ? k8_swizzle<C::KCH>(row) : k_swizzle<DQK>(row);
    koff[i] = (uint32_t)row * (uint32_t)(p.c.k_slot * C::E) + (uint32_t)((x % C::KCH) ^ sw) * 16u;
  }
#pragma unroll
  for (int i = 0; i < C::VL; ++i) {
    const int x = i * 64 + lane, row = x / C::VCH;
    const int sw = FP8 ? v8_swizzle<C::VCH>(row) : v_swizzle<DV>(row);
    voff[i] = (uint32_t)row * (uint32_t)(p.c.v_slot * C::E) + (uint32_t)((x % C::VCH) ^ sw) * 16u;
  }
  // Lane constants of the V transpose reads: the key of a 16-key step and the chunk this lane points at.
  const int v_key = FP8 ? 8 * h + ((lane & 15) >> 1) : 8 * h + ((lane & 15) >> 2);
  const int v_t = FP8 ? (((lane >> 4) & 1) ^ v8_swizzle<C::VCH>(v_key))
                      : ((2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ v_swizzle<DV>(v_key));
  const int v_half = (lane & 1) * 8;

  int r = r0;
  PagedSeq s{uniform(sl.q0), uniform(sl.q_end), uniform(sl.n_q), uniform(sl.kv), uniform(sl.pre)};
  b = uniform(b), start = uniform(start);
  while (r < r1) {
    SeqWork<TILE, COLS, FORM> sw(s, p, few_cols);
    while (sw.units == 0 || (uint32_t)(r - start) >= sw.units) {
      start += (int)sw.units;
      if (++b >= p.bt.n_seq) return;  // not reached: r < total
      s = load_seq<FORM>(p, b);
      sw = SeqWork<TILE, COLS, FORM>(s, p, few_cols);
    }
    const int cost = sw.cost;
    const int item = uniform((int)((uint32_t)(r - start) / (uint32_t)cost)), item0 = start + item * cost;
    const int g = uniform((int)((uint32_t)item / (uint32_t)sw.n_cb)), cb = item - g * sw.n_cb;
    const int end = min(r1 - item0, cost) + item0;
    // Tiles of the item in this workgroup; the item belongs to the workgroups that have tiles of it (one without
    // a tile to that of its first unit).
    int t0 = 0, t1 = sw.tiles, first_wg = me, n_parts = 1;
    bool skip = false;
    if (!p.whole) {
      t0 = max(0, r - item0 - kItemCost), t1 = end - item0 - kItemCost;
      skip = sw.tiles == 0 ? item0 < r0 : t1 <= t0;
      if (sw.tiles != 0) {
        first_wg = uniform((int)((uint32_t)(item0 + kItemCost) / (uint32_t)per));
        // (The line ends inside an item only if q_starts decreases and so many sequences share tokens that it was cut.)
        n_parts = uniform((int)((min((uint32_t)item0 + (uint32_t)cost, (uint32_t)total) - 1u) / (uint32_t)per)) - first_wg + 1;
      }
    }
    r = end;
    if (skip) continue;

    // Columns of this lane, one per 32-column block. Columns past the item's rows repeat the last and are never stored.
    const int cols = s.n_q * p.group, c0 = cb * COLS;
    int last_key[QB];  // without forms
    SeenRow row[QB];   // with them
    float slope[QB];   // times log2(e)
    bf16x8 qf[QB][KS];
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
      const int c = min(c0 + 32 * qb + i32, cols - 1);
      const int qi = (int)fast_div((uint32_t)c, p.m_group, p.sh_group), member = c - qi * p.group;
      if constexpr (FORM) {
        row[qb].init(p.f, s, qi);
        slope[qb] = p.f.slopes != nullptr ? bounded_slope(p.f.slopes[g * p.group + member] * kLog2e) : 0.f;
      } else {
        last_key[qb] = p.causal ? s.kv - s.n_q + qi : s.kv - 1;
      }
      const uint16_t* qp = p.q + (int64_t)(s.q0 + qi) * p.q_token + (int64_t)(g * p.group + member) * p.q_head;
      // bf16: k-step ks holds dims 16 ks + 8 h .. + 7. e4m3: a lane reads 16 bytes of K at once, dims 32 m +
      // 16 h .. + 15, which serve k-steps 2 m and 2 m + 1; Q takes the same order.
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
        load_q16(qf[qb][ks], qp + (FP8 ? 32 * (ks / 2) + 16 * h + 8 * (ks & 1) : 16 * ks + 8 * h));
    }
    // Keys visible to the block's last row; tiles behind them are left out.
    const int last_row = (int)fast_div((uint32_t)min(c0 + COLS - 1, cols - 1), p.m_group, p.sh_group);
    int k_end = p.causal ? max(0, s.kv - s.n_q + last_row + 1) : s.kv;
    int nt = max(0, min(t1, (k_end + TILE - 1) / TILE) - t0);
    // With forms: the sequence's tiles (those of all its rows), and what this block's rows see of them.
    const SeenTiles<TILE> seen(p.f, s, 0, s.n_q - 1);
    auto tile_of = [&](int t) { return FORM ? seen.tile(t) : t; };
    if constexpr (FORM) {
      k_end = SeenTiles<TILE>(p.f, s, 0, last_row).end;
      nt = max(0, min(t1, seen.before((k_end + TILE - 1) / TILE)) - t0);
    }

    const unsigned char* kbase = static_cast<const unsigned char*>(p.c.k) + (int64_t)g * p.c.k_head * C::E;
    const unsigned char* vbase = static_cast<const unsigned char*>(p.c.v) + (int64_t)g * p.c.v_head * C::E;
    const int* table = p.bt.block_table + (int64_t)b * p.bt.table_stride;
    const int smask = (1 << p.c.page_shift) - 1;
    // The pages of this wave's two halves of tile t (an index past the sequence's last page repeats that).
    auto page_of = [&](int t, int u) {
      const int key = min(tile_of(t) * TILE + 32 * wave + 16 * u, s.kv - 1);
      return key < 0 ? -1 : scalar_load(table + (key >> p.c.page_shift));
    };
    // Buffer over the slots of a half that hold keys below `lim`: none where the page is none of the cache's.
    auto half_rsrc = [&](const unsigned char* base, int64_t page_str, int64_t slot_str, int page, int key0, int lim) {
      const bool ok = page >= 0 && page < p.c.n_pages;
      const int64_t at = ((int64_t)(ok ? page : 0) * page_str + (int64_t)(key0 & smask) * slot_str) * C::E;
      const int rows = ok ? max(0, min(16, lim - key0)) : 0;
      const uint64_t a = reinterpret_cast<uint64_t>(base) + (uint64_t)at;
      return u32x4{(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)a),
                   (uint32_t)__builtin_amdgcn_readfirstlane((int)((uint32_t)(a >> 32) & 0xffffu)),
                   (uint32_t)__builtin_amdgcn_readfirstlane(rows * (int)(slot_str * C::E)), 0x00020000u};
    };
    auto issue = [&](int t, int pg0, int pg1) {
      const uint32_t l = (uint32_t)uniform((int)(ring_lds + (uint32_t)((unsigned)t % C::SLOTS) * C::WSLOT));
      const int key0 = tile_of(t) * TILE + 32 * wave;
      const int lim = FORM && seen.gap > 0 && t < seen.pre ? min(s.pre, k_end) : k_end;
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const u32x4 rs = half_rsrc(kbase, p.c.k_page, p.c.k_slot, u ? pg1 : pg0, key0 + 16 * u, lim);
#pragma unroll
        for (int i = 0; i < C::KL; ++i) dma16_buffer<C::STREAM>(rs, koff[i], l + (u * C::KL + i) * 1024);
      }
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const u32x4 rs = half_rsrc(vbase, p.c.v_page, p.c.v_slot, u ? pg1 : pg0, key0 + 16 * u, lim);
#pragma unroll
        for (int i = 0; i < C::VL; ++i) dma16_buffer<C::STREAM>(rs, voff[i], l + C::K_BYTES + (u * C::VL + i) * 1024);
      }
    };
    // Bits 2 k, 2 k + 1: whether the two halves of the k-th tile from the current one on have a page.
    uint32_t valid = 0;
    auto page_bits = [&](int pg0, int pg1) {
      return (uint32_t)(pg0 >= 0 && pg0 < p.c.n_pages) | (uint32_t)(pg1 >= 0 && pg1 < p.c.n_pages) << 1;
    };

    const float ks = FP8 && p.c.k_scale != nullptr ? scalar_load(p.c.k_scale + g) : 1.f;
    const float cs = p.cs * ks, cap_b = FORM ? cap_factor(p.f, cs) : 0.f;
    f32x16 oacc[DB][QB];
    float m_run[QB], l_run[QB];
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
      m_run[qb] = -INFINITY, l_run[qb] = 0.f;
#pragma unroll
      for (int db = 0; db < DB; ++db) oacc[db][qb] = f32x16{};
    }
    const int n0t = t0, n1t = t0 + nt;
    // (Also without a tile: behind k_end nothing is read, and every path waits for Q the same way.)
#pragma unroll
    for (int k = 0; k < D; ++k) {
      const int a = page_of(n0t + k, 0), z = page_of(n0t + k, 1);
      issue(n0t + k, a, z);
      valid |= page_bits(a, z) << (2 * k);
    }
    int pgn0 = page_of(n0t + D, 0), pgn1 = page_of(n0t + D, 1);
    wait_vmcnt<D * C::L>();  // Q
#pragma unroll
    for (int qb = 0; qb < QB; ++qb)
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) q_settled(qf[qb][ks]);

    for (int t = n0t; t < n1t; ++t) {
      compiler_fence();
      issue(t + D, pgn0, pgn1);
      valid |= page_bits(pgn0, pgn1) << (2 * D);
      pgn0 = page_of(t + D + 1, 0), pgn1 = page_of(t + D + 1, 1);
      compiler_fence();
      wait_vmcnt<2 * C::VL + D * C::L>();  // K(t)
      compiler_fence();
      const unsigned char* sK = ring + ((unsigned)t % C::SLOTS) * C::WSLOT;
      const unsigned char* sV = sK + C::K_BYTES;
      const int n0 = tile_of(t) * TILE + 32 * wave;

      // Scores: register r holds key n0 + 16 (r / 8) + 8 h + r % 8 of column i32 (of block qb).
      f32x16 sc[QB];
      const unsigned char* krow = sK + perm32(i32) * C::KROW;
#pragma unroll
      for (int m = 0; m < (FP8 ? KS / 2 : KS); ++m) {
        const u32x4 a =
            *reinterpret_cast<const u32x4*>(krow + (((2 * m + h) ^ (FP8 ? k8_swizzle<C::KCH>(perm32(i32) & 15)
                                                                        : k_lane_swizzle<DQK>(i32))) << 4));
        if constexpr (FP8) {
          const bf16x8 lo = widen_bf16(a[0], a[1]), hi = widen_bf16(a[2], a[3]);
#pragma unroll
          for (int qb = 0; qb < QB; ++qb)
            sc[qb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(lo, qf[qb][2 * m], m == 0 ? f32x16{} : sc[qb], 0, 0, 0);
#pragma unroll
          for (int qb = 0; qb < QB; ++qb)
            sc[qb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(hi, qf[qb][2 * m + 1], sc[qb], 0, 0, 0);
        } else {
#pragma unroll
          for (int qb = 0; qb < QB; ++qb)
            sc[qb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(bit_cast<bf16x8>(a), qf[qb][m], m == 0 ? f32x16{} : sc[qb],
                                                             0, 0, 0);
        }
      }
      const bool there0 = valid & 1u, there1 = valid & 2u;
      valid >>= 2;
      u32x4 pw[QB][2];
#pragma unroll
      for (int qb = 0; qb < QB; ++qb) {
        // Mask keys past the column's last visible key and those of halves without a page.
        float mt = -INFINITY;
        if constexpr (FORM) {
          if (p.f.cap_a != 0.f) {
#pragma unroll
            for (int e = 0; e < 16; ++e) sc[qb][e] = capped(sc[qb][e], p.f.cap_a, cap_b);
          } else {
            sc[qb] *= cs;
          }
          if (p.f.slopes != nullptr) {
            const float far = (float)(row[qb].pos - n0 - 8 * h);  // from the lane's first key
#pragma unroll
            for (int e = 0; e < 16; ++e) sc[qb][e] -= slope[qb] * fabsf(far - (float)(16 * (e >> 3) + (e & 7)));
          }
          const uint32_t held = (there0 ? 0xffffu : 0u) | (there1 ? 0xffff0000u : 0u);
          const uint32_t v = (seen_bits(p.f, s, row[qb], n0) & held) >> (8 * h);
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const float x = (v >> (16 * (e >> 3) + (e & 7))) & 1u ? sc[qb][e] : -INFINITY;
            sc[qb][e] = x;
            mt = fmaxf(mt, x);
          }
        } else {
          const int lim = last_key[qb] - n0 - 8 * h;
          const int lim0 = there0 ? lim : -1, lim1 = there1 ? lim : -1;
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const float x = (16 * (e >> 3) + (e & 7)) > (e < 8 ? lim0 : lim1) ? -INFINITY : sc[qb][e] * cs;
            sc[qb][e] = x;
            mt = fmaxf(mt, x);
          }
        }
        mt = half_swap_max(mt);
        // The reference follows the maximum only where some column's has risen over it by more than 8 (P then stays
        // within 2^8, O / l does not depend on it): O is rescaled in few tiles. It starts at the first visible key's tile.
        if (__builtin_amdgcn_ballot_w64(mt > m_run[qb] + kRise) != 0) {
          const float m_new = fmaxf(m_run[qb], mt);
          const float alpha = __builtin_amdgcn_exp2f(m_run[qb] - (m_new == -INFINITY ? 0.f : m_new));
          m_run[qb] = m_new;
          l_run[qb] *= alpha;
#pragma unroll
          for (int db = 0; db < DB; ++db) oacc[db][qb] *= alpha;
        }
        const float mref = m_run[qb] == -INFINITY ? 0.f : m_run[qb] - C::P_LOG2;
        float rs = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float e0 = __builtin_amdgcn_exp2f(sc[qb][2 * e] - mref);
          const float e1 = __builtin_amdgcn_exp2f(sc[qb][2 * e + 1] - mref);
          rs += e0 + e1;
          pw[qb][e / 4][e % 4] = FP8 ? pack_f16x2(e0, e1) : pack_bf16x2(e0, e1);
        }
        l_run[qb] += rs;
      }
      compiler_fence();
      wait_vmcnt<D * C::L>();  // V(t)
      compiler_fence();
#pragma unroll
      for (int ps = 0; ps < 2; ++ps) {
#pragma unroll
        for (int db = 0; db < DB; ++db) {
          if constexpr (FP8) {
            const unsigned char* vb = sV + (16 * ps + v_key) * C::VROW + (((2 * db) ^ v_t) << 4) + v_half;
            const i32x2 w = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_i32x2*)(vb));
            const f16x8 va = widen_f16(w.x, w.y);
#pragma unroll
            for (int qb = 0; qb < QB; ++qb)
              oacc[db][qb] = __builtin_amdgcn_mfma_f32_32x32x16_f16(va, bit_cast<f16x8>(pw[qb][ps]), oacc[db][qb], 0, 0, 0);
          } else {
            const unsigned char* vb = sV + (16 * ps + v_key) * C::VROW + (((4 * db) ^ v_t) << 4) + v_half;
            const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(vb));
            const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(vb + 4 * C::VROW));
            const bf16x8 va = bit_cast<bf16x8>(__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
            for (int qb = 0; qb < QB; ++qb)
              oacc[db][qb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(va, bit_cast<bf16x8>(pw[qb][ps]), oacc[db][qb], 0, 0, 0);
          }
        }
      }
    }

    // Join the waves through LDS: no load may still be writing the ring, and every wave must be done with its
    // last tile.
    compiler_fence();
    wait_vmcnt<0>();
    compiler_fence();
    __syncthreads();
    float* ob = reinterpret_cast<float*>(smem);               // [wave][column][OROW]
    float* mb = reinterpret_cast<float*>(smem + C::O_BYTES);  // [wave][column]
    float* lb = mb + NW * COLS;                               // [wave][column]
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
      const int at = wave * COLS + 32 * qb + i32;
      const float l_tot = half_swap_sum(l_run[qb]);
      if (h == 0) {
        mb[at] = m_run[qb];
        lb[at] = l_tot;
      }
      float* orow = ob + at * C::OROW + 4 * h;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int g4 = 0; g4 < 4; ++g4)
          *reinterpret_cast<f32x4*>(orow + 32 * db + 8 * g4) = f32x4{oacc[db][qb][4 * g4], oacc[db][qb][4 * g4 + 1],
                                                                     oacc[db][qb][4 * g4 + 2], oacc[db][qb][4 * g4 + 3]};
    }
    __syncthreads();

    constexpr int TPC = NW * 64 / COLS;  // threads per column
    static_assert(DV % (8 * TPC) == 0, "a thread finishes whole 16-byte chunks of the output");
    const int col = tid / TPC, d0 = (tid % TPC) * (DV / TPC);
    if (c0 + col < cols) {
      float mw[NW], M = -INFINITY;
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        mw[w] = mb[w * COLS + col];
        M = fmaxf(M, mw[w]);
      }
      float wt[NW], Lsum = 0.f;
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        wt[w] = mw[w] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mw[w] - M);
        Lsum += wt[w] * lb[w * COLS + col];
      }
      const bool some = Lsum > 0.f;  // else no visible key, or a score that is no number: O = 0, LSE = -inf
      const float vs = FP8 && p.c.v_scale != nullptr ? scalar_load(p.c.v_scale + g) : 1.f;
      const float inv = some ? vs / Lsum : 0.f;
      const float lse = some ? (M - C::P_LOG2 + log2f(Lsum)) * kLn2 : -INFINITY;
      f32x4 o[DV / TPC / 4];
#pragma unroll
      for (int d = 0; d < DV / TPC; d += 4) {
        f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < NW; ++w)
          acc += wt[w] * *reinterpret_cast<const f32x4*>(ob + (w * COLS + col) * C::OROW + d0 + d);
        o[d / 4] = some ? acc * inv : f32x4{0.f, 0.f, 0.f, 0.f};
      }
      if (n_parts == 1) {
        const int row = (int)fast_div((uint32_t)(c0 + col), p.m_group, p.sh_group), mem = (c0 + col) - row * p.group;
        const int head = g * p.group + mem;
        const int64_t tok = s.q0 + row;
        uint16_t* dst = p.o + tok * p.o_token + (int64_t)head * p.o_head + d0;
#pragma unroll
        for (int d = 0; d < DV / TPC; d += 8) {
          const f32x4 x = o[d / 4], y = o[d / 4 + 1];
          *reinterpret_cast<u32x4*>(dst + d) =
              u32x4{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3])};
        }
        if (tid % TPC == 0 && p.lse != nullptr) p.lse[tok * p.hq + head] = lse;
      } else {
        // Place 2 me: a part of an item that begins before; 2 me + 1: the first part of one.
        const int64_t place = 2 * (int64_t)me + (me == first_wg ? 1 : 0);
        float* dst = p.o_part + (place * p.part_cols + col) * DV + d0;
#pragma unroll
        for (int d = 0; d < DV / TPC; d += 4) *reinterpret_cast<f32x4*>(dst + d) = o[d / 4];
        if (tid % TPC == 0) p.lse_part[place * p.part_cols + col] = isnan(Lsum) ? NAN : lse;
      }
    }
    if (n_parts > 1 && me == first_wg && tid == 0)
      p.desc[me] = PagedItem{n_parts, s.q0, min(COLS, cols - c0), c0, g, me};
    __syncthreads();  // the next item's loads overwrite the buffers above
  }
}

// Instances by head dimensions, cache type and 32-column blocks; as many ring slots as leave two workgroups to a CU
// where the waves' join fits in 80 KiB of LDS, else one.
template <int DQK, int DV, bool FP8, int QB, bool STREAM, bool FORM = false>
struct FewInstance {
  static constexpr int kSlots = FP8 && (QB == 2 || DQK == 64) ? 4 : 2;
  using C = FewCfg<DQK, DV, FP8, QB, STREAM, kSlots, FORM>;
  static constexpr int kWorkgroups = C::LDS_BYTES <= 81920 ? 512 : 256;
};

template <class C>
hipError_t launch_few(PagedParams p, hipStream_t stream) {
  void* args[] = {&p};
  return hipLaunchKernel(reinterpret_cast<const void*>(&fa_paged_few_kernel<C>), dim3(p.n_wg), dim3(C::NW * 64), args, 0,
                         stream);
}

// What the launchers fill in.
inline void few_constants(PagedParams& p) {
  p.min_units = kMinUnits;
  p.wg_log = 0;
  while ((1 << p.wg_log) < p.n_wg) ++p.wg_log;
  const FastDiv fg = make_fastdiv(p.group);
  p.m_group = fg.m;
  p.sh_group = fg.sh;
}

}  // namespace
}  // namespace fa
