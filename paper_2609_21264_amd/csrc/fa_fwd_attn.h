// The pipelined attention step of the fused forward kernels (gfx950): matrix-instruction helpers, the compile-time
// configuration of an instance, and the per-wave state and math of a step. The head comment of
// fa_fwd_kernel.hip describes the mapping onto the chip; fa_paged_fwd_kernel.hip runs the same step over a paged
// cache. Internal; included by the kernel sources only.
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <type_traits>

#include "fa_device.h"
#include "fa_e4m3.h"
#include "fa_fastdiv.h"

namespace fa {
namespace {

// A tile's exponentials are accepted when every lane's sum of them is at most 2^8: then no
// probability exceeds 2^8 relative to the reference maximum.
constexpr float kOverflowSum = 256.0f;

// Layout of the output tile staged in LDS for coalesced stores: row R of a wave's tile (DV bf16,
// 16-byte chunks) keeps logical chunk c at chunk c ^ o_swizzle(R), with the chunk's two 8-byte
// halves exchanged when o_half(R) = 1. The accumulator layout writes 8 bytes per lane for 32 rows at
// once and the coalesced read takes 8 bytes per lane across consecutive rows; with this layout both
// touch 32 different 8-byte bank slots per cycle.
template <int DV>
__device__ __forceinline__ int o_swizzle(int r) { return DV >= 128 ? (r & 15) : ((r >> 1) & 7); }
template <int DV>
__device__ __forceinline__ int o_half(int r) { return DV >= 128 ? ((r ^ (r >> 4)) & 1) : (((r >> 1) ^ (r >> 4)) & 1); }

// The P V product is issued through inline asm so that its accumulators O stay in AGPRs for the
// whole kernel (the score product uses the builtin; its accumulators are VGPRs). The compiler does
// not model hazards of inline asm, so:
//  * mfma_out starts with s_nop 1: its P operand may have just been written by VALU, which needs
//    2 wait states before an MFMA reads it (mfma_out_settled omits them where P is old);
//  * agpr_fence() separates asm MFMA writes of O from compiler-generated accesses (initialisation,
//    rescale, epilogue) in both directions: 18 wait states cover the MFMA write-to-read distance,
//    and the operand tie keeps the order;
//  * consecutive MFMAs accumulating into exactly the same registers need no wait states.
// AG selects where O and Q live: AGPRs (one wave per SIMD, where the VGPRs alone cannot hold the
// step's scores, probabilities and fragments next to them) or VGPRs (two waves per SIMD: the
// compiler splits a wave's 256 registers evenly between the two files as soon as any AGPR is used,
// which would leave 128 VGPRs for the step; with no AGPR all 256 are VGPRs).
template <bool AG>
__device__ __forceinline__ void mfma_out(f32x16& acc, const bf16x8& v, const bf16x8& pt) {
  if constexpr (AG)
    asm("s_nop 1\n\tv_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+a"(acc) : "v"(v), "v"(pt));
  else
    asm("s_nop 1\n\tv_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+v"(acc) : "v"(v), "v"(pt));
}
// Same without the leading wait states, for operands no VALU instruction has written recently: in
// the pipelined step, P was packed a whole step earlier and V comes from LDS.
template <bool AG>
__device__ __forceinline__ void mfma_out_settled(f32x16& acc, const bf16x8& v, const bf16x8& pt) {
  if constexpr (AG)
    asm("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+a"(acc) : "v"(v), "v"(pt));
  else
    asm("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+v"(acc) : "v"(v), "v"(pt));
}
// The same for operands in fp16 (over e4m3 tiles).
template <bool AG>
__device__ __forceinline__ void mfma_out_f16(f32x16& acc, const bf16x8& v, const bf16x8& pt) {
  if constexpr (AG)
    asm("s_nop 1\n\tv_mfma_f32_32x32x16_f16 %0, %1, %2, %0" : "+a"(acc) : "v"(v), "v"(pt));
  else
    asm("s_nop 1\n\tv_mfma_f32_32x32x16_f16 %0, %1, %2, %0" : "+v"(acc) : "v"(v), "v"(pt));
}
template <bool AG>
__device__ __forceinline__ void mfma_out_settled_f16(f32x16& acc, const bf16x8& v, const bf16x8& pt) {
  if constexpr (AG)
    asm("v_mfma_f32_32x32x16_f16 %0, %1, %2, %0" : "+a"(acc) : "v"(v), "v"(pt));
  else
    asm("v_mfma_f32_32x32x16_f16 %0, %1, %2, %0" : "+v"(acc) : "v"(v), "v"(pt));
}
template <bool AG>
__device__ __forceinline__ void agpr_fence(f32x16& acc) {
  if constexpr (AG)
    asm volatile("s_nop 7\n\ts_nop 7\n\ts_nop 3" : "+a"(acc));
  else
    asm volatile("s_nop 7\n\ts_nop 7\n\ts_nop 3" : "+v"(acc));
}
// 16 bytes of Q straight into its register tuple (only read as an MFMA operand, so it never needs a
// copy). The load is not waited for here: the caller waits on vmcnt and then passes the value
// through q_ready(), which keeps every read of it after that wait.
template <bool AG>
__device__ __forceinline__ void load_q(bf16x8& r, const void* ptr) {
  if constexpr (AG)
    asm volatile("global_load_dwordx4 %0, %1, off" : "=a"(r) : "v"(ptr) : "memory");
  else
    asm volatile("global_load_dwordx4 %0, %1, off" : "=v"(r) : "v"(ptr) : "memory");
}
template <bool AG>
__device__ __forceinline__ void q_ready(bf16x8& r) {
  if constexpr (AG)
    asm volatile("" : "+a"(r));
  else
    asm volatile("" : "+v"(r));
}

// Slot of a tile in a ring of N slots of STEP bytes. A ring of 2 or 4 slots takes the low bits of the
// tile index. For 3 slots the remainder would cost a multiply-high chain in front of each step's first
// LDS reads, so the offset is carried from tile to tile instead (next()): one add, compare and select,
// in inline assembly so that they stay scalar: the loads' LDS base (M0) must be a scalar, and a select
// that also feeds vector addresses is selected as a vector instruction. Measured (interleaved, one
// box): H4 777 x 3001 d128 28.5 -> 26.7 us, one head S16384 d128 153.9 -> 145.2 us, B2 28/4 777 x 5001
// 119.5 -> 114.3 us; carrying the power-of-two rings too cost B8 H12 S512 d64 2.5 %, so they are not.
template <int STEP, int N>
struct Ring {
  static constexpr bool kCarried = (N & (N - 1)) != 0;
  int off;  // carried offset
  __device__ __forceinline__ explicit Ring(int tile) : off(tile % N * STEP) {}
  __device__ __forceinline__ void next() {
    if constexpr (kCarried)
      asm("s_add_u32 %0, %0, %1\n\ts_cmp_eq_u32 %0, %2\n\ts_cselect_b32 %0, 0, %0"
          : "+s"(off)
          : "i"(STEP), "i"(STEP * N)
          : "scc");
  }
  // Offset of tile `t`, which is the tile the carried offset stands at.
  __device__ __forceinline__ int at(int t) const {
    if constexpr (kCarried) return off;
    return (int)((unsigned)t % N) * STEP;
  }
};

// Forms of an instance: keys may be hidden otherwise than by a last one, and scores be capped, or be biased by distance and perhaps
// capped.
constexpr int kFormNone = 0, kFormMasked = 1, kFormCapped = 2, kFormBiased = 3;

// Compile-time configuration of one kernel instance: head dimensions, key-tile width, waves per
// workgroup, 32-row query blocks per wave, causal masking, split mode, workgroups sharing a CU (OCC),
// K and V fragments read ahead from LDS (KPF, VPF), K and V ring slots in LDS (NKR, NVR), and the
// parts each key tile is split into between the waves (KSPLIT).
template <int DQK_, int DV_, int BN_, int NWAVES_, int QB_, bool CAUSAL_, bool SPLIT_, int OCC_, int KPF_, int VPF_,
          int NKR_, int NVR_, int KSPLIT_ = 1, bool PAGED_ = false, bool E4M3_ = false, int FORM_ = kFormNone>
struct Cfg {
  static constexpr int DQK = DQK_, DV = DV_, BN = BN_, NWAVES = NWAVES_, QB = QB_;
  // KSPLIT = 2: the waves form two sets of NWAVES / 2 (RWAVES) that own the same query rows; set k
  // takes the k-th 32-key half of every key tile (WBN keys per wave and tile), and the two partial
  // results of each row are merged in LDS at the end.
  static constexpr int KSPLIT = KSPLIT_, RWAVES = NWAVES / KSPLIT_, WBN = BN_ / KSPLIT_;
  static constexpr int KPF = KPF_, VPF = VPF_;
  static constexpr int OCC = OCC_;  // workgroups sharing a CU
  static constexpr bool CAUSAL = CAUSAL_;
  // SPLIT: each workgroup takes one of n_split contiguous parts of its query block's key tiles and
  // writes a partial result (O normalised by its own row sum, fp32, and its LSE) for a merge pass.
  static constexpr bool SPLIT = SPLIT_;
  // PAGED: the keys lie in pages (PagedKeys below), the columns of a wave are any rows of any of the group's heads,
  // and the last key each of them sees is in a register.
  static constexpr bool PAGED = PAGED_;
  static constexpr int FORM = FORM_;  // by FormKeys, which the paged kernel defines
  // E4M3: K and V tiles are 8-bit. They stay so in LDS and are widened as fragments are read: K to bf16, V to fp16, with
  // P in fp16 too. The order of the dims in a score product follows the 16-byte reads of K: k-steps 2 m and 2 m + 1
  // take dims 32 m + 16 h + 0 .. 7 and + 8 .. 15 in lane half h.
  static constexpr bool E4M3 = E4M3_;
  static constexpr int E = E4M3_ ? 1 : 2;  // bytes per element of K and V
  static constexpr float P_LOG2 = E4M3_ ? kE4m3PLog2 : 0.f;  // probabilities and their sums are held times 2^P_LOG2
  static constexpr float OVERFLOW_SUM = kOverflowSum * (E4M3_ ? 1 << (int)kE4m3PLog2 : 1);
  static constexpr bool CHUNKED = QB > 1;  // long instance: key/value heads in chunks (launch_cfg)
  static constexpr int NT = NWAVES * 64;
  // Waves per SIMD the registers are budgeted for: the workgroup's own (4 SIMDs per CU) times the
  // workgroups that share a CU (OCC_).
  static constexpr int WPE = (NWAVES > 4 ? NWAVES / 4 : 1) * OCC_;
  static constexpr int BM = RWAVES * 32 * QB;  // query rows per workgroup holding one query head
  static constexpr int KCH = DQK * E / 16;          // 16-byte chunks per K-tile row
  static constexpr int VCH = DV * E / 16;           // 16-byte chunks per V-tile row
  static constexpr int K_BYTES = BN * DQK * E;
  static constexpr int V_BYTES = BN * DV * E;
  // Ring slots. Step j loads K(j + KA) into the slot of K(j) and V(j + VA) into the slot of V(j-2):
  // both were last read in step j-1, which every wave has finished at the barrier of step j.
  static constexpr int NKR = NKR_, NVR = NVR_;
  static constexpr int KA = NKR, VA = NVR - 2;  // how far ahead step j loads K and V tiles
  static constexpr int RING_BYTES = NKR * K_BYTES + NVR * V_BYTES;
  // The rings' LDS also stages the output tile (STAGE_BYTES) and, behind it, the exchange of the key
  // parts' results (XCH_BYTES: per lane of every row chunk, O of all parts but one and every part's
  // reference maximum and row sum); with small key tiles these are the larger.
  static constexpr int STAGE_BYTES = RWAVES * 32 * QB * DV * 2;
  static constexpr int XCH_BYTES =
      KSPLIT > 1 ? RWAVES * ((KSPLIT - 1) * (DV / 2) + KSPLIT * 2) * QB * 64 * 4 : 0;
  static constexpr int LDS_BYTES =
      RING_BYTES > STAGE_BYTES + XCH_BYTES ? RING_BYTES : STAGE_BYTES + XCH_BYTES;
  // Direct-to-LDS loads per wave per tile (each moves 64 lanes x 16 bytes).
  static constexpr int K_LOADS = BN * KCH / 64 / NWAVES;
  static constexpr int V_LOADS = BN * VCH / 64 / NWAVES;
  static_assert(DQK % 32 == 0 && DV % 64 == 0, "head dims: d_qk multiple of 32, d_v multiple of 64");
  static_assert(WBN % 32 == 0, "every wave takes whole 32-key blocks of a tile");
  static_assert((BN * KCH) % (64 * NWAVES) == 0 && (BN * VCH) % (64 * NWAVES) == 0, "tile split over waves");
  // KA - 1 <= VA <= KA: V(j-1) is issued before K(j+1) (so one counted wait covers both), and the
  // prologue's groups j = -KA .. -1 hold every tile's first load.
  static_assert(NKR >= 2 && NKR + 1 <= NVR && NVR <= NKR + 2, "ring sizes");
  static_assert(V_LOADS + KA * (K_LOADS + V_LOADS) < 64 && VA * (K_LOADS + V_LOADS) < 64, "vmcnt range");
  static_assert(LDS_BYTES * OCC_ <= 163840, "LDS budget of the workgroups sharing a CU");
  static_assert(KSPLIT == 1 || (!SPLIT && NWAVES % KSPLIT == 0), "key parts: equal wave sets, not split mode");
};

// What the step needs to know of a paged sequence (nothing otherwise): the last key that each of the lane's
// columns sees, the pages, and whether some page that it visits is not there (its keys are masked then).
template <bool PAGED, int QB>
struct PagedKeys {};
template <int QB>
struct PagedKeys<true, QB> {
  int last_key[QB];
  const int* table;
  int64_t page_stride, slot_stride;
  int page_shift, n_pages;
  bool holes;
  __device__ __forceinline__ int page_of(int key) const {
    return *(const __attribute__((address_space(4))) int*)(uintptr_t)(table + (key >> page_shift));
  }
};

// Per-wave state and the math of the pipelined step.
//
// Reference maximum (the lazy form of Alg. 1's running maximum): the first tile sets m_run to the
// exact row maximum. Afterwards the per-element maximum is not computed: each lane's sum of its
// tile exponentials bounds every one of them, so when all lane sums stay <= 2^8 no probability
// exceeds 2^8 and the tile is final. Otherwise (a new maximum well above the reference; rare) the
// tile is redone from its exact row maximum, with O and l rescaled by 2^(m_old - m_new) (rebase).
// O / l is invariant under the choice of reference, and l >= 1 since the reference is always a
// score that has been seen.
template <class C>
struct FormKeys;
struct NoForms {};
template <class C>
struct Attn : PagedKeys<C::PAGED, C::QB>, std::conditional_t<C::FORM != kFormNone, FormKeys<C>, NoForms> {
  static constexpr int DQK = C::DQK, DV = C::DV, BN = C::WBN, QB = C::QB;  // BN: this wave's keys of a tile
  static constexpr int KS = DQK / 16;  // k-steps of the score product
  static constexpr int KB = BN / 32;   // 32-key blocks per tile
  static constexpr int DB = DV / 32;   // 32-dim blocks of the output
  static constexpr int PS = BN / 16;   // k-steps of the P V product (16-key chunks)

  typedef f32x16 Scores[KB][QB];    // S^T of one tile, raw (unscaled)
  typedef uint32_t Probs[KB][QB][8];  // P of one tile as packed bf16 pairs

  static constexpr int NMS = KS * KB * QB;  // score MFMAs per tile
  static constexpr int NMP = PS * DB * QB;  // P V MFMAs per tile
  static constexpr int NSL = NMS + NMP;     // MFMA slots per step
  static constexpr bool AG = C::WPE == 1;   // O and Q in AGPRs
  static constexpr int NEP = KB * QB * 8;   // exponential pairs per lane per tile
  static constexpr int NVF = PS * DB;       // V fragments per tile
  static constexpr int KPF = C::KPF;        // K fragments read ahead
  static constexpr int VPF = C::VPF;        // V fragments read ahead

  int i32, h, qw, diag, sk;
  const uint16_t* kg;  // this workgroup's K head in global memory (rebase only)
  float cs;            // scale * log2(e), signed
  float mask_val;      // a score that cs maps to -inf
  int v_key, v_t, v_half;
  bf16x8 qf[QB][KS];
  f32x16 oacc[DB][QB];
  float m_run[QB], l_run[QB];

  // Slot order of a step: the P V MFMAs of tile j-1 first (chunk c of P, 16 keys, in slots
  // [c * E0, (c + 1) * E0)), then the score MFMAs of tile j+1 (32-key-block-major, so that the score
  // accumulators of block kb of the new tile are written only after the exponentials of block kb of
  // the current one, and the two score tiles overlap in registers only partly).
  static constexpr int E0 = NMP / PS;
  static constexpr bool slot_is_score(int sl) { return sl >= NMP; }

  __device__ __forceinline__ u32x4 kfrag(const unsigned char* sK, int ks, int kb) const {
    const int row = kb * 32 + perm32(i32);
    if constexpr (C::E4M3)  // ks even: both of k-steps ks and ks + 1
      return *reinterpret_cast<const u32x4*>(sK + row * DQK + (((ks + h) ^ k8_swizzle<C::KCH>(perm32(i32) & 15)) << 4));
    return *reinterpret_cast<const u32x4*>(sK + row * (DQK * 2) + (((ks * 2 + h) ^ k_lane_swizzle<DQK>(i32)) << 4));
  }
  // A operand V^T[dims db*32 + 0..31][keys 16*ps + 0..15]: lane (group G, slot j) points the
  // transpose read at key 16*ps + 8*(G/2) + j/4 (then +4), dims db*32 + 16*(G%2) + 4*(j%4).
  __device__ __forceinline__ bf16x8 vfrag(const unsigned char* sV, int ps, int db) const {
    if constexpr (C::E4M3) {  // 8-bit yet: the first two registers
      const unsigned char* at = sV + (ps * 16 + v_key) * DV + (((db * 2) ^ v_t) << 4) + v_half;
      const i32x2 w = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_i32x2*)(at));
      return bit_cast<bf16x8>(u32x4{(uint32_t)w.x, (uint32_t)w.y, 0u, 0u});
    }
    const unsigned char* base = sV + (ps * 16 + v_key) * (DV * 2) + (((db * 4) ^ v_t) << 4) + v_half;
    const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(base));
    const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(base + 4 * DV * 2));
    return bit_cast<bf16x8>(__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  }

  // Score MFMA number i of a tile in 32-key-block-major order (kb, ks, qb); K fragments (sequence
  // f = kb*KS + ks) are read KPF ahead.
  __device__ __forceinline__ void score_mfma(Scores& s, u32x4 (&kf)[KB * KS], const unsigned char* sK, int i) {
    const int kb = i / (KS * QB), ks = (i / QB) % KS, qb = i % QB, f = kb * KS + ks;
    if constexpr (C::E4M3) {
      // kf[f] of an even f holds the 8-bit fragments f and f + 1, kf[f + 1] the widened one in use; KPF reads ahead.
      if (qb == 0) {
        if (f % 2 == 0 && f + 2 * KPF < KB * KS) kf[f + 2 * KPF] = kfrag(sK, (f + 2 * KPF) % KS, (f + 2 * KPF) / KS);
        kf[f | 1] = f % 2 == 0 ? bit_cast<u32x4>(widen_bf16(kf[f][0], kf[f][1]))
                               : bit_cast<u32x4>(widen_bf16(kf[f - 1][2], kf[f - 1][3]));
      }
      s[kb][qb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(bit_cast<bf16x8>(kf[f | 1]), qf[qb][ks],
                                                          ks == 0 ? f32x16{} : s[kb][qb], 0, 0, 0);
      return;
    }
    if (qb == 0 && f + KPF < KB * KS) kf[f + KPF] = kfrag(sK, (f + KPF) % KS, (f + KPF) / KS);
    s[kb][qb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(bit_cast<bf16x8>(kf[f]), qf[qb][ks],
                                                        ks == 0 ? f32x16{} : s[kb][qb], 0, 0, 0);
  }
  // The first KPF reads of a tile's K fragments.
  __device__ __forceinline__ void first_kfrags(u32x4 (&kf)[KB * KS], const unsigned char* sK) const {
    constexpr int EACH = C::E4M3 ? 2 : 1;  // fragments per read
#pragma unroll
    for (int f = 0; f < KPF * EACH && f < KB * KS; f += EACH) kf[f] = kfrag(sK, f % KS, f / KS);
  }
  __device__ __forceinline__ void scores(Scores& s, const unsigned char* sK) {
    u32x4 kf[KB * KS];
    first_kfrags(kf, sK);
#pragma unroll
    for (int i = 0; i < NMS; ++i) score_mfma(s, kf, sK, i);
  }

  // Masked keys of tile n0 (key > i + diag, or key >= Sk) get mask_val. The select is a bit
  // select on the sign of (lim - key offset): a compare per element would need a scalar register
  // pair per mask, and the scheduler hoists all 64 of them.
  __device__ __forceinline__ void mask_tile(Scores& s, int n0) const {
    const uint32_t mv = __float_as_uint(mask_val);
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
      int last_key;
      if constexpr (C::PAGED) {
        last_key = this->last_key[qb];
      } else {
        const int row = qw + qb * 32 + i32;
        last_key = C::CAUSAL ? min(row + diag, sk - 1) : sk - 1;
      }
      const int lim = last_key - n0 - 8 * h;  // key offset kb*32 + 16*(r/8) + r%8 is masked iff > lim
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const uint32_t m = (uint32_t)((lim - (kb * 32 + 16 * (r >> 3) + (r & 7))) >> 31);  // all ones if masked
          s[kb][qb][r] = __uint_as_float((__float_as_uint(s[kb][qb][r]) & ~m) | (mv & m));
        }
    }
    if constexpr (C::PAGED) {
      if (!this->holes) return;
      // Registers 8 u .. 8 u + 7 of block kb hold keys of one page.
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const int key = n0 + kb * 32 + 16 * u;
          const int page = key < sk ? this->page_of(key) : 0;
          const uint32_t m = page < 0 || page >= this->n_pages ? ~0u : 0u;
#pragma unroll
          for (int qb = 0; qb < QB; ++qb)
#pragma unroll
            for (int r = 8 * u; r < 8 * u + 8; ++r)
              s[kb][qb][r] = __uint_as_float((__float_as_uint(s[kb][qb][r]) & ~m) | (mv & m));
        }
    }
  }

  // Exact maximum of cs * score over the row (both lane halves), -inf if every key is masked.
  __device__ __forceinline__ float row_max(const Scores& s, int qb) const {
    float m = -INFINITY;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int r = 0; r < 16; ++r) m = fmaxf(m, s[kb][qb][r] * cs);
    return half_swap_max(m);
  }
  // The same of mul * score + add (which the halves may have each for itself), multiplied last.
  __device__ __forceinline__ float row_max_of(const Scores& s, int qb, float mul, float add) const {
    float m = s[0][qb][0];
    if (mul >= 0.f) {
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r) m = fmaxf(m, s[kb][qb][r]);
    } else {
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r) m = fminf(m, s[kb][qb][r]);
    }
    return half_swap_max(fmaf(m, mul, add));
  }

  // Element schedule of the step: the NEL = 2 * NEP exponentials of a tile are spread
  // one by one over the NSL MFMA slots (element e in slot e * NSL / NEL), each as one fma and one
  // exp2 right after the slot's MFMA; the two adds and the pack of pair u follow in the slot after
  // the one of its second element. At d = 128 a slot then carries 3 and 6 full-rate-equivalent VALU
  // instructions in turn, within what a 32-cycle MFMA absorbs. A pair's pack writes P chunk c only
  // after the P V MFMAs of chunk c (slots [c * E0, (c + 1) * E0)) for every c >= 1, so the old and new
  // P share registers there; chunk 0 is written earlier and takes registers of its own.
  static constexpr int NEL = 2 * NEP;
  static constexpr int elem_begin(int sl) { return (sl * NEL + NSL - 1) / NSL; }
  static constexpr int elem_end(int sl) { return ((sl + 1) * NEL + NSL - 1) / NSL; }
  static constexpr bool packs_follow_pv() {
    for (int u = 0; u < NEP; ++u) {
      int sl = 0;
      while (elem_end(sl) <= 2 * u + 1) ++sl;  // slot of element 2u+1
      const int c = u / (QB * 4);             // P chunk (16 keys) of pair u
      if (c >= 1 && sl + 1 < (c + 1) * E0) return false;
    }
    return true;
  }
  static_assert(packs_follow_pv(), "a pack would overwrite P of a chunk before its P V MFMAs");
  static constexpr bool at_most_two_elems_per_slot() {
    for (int sl = 0; sl < NSL; ++sl)
      if (elem_end(sl) - elem_begin(sl) > 2) return false;
    return true;
  }

  // Element e of a tile: p = 2^(mul * s - m_ref), mul = cs without forms.
  __device__ __forceinline__ float exp_elem(int e, const Scores& cur, const float (&mref)[QB], float mul) const {
    const int u = e >> 1, qb = u % QB, rp = (u / QB) % 8, kb = u / (QB * 8);
    float x = __builtin_amdgcn_exp2f(fmaf(cur[kb][qb][2 * rp + (e & 1)], mul, -mref[qb]));
    asm volatile("" : "+v"(x));
    return x;
  }
  // Pair u: the lane's row sum and the bf16 pair. The first pair of each row block starts the sum.
  __device__ __forceinline__ void pack_pair(int u, float e0, float e1, Probs& pk, float (&rs)[QB]) const {
    const int qb = u % QB, rp = (u / QB) % 8, kb = u / (QB * 8);
    if (u < QB)
      rs[qb] = e0 + e1;
    else
      rs[qb] += e0 + e1;
    pk[kb][qb][rp] = C::E4M3 ? pack_f16x2(e0, e1) : pack_bf16x2(e0, e1);
    asm volatile("" : "+v"(pk[kb][qb][rp]));
  }

  // P V MFMA number p of a tile (order ps, db, qb), V fragments read VPF ahead. `settled`: P was
  // written long before (in the step: one step earlier), so no wait states are needed.
  __device__ __forceinline__ void pv_mfma(int p, const Probs& pk, bf16x8 (&vf)[NVF], const unsigned char* sV,
                                          bool settled = false) {
    const int t = p / QB, qb = p % QB, ps = t / DB, db = t % DB;
    if (qb == 0 && t + VPF < NVF) vf[t + VPF] = vfrag(sV, (t + VPF) / DB, (t + VPF) % DB);
    const int kb = ps >> 1, base = (ps & 1) * 4;
    const u32x4 w = {pk[kb][qb][base], pk[kb][qb][base + 1], pk[kb][qb][base + 2], pk[kb][qb][base + 3]};
    if constexpr (C::E4M3) {
      if (qb == 0) {
        const u32x4 raw = bit_cast<u32x4>(vf[t]);
        vf[t] = bit_cast<bf16x8>(widen_f16(raw[0], raw[1]));
      }
      if (settled && qb > 0)  // widened a slot ago
        mfma_out_settled_f16<AG>(oacc[db][qb], vf[t], bit_cast<bf16x8>(w));
      else
        mfma_out_f16<AG>(oacc[db][qb], vf[t], bit_cast<bf16x8>(w));
      return;
    }
    if (settled)
      mfma_out_settled<AG>(oacc[db][qb], vf[t], bit_cast<bf16x8>(w));
    else
      mfma_out<AG>(oacc[db][qb], vf[t], bit_cast<bf16x8>(w));
  }

  // All P V MFMAs of one tile (the last tile, after the loop).
  __device__ __forceinline__ void pv_tile(const Probs& pk, const unsigned char* sV) {
    bf16x8 vf[NVF];
#pragma unroll
    for (int t = 0; t < VPF && t < NVF; ++t) vf[t] = vfrag(sV, t / DB, t % DB);
#pragma unroll
    for (int pi = 0; pi < NMP; ++pi) pv_mfma(pi, pk, vf, sV);
  }

  // Redo a tile's exponentials from its exact row maximum; O and l follow the new reference. The
  // tile's scores are recomputed from K in global memory (rows clamped to Sk-1, masked anyway): by
  // the end of the step the raw scores are gone and the tile's LDS slot holds a later tile.
  __device__ __forceinline__ void rebase(Probs& pk, float (&rs)[QB], int n0, bool masked) {
    Scores cur;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      const int row = min(n0 + kb * 32 + perm32(i32), sk - 1);
      const uint16_t* krow;
      const uint8_t* krow8 = nullptr;
      bool there = true;
      if constexpr (C::PAGED) {
        const int page = this->table[row >> this->page_shift];
        there = page >= 0 && page < this->n_pages;
        const int64_t at = page * this->page_stride + (row & ((1 << this->page_shift) - 1)) * this->slot_stride;
        krow = kg + at + 8 * h;
        krow8 = reinterpret_cast<const uint8_t*>(kg) + at + 16 * h;
      } else {
        krow = kg + (size_t)row * DQK + 8 * h;
      }
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        u32x4 a = {0u, 0u, 0u, 0u};
        if constexpr (C::E4M3) {
          if (there) {
            const uint2 w = *reinterpret_cast<const uint2*>(krow8 + 32 * (ks / 2) + 8 * (ks & 1));
            a = bit_cast<u32x4>(widen_bf16(w.x, w.y));
          }
        } else if (!C::PAGED || there) {
          a = *reinterpret_cast<const u32x4*>(krow + 16 * ks);
        }
#pragma unroll
        for (int qb = 0; qb < QB; ++qb)
          cur[kb][qb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(bit_cast<bf16x8>(a), qf[qb][ks],
                                                                ks == 0 ? f32x16{} : cur[kb][qb], 0, 0, 0);
      }
    }
    if (masked) mask_tile(cur, n0);
    float mref[QB];
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
      const float m_new = fmaxf(m_run[qb], row_max(cur, qb));
      const float alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_run[qb] - m_new);
      m_run[qb] = m_new;
      l_run[qb] *= alpha;
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        agpr_fence<AG>(oacc[db][qb]);
        oacc[db][qb] *= alpha;
        agpr_fence<AG>(oacc[db][qb]);
      }
      mref[qb] = m_new == -INFINITY ? 0.f : m_new - C::P_LOG2;
    }
#pragma unroll
    for (int u = 0; u < NEP; ++u) {
      const float e0 = exp_elem(2 * u, cur, mref, cs), e1 = exp_elem(2 * u + 1, cur, mref, cs);
      pack_pair(u, e0, e1, pk, rs);
    }
  }

  // One pipeline step: P V of tile j-1 (pk_old, V slot sVo), exponentials of tile j (cur, key n0,
  // into pk_new) and scores of tile j+1 (K slot sKn, into nxt).
  // `issue(k)` starts load k (0 <= k < LOADS) of the tiles this step prefetches; the loads are spread
  // one every NSL / LOADS slots, between MFMAs (a burst of them would stall the wave).
  template <class Issue>
  __device__ __forceinline__ void step(Scores& cur, Scores& nxt, Probs& pk_new, const Probs& pk_old,
                                       const unsigned char* sKn, const unsigned char* sVo, bool masked, int n0,
                                       Issue&& issue) {
    float mul = cs, add[QB], alpha[QB];
    bool rescale = false;
    if constexpr (C::FORM != kFormNone) {
      // With forms the maximum is computed for every tile: rows may see their first key in any, and a bias makes maxima rise.
      // The reference follows where some row's has risen over it by more than 2^3 (in log2); O and the sums, which
      // hold the tiles before this one only after the step, follow at its end.
      __builtin_amdgcn_s_setprio(0);
      mul = this->values(cur, add, n0, masked, cs, h, *this);
      float mt[QB];
      bool up = false;
#pragma unroll
      for (int qb = 0; qb < QB; ++qb) {
        mt[qb] = row_max_of(cur, qb, mul, add[qb]);
        up = up || mt[qb] > m_run[qb] + 8.f;
        alpha[qb] = 1.f;
      }
      rescale = __builtin_amdgcn_ballot_w64(up) != 0;
      if (rescale) {
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) {
          const float m_new = fmaxf(m_run[qb], mt[qb]);
          alpha[qb] = __builtin_amdgcn_exp2f(m_run[qb] - (m_new == -INFINITY ? 0.f : m_new));
          m_run[qb] = m_new;
        }
      }
    } else {
      if (masked) mask_tile(cur, n0);
    }
    // The SIMD's other wave may be at its values meanwhile: the matrix instructions' wave goes first (a prompt with slopes, d = 64
    // 166 us -> 160, trees of 60 tokens 128 -> 125; capped prompts level).
    if constexpr (C::FORM != kFormNone) __builtin_amdgcn_s_setprio(1);
    float mref[QB], rs[QB];
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
      mref[qb] = m_run[qb] == -INFINITY ? 0.f : m_run[qb] - C::P_LOG2;
      if constexpr (C::FORM != kFormNone) mref[qb] -= add[qb];
      rs[qb] = 0.f;
    }
    // V fragments first: the step's first MFMAs are P V's, so with one wave per SIMD every LDS read in
    // front of them is latency the wave waits out (one head S16384 d64 112.4 -> 107.4 us, GPT-2 S2048
    // 15.9 -> 15.6 us against K first; level where other waves fill the wait).
    bf16x8 vf[NVF];
#pragma unroll
    for (int t = 0; t < VPF && t < NVF; ++t) vf[t] = vfrag(sVo, t / DB, t % DB);
    __builtin_amdgcn_sched_barrier(0);
    u32x4 kf[KB * KS];
    first_kfrags(kf, sKn);
    static_assert(at_most_two_elems_per_slot(), "ev holds the elements of two slots");
    float ev[4];  // exponentials in flight, element e in ev[e % 4]
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int sl = 0; sl < NSL; ++sl) {
      {
        constexpr int NLD = C::K_LOADS + C::V_LOADS, SP = NSL / NLD;
        static_assert(SP >= 1, "more loads than slots");
        if (sl % SP == SP / 2 && sl / SP < NLD) issue(sl / SP);
      }
      if (slot_is_score(sl))
        score_mfma(nxt, kf, sKn, sl - NMP);
      else
        pv_mfma(sl, pk_old, vf, sVo, true);
      __builtin_amdgcn_sched_barrier(0);  // the slot's MFMA is issued before its VALU work
      if (sl > 0) {
#pragma unroll
        for (int e = elem_begin(sl - 1); e < elem_end(sl - 1); ++e)
          if (e & 1) pack_pair(e >> 1, ev[(e - 1) % 4], ev[e % 4], pk_new, rs);
      }
#pragma unroll
      for (int e = elem_begin(sl); e < elem_end(sl); ++e) ev[e % 4] = exp_elem(e, cur, mref, mul);
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int e = elem_begin(NSL - 1); e < elem_end(NSL - 1); ++e)
      if (e & 1) pack_pair(e >> 1, ev[(e - 1) % 4], ev[e % 4], pk_new, rs);
    if constexpr (C::FORM != kFormNone) {
      if (rescale) {
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) {
          l_run[qb] *= alpha[qb];
#pragma unroll
          for (int db = 0; db < DB; ++db) {
            agpr_fence<AG>(oacc[db][qb]);
            oacc[db][qb] *= alpha[qb];
            agpr_fence<AG>(oacc[db][qb]);
          }
        }
      }
    } else {
      bool over = false;
#pragma unroll
      for (int qb = 0; qb < QB; ++qb) over = over || !(rs[qb] <= C::OVERFLOW_SUM);
      // Without pages that are not there a row that sees any key of its range sees the first, so it has a reference from
      // tile 0 on; with them it takes one as soon as a tile has a key for it.
      if constexpr (C::PAGED) {
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) over = over || (this->holes && m_run[qb] == -INFINITY);
      }
      if (__builtin_amdgcn_ballot_w64(over) != 0) rebase(pk_new, rs, n0, masked);
    }
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) l_run[qb] += rs[qb];
  }
};

}  // namespace
}  // namespace fa
