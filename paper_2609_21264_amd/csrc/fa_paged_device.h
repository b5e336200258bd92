// Device helpers of the paged kernels: the batch's arrays (lengths, token ranges, page numbers) are device
// data that the host has not seen, so what is read from them is clamped here to what the arrays and
// buffers hold. Internal; included by the kernel sources only.
#pragma once

#include <float.h>

#include "fa_internal.h"

namespace fa {
namespace {

// A wave-uniform load through the scalar cache of an array that the kernel does not write. (Behind an asm
// statement with a memory clobber the compiler would use a vector load.)
__device__ __forceinline__ int scalar_load(const int* p) {
  return *(const __attribute__((address_space(4))) int*)(uintptr_t)p;
}
__device__ __forceinline__ float scalar_load(const float* p) {
  return *(const __attribute__((address_space(4))) float*)(uintptr_t)p;
}

// A value that is the same for the whole wave, in a scalar register (some divisions and scans would leave it in a vector one).
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ float uniform(float x) { return __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(x))); }

// One sequence: its new tokens are the packed ones [q0, q_end), the last of its kv keys.
struct PagedSeq {
  int q0, q_end, n_q, kv;
  int pre;  // with forms: leading keys that all its tokens see
};
__device__ __forceinline__ PagedSeq make_seq(const PagedBatch& bt, int first, int last, int keys) {
  PagedSeq s;
  s.q0 = min(max(first, 0), bt.n_tokens);
  s.q_end = min(max(last, 0), bt.n_tokens);
  s.n_q = max(s.q_end - s.q0, 0);
  s.kv = min(max(keys, 0), bt.max_keys);
  s.pre = 0;
  return s;
}
// Sequence b, the same for the whole wave; and one sequence per lane.
__device__ __forceinline__ PagedSeq load_seq(const PagedBatch& bt, int b) {
  return make_seq(bt, scalar_load(bt.q_starts + b), scalar_load(bt.q_starts + b + 1), scalar_load(bt.kv_lens + b));
}
__device__ __forceinline__ PagedSeq load_seq_lane(const PagedBatch& bt, int b) {
  return make_seq(bt, bt.q_starts[b], bt.q_starts[b + 1], bt.kv_lens[b]);
}
// The same with a prefix, where the kernel has forms.
template <bool FORM>
__device__ __forceinline__ PagedSeq load_seq(const PagedParams& p, int b) {
  PagedSeq s = load_seq(p.bt, b);
  if (FORM && p.f.prefix_lens != nullptr) s.pre = min(max(scalar_load(p.f.prefix_lens + b), 0), s.kv);
  return s;
}
template <bool FORM>
__device__ __forceinline__ PagedSeq load_seq_lane(const PagedParams& p, int b) {
  PagedSeq s = load_seq_lane(p.bt, b);
  if (FORM && p.f.prefix_lens != nullptr) s.pre = min(max(p.f.prefix_lens[b], 0), s.kv);
  return s;
}

__device__ __forceinline__ PagedSeq seq_of_lane(const PagedSeq& s, int l) {
  return PagedSeq{__builtin_amdgcn_readlane(s.q0, l), __builtin_amdgcn_readlane(s.q_end, l),
                  __builtin_amdgcn_readlane(s.n_q, l), __builtin_amdgcn_readlane(s.kv, l), __builtin_amdgcn_readlane(s.pre, l)};
}

// Sums over the wave, and inclusive prefix sums, that stop at 2^32 - 1: whatever the batch's arrays hold, a prefix never
// comes before an earlier one.
__device__ __forceinline__ uint32_t add_sat(uint32_t a, uint32_t b) { return __builtin_elementwise_add_sat(a, b); }
// (Lane moves inside the vector instructions: exchanges through LDS would be 0.3 us a scan.)
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t add_moved(uint32_t x) {
  return add_sat(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, ROWS, 0xf, false));
}
__device__ __forceinline__ uint32_t wave_scan(uint32_t x) {
  x = add_moved<0x111, 0xf>(x);  // from 1, 2, 4 and 8 lanes before, within the rows of 16
  x = add_moved<0x112, 0xf>(x);
  x = add_moved<0x114, 0xf>(x);
  x = add_moved<0x118, 0xf>(x);
  x = add_moved<0x142, 0xa>(x);  // the last lane of rows 0 and 2 to rows 1 and 3
  x = add_moved<0x143, 0xc>(x);  // lane 31 to rows 2 and 3
  return x;
}
__device__ __forceinline__ uint32_t wave_sum(uint32_t x) {
  return (uint32_t)__builtin_amdgcn_readlane((int)wave_scan(x), 63);
}
__device__ __forceinline__ uint32_t lane_of(uint32_t x, int l) { return (uint32_t)__builtin_amdgcn_readlane((int)x, l); }

// The work of the sequences with more than few_cols row-heads per key/value head, as the kernel for few rows would have
// it: items of 64 row-heads, each 5 units and one per 128 keys that its rows see on average (one for the rest). Counted
// alike by both attention kernels. sl: the first 64 sequences, one per lane.
template <bool FORM>
__device__ __forceinline__ uint32_t big_work(const PagedParams& p, const PagedSeq& sl, int lane) {
  auto of = [&](const PagedSeq& s) {
    const int64_t cols = (int64_t)s.n_q * p.group;
    if (cols <= p.few_cols) return 0u;
    int64_t keys2 = 2 * (int64_t)s.kv - (p.causal ? min(s.n_q, s.kv) : 0);
    if (FORM && p.f.window != 0) keys2 = min(keys2, 2 * ((int64_t)p.f.window * (p.causal ? 1 : 2) + s.pre));
    const int64_t units = (cols + 63) / 64 * p.c.hkv * (6 + (keys2 >> 8));  // below 2^62: cols * hkv < 2^31 + 2^31
    return (uint32_t)min(units, (int64_t)UINT32_MAX);
  };
  uint32_t sum = of(sl);
  for (int c = 64 + lane; c < p.bt.n_seq; c += 64) sum = add_sat(sum, of(load_seq_lane<FORM>(p, c)));
  return wave_sum(sum);
}

// ---- forms: scores capped or biased, and which keys a token sees beyond causal masking ----------------
//
// The token at position pos sees key j where j < pre, or where j is inside its window (|pos - j| < window) and, when
// causal, j <= pos; with a tree of drafted tokens it sees the cached keys, and of the new ones those whose bits are set.

// Keys [0, end) from which rows row0 .. row1 of a sequence see any, in tiles of TILE keys without those that lie between
// the prefix and the first row's window: tile t of n is tile t of the keys for t < pre, else t + gap.
template <int TILE>
struct SeenTiles {
  int end, pre, gap, n;
  __device__ __forceinline__ SeenTiles(const PagedForms& f, const PagedSeq& s, int row0, int row1) {
    const int p0 = max(s.kv - s.n_q + row0, 0), p1 = max(s.kv - s.n_q + row1, -1), w = f.window;
    end = s.kv;
    if (f.mask == nullptr && (f.causal || w != 0)) end = max(min(s.kv, f.causal ? p1 + 1 : p1 + w), s.pre);
    n = (end + TILE - 1) / TILE;
    const int from = w != 0 ? min(max(p0 - w + 1, 0) / TILE, n) : 0, pre_tiles = (s.pre + TILE - 1) / TILE;
    gap = max(from - pre_tiles, 0);
    pre = gap > 0 ? pre_tiles : n;
    n -= gap;
  }
  __device__ __forceinline__ int tile(int t) const { return t < pre ? t : t + gap; }
  // How many of the tiles lie before tile t of the keys.
  __device__ __forceinline__ int before(int t) const { return t <= pre ? t : max(pre, t - gap); }
};

// What one row sees.
struct SeenRow {
  int pos;             // -2^30 at least
  int first, last;     // of its window
  const uint32_t* bits;
  __device__ __forceinline__ void init(const PagedForms& f, const PagedSeq& s, int row) {
    pos = max(s.kv - s.n_q + row, -(1 << 30));
    const int w = f.window;
    first = w != 0 ? pos - w + 1 : 0;
    last = min(f.causal ? pos : w != 0 ? pos + w - 1 : s.kv - 1, s.kv - 1);
    bits = nullptr;
    if (f.mask != nullptr) {
      last = min(s.kv - s.n_q, s.kv) - 1;
      bits = f.mask + (int64_t)(s.q0 + row) * f.mask_stride;
    }
  }
};
// The first k of 32 bits (none below 0, all from 32 on).
__device__ __forceinline__ uint32_t first_bits(int k) {
  return (uint32_t)(0xffffffffull >> (32 - min(max(k, 0), 32)));
}
// Bit i: whether the row sees key `base` + i (base the same for the whole wave).
__device__ __forceinline__ uint32_t seen_bits(const PagedForms& f, const PagedSeq& s, const SeenRow& r, int base) {
  uint32_t v = (first_bits(r.last + 1 - base) & ~first_bits(r.first - base)) | first_bits(s.pre - base);
  if (f.mask != nullptr) {
    const int o = base - (s.kv - s.n_q), words = f.mask_words;  // the new token that is key `base`
    if (o > -32 && o < 32 * words && base < s.kv) {
      const int w = o >> 5;
      const uint32_t lo = w >= 0 ? r.bits[w] : 0u, hi = w + 1 < words ? r.bits[w + 1] : 0u;
      v |= (uint32_t)((((uint64_t)hi << 32) | lo) >> (o & 31)) & first_bits(s.kv - base);
    }
  }
  return v;
}

// A bias by distance in units of log2. Beyond 2^96 it stays at that, so that it times a distance below 2^31 is finite: 0 times an
// infinity would be no number.
__device__ __forceinline__ float bounded_slope(float s) {
  constexpr float kMost = 0x1p96f;
  return s > kMost ? kMost : s < -kMost ? -kMost : s;
}

// A score in units of log2: cap * tanh(x / cap) = cap (1 - 2 / (1 + e^(2 x / cap))). Its error of 2^-23 cap log2(e), mostly of the
// last sum, is why caps end at 1024, where it moves a probability by less than its rounding to fp16 does.
// a: cap_a; b: cap_factor() of what takes raw scores to units of log2.
__device__ __forceinline__ float cap_factor(const PagedForms& f, float cs) {
  return fminf(fmaxf(cs * f.cap_r, -FLT_MAX), FLT_MAX);  // finite, so that a score of 0 stays 0
}
__device__ __forceinline__ float capped(float s, float a, float b) {
  return fmaf(-2.f * a, __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(b * s)), a);
}

}  // namespace
}  // namespace fa
