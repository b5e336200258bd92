// Device helpers of the paged kernels: the batch's arrays (lengths, token ranges, page numbers) are device
// data that the host has not seen, so what is read from them is clamped here to what the arrays and
// buffers hold. Internal; included by the kernel sources only.
#pragma once

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

// One sequence: its new tokens are the packed ones [q0, q_end), the last of its kv keys.
struct PagedSeq {
  int q0, q_end, n_q, kv;
};
__device__ __forceinline__ PagedSeq make_seq(const PagedBatch& bt, int first, int last, int keys) {
  PagedSeq s;
  s.q0 = min(max(first, 0), bt.n_tokens);
  s.q_end = min(max(last, 0), bt.n_tokens);
  s.n_q = max(s.q_end - s.q0, 0);
  s.kv = min(max(keys, 0), bt.max_keys);
  return s;
}
// Sequence b, the same for the whole wave; and one sequence per lane.
__device__ __forceinline__ PagedSeq load_seq(const PagedBatch& bt, int b) {
  return make_seq(bt, scalar_load(bt.q_starts + b), scalar_load(bt.q_starts + b + 1), scalar_load(bt.kv_lens + b));
}
__device__ __forceinline__ PagedSeq load_seq_lane(const PagedBatch& bt, int b) {
  return make_seq(bt, bt.q_starts[b], bt.q_starts[b + 1], bt.kv_lens[b]);
}

__device__ __forceinline__ PagedSeq seq_of_lane(const PagedSeq& s, int l) {
  return PagedSeq{__builtin_amdgcn_readlane(s.q0, l), __builtin_amdgcn_readlane(s.q_end, l),
                  __builtin_amdgcn_readlane(s.n_q, l), __builtin_amdgcn_readlane(s.kv, l)};
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
__device__ __forceinline__ uint32_t big_work(const PagedParams& p, const PagedSeq& sl, int lane) {
  auto of = [&](const PagedSeq& s) {
    const int64_t cols = (int64_t)s.n_q * p.group;
    if (cols <= p.few_cols) return 0u;
    const int64_t keys2 = 2 * (int64_t)s.kv - (p.causal ? min(s.n_q, s.kv) : 0);
    const int64_t units = (cols + 63) / 64 * p.c.hkv * (6 + (keys2 >> 8));  // below 2^62: cols * hkv < 2^31 + 2^31
    return (uint32_t)min(units, (int64_t)UINT32_MAX);
  };
  uint32_t sum = of(sl);
  for (int c = 64 + lane; c < p.bt.n_seq; c += 64) sum = add_sat(sum, of(load_seq_lane(p.bt, c)));
  return wave_sum(sum);
}

}  // namespace
}  // namespace fa
