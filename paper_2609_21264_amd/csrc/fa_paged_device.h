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

}  // namespace
}  // namespace fa
