// Around the paged key/value cache (gfx950): the mask and positions of a tree of drafted tokens, closing up the
// tokens that a sequence keeps of its new ones, and copies of pages.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "fa.h"
#include "fa_fastdiv.h"
#include "fa_paged_device.h"

namespace fa {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// ---- tree of drafted tokens ------------------------------------------------------------------------------
//
// A token sees itself and its ancestors: bit j of its row says so of the j-th new token of its sequence. A workgroup per
// sequence, whose parents it keeps in LDS; a thread per token, which walks up its parents and, as their numbers only fall,
// writes its row's words from the last to the first as it passes them. A parent comes before its child; what is no such number
// (the root's -1 too) ends the walk. A chain of n tokens takes n / 2 steps a token, so a sequence of more than FA_TREE_TOKENS
// tokens is left out, where a walk could go on for long. Bound by the chain of launch, lengths, parents and walk: 26 or 64 x 60
// tokens 2.3 us.
constexpr int kTreeThreads = 256;

__global__ __launch_bounds__(kTreeThreads) void fa_tree_mask_kernel(TreeParams p) {
  __shared__ int parent[FA_TREE_TOKENS];
  // Unsigned: a step past the last sequence may lead behind 2^31.
  for (uint32_t b = blockIdx.x; b < (uint32_t)p.bt.n_seq; b += gridDim.x) {
    const PagedSeq s = load_seq(p.bt, (int)b);
    if (s.n_q > FA_TREE_TOKENS) continue;
    __syncthreads();  // the last sequence's walks are done
    for (int i = threadIdx.x; i < s.n_q; i += kTreeThreads) parent[i] = p.parents[s.q0 + i];
    __syncthreads();
    for (int i = threadIdx.x; i < s.n_q; i += kTreeThreads) {
      uint32_t* row = p.mask + (int64_t)(s.q0 + i) * p.mask_stride;
      int left = p.words, depth = -1;  // words from `left` on are written
      uint32_t bits = 0;
      auto down_to = [&](int w) {  // zeros in the words behind word w
        for (; left > w + 1; --left) row[left - 1] = 0;
      };
      int word = i >> 5;
      for (int at = i; at >= 0;) {
        if ((at >> 5) != word) {
          down_to(word);
          if (word < p.words) row[word] = bits, left = word;
          word = at >> 5, bits = 0;
        }
        bits |= 1u << (at & 31);
        ++depth;
        const int up = parent[at];
        at = up < at ? up : -1;
      }
      down_to(word);
      if (word < p.words) row[word] = bits, left = word;
      down_to(-1);
      p.positions[s.q0 + i] = s.kv - s.n_q + depth;
    }
  }
}

// ---- closing up ----------------------------------------------------------------------------------------
//
// Token kept[i] of a sequence's new ones moves to the i-th place behind its cached keys. A thread owns 16 bytes of
// a head of K or V and takes them from place to place in order, up to kMoves at a time whose loads are in flight together: as
// the numbers kept increase, no place is written before it has been read. Bound by the bytes moved and the chain
// lengths -> kept -> pages -> load -> store: 64 sequences' tokens in 32 layers of 8 heads 17 us, 4.1 TB/s (e4m3 10 us, 3.5).
constexpr int kMoveThreads = 256, kMoves = 8;

__global__ __launch_bounds__(kMoveThreads) void fa_kv_compact_kernel(CompactParams p) {
  const int b = (int)blockIdx.y + (int)blockIdx.z * kMoveRows;
  if (b >= p.bt.n_seq) return;
  const PagedSeq s = load_seq(p.bt, b);
  const int n = min(min(max(scalar_load(p.n_kept + b), 0), p.max_kept), s.n_q);
  const int base = s.kv - s.n_q;  // may be negative: places before the first key are none
  if (blockIdx.x == 0 && threadIdx.x == 0) p.lens_out[b] = max(base + n, 0);
  // Chunk of this thread: those of K first.
  uint32_t c = blockIdx.x * kMoveThreads + threadIdx.x;
  const uint32_t n_k = (uint32_t)p.c.hkv * p.k_chunks, n_all = n_k + (uint32_t)p.c.hkv * p.v_chunks;
  if (c >= n_all) return;
  const bool is_v = c >= n_k;
  c -= is_v ? n_k : 0u;
  const uint32_t head = is_v ? fast_div(c, p.m_v, p.sh_v) : fast_div(c, p.m_k, p.sh_k);
  const uint32_t ch = c - head * (is_v ? p.v_chunks : p.k_chunks);
  unsigned char* const at = static_cast<unsigned char*>(is_v ? p.c.v : p.c.k) +
                            (int64_t)head * (is_v ? p.c.v_head : p.c.k_head) * p.elem + ch * 16u;
  const int64_t page_bytes = (is_v ? p.c.v_page : p.c.k_page) * p.elem, slot_bytes = (is_v ? p.c.v_slot : p.c.k_slot) * p.elem;
  const int* table = p.bt.block_table + b * p.bt.table_stride;
  const int* kept = p.kept + b * p.kept_stride;
  const int smask = (1 << p.c.page_shift) - 1;
  // Address of a key's chunk; nullptr where the key or its page is not there.
  auto place = [&](int key) -> unsigned char* {
    if (key < 0 || key >= s.kv) return nullptr;
    const int page = scalar_load(table + (key >> p.c.page_shift));
    if (page < 0 || page >= p.c.n_pages) return nullptr;
    return at + page * page_bytes + (key & smask) * slot_bytes;
  };
  for (int i0 = 0; i0 < n; i0 += kMoves) {
    u32x4 x[kMoves];
    unsigned char* to[kMoves];
#pragma unroll
    for (int i = 0; i < kMoves; ++i) {
      to[i] = nullptr;
      if (i0 + i >= n) continue;
      const int k = scalar_load(kept + i0 + i);
      if (k < 0 || k >= s.n_q || k == i0 + i) continue;
      const unsigned char* from = place(base + k);
      if (from == nullptr) continue;
      to[i] = place(base + i0 + i);
      x[i] = *reinterpret_cast<const u32x4*>(from);
    }
#pragma unroll
    for (int i = 0; i < kMoves; ++i)
      if (to[i] != nullptr) *reinterpret_cast<u32x4*>(to[i]) = x[i];
  }
}

// ---- copies of pages -------------------------------------------------------------------------------------
//
// Page src[i] goes to page dst[i]. A workgroup moves 256 chunks of 16 bytes of one page's K or V, past the caches. Runs of chunks
// that lie one after the other in memory are found by the host (a page whose heads and slots follow each other is
// one). Bound by the bytes: copies of 500 pages of 2 x 1 MiB 366 to 372 us, 5.6 to 5.7 TB/s read and written (e4m3, half the bytes, 186).
// On a box where that took 355: with 2, 4, 8 or 16 chunks a thread 383 to 392, through the caches 387 (one chunk) to 411.

__global__ __launch_bounds__(kMoveThreads) void fa_kv_copy_kernel(CopyParams p) {
  const CopySide& c = p.side[blockIdx.y];
  const uint32_t pair = fast_div(blockIdx.x, p.m_parts, p.sh_parts), part = blockIdx.x - pair * p.parts;
  const int src = scalar_load(p.src + pair), dst = scalar_load(p.dst + pair);
  if (src < 0 || src >= p.n_pages || dst < 0 || dst >= p.n_pages || src == dst) return;
  const uint32_t k = part * kMoveThreads + threadIdx.x;
  if (k >= c.chunks) return;
  const uint32_t row = fast_div(k, c.m_run, c.sh_run), head = fast_div(row, c.m_rows, c.sh_rows);
  const int64_t at = head * c.head + (row - head * c.rows) * c.row + (int64_t)(k - row * c.run) * 16;
  const u32x4 x = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(c.base + src * c.page + at));
  __builtin_nontemporal_store(x, reinterpret_cast<u32x4*>(c.base + dst * c.page + at));
}

CopySide copy_side(void* base, int64_t page, int64_t head, int64_t slot, int heads, int slots, int d, int elem) {
  CopySide s{};
  s.base = static_cast<unsigned char*>(base);
  s.page = page * elem;
  // Heads of rows of runs; what follows without a gap joins the run.
  int64_t run = (int64_t)d * elem, rows = slots, row = slot * elem, n = heads, step = head * elem;
  if (rows == 1 || row == run) run *= rows, rows = n, row = step, n = 1, step = 0;
  if (n == 1 && (rows == 1 || row == run)) run *= rows, rows = 1, row = 0;
  s.head = step, s.row = row;
  s.rows = (uint32_t)rows, s.run = (uint32_t)(run / 16);
  s.chunks = (uint32_t)(n * rows * (run / 16));
  const FastDiv a = make_fastdiv(s.run), b = make_fastdiv(s.rows);
  s.m_run = a.m, s.sh_run = a.sh, s.m_rows = b.m, s.sh_rows = b.sh;
  return s;
}

}  // namespace

hipError_t launch_tree_mask(TreeParams p, hipStream_t stream) {
  void* args[] = {&p};
  constexpr int kMost = 1 << 20;
  return hipLaunchKernel(reinterpret_cast<const void*>(&fa_tree_mask_kernel), dim3(p.bt.n_seq < kMost ? p.bt.n_seq : kMost),
                         dim3(kTreeThreads), args, 0, stream);
}

int64_t kv_compact_blocks(int hkv, int d_qk, int d_v, int elem) {
  const int64_t chunks = (int64_t)hkv * ((d_qk + d_v) * elem / 16);  // of 16 bytes; below 2^31 by the host's check
  return chunks == 0 ? 1 : (chunks + kMoveThreads - 1) / kMoveThreads;
}

hipError_t launch_kv_compact(CompactParams p, hipStream_t stream) {
  p.k_chunks = (uint32_t)(p.c.d_qk * p.elem / 16), p.v_chunks = (uint32_t)(p.c.d_v * p.elem / 16);
  const FastDiv k = make_fastdiv(p.k_chunks), v = make_fastdiv(p.v_chunks);
  p.m_k = k.m, p.sh_k = k.sh, p.m_v = v.m, p.sh_v = v.sh;
  const int n = p.bt.n_seq;  // below 2^24, with the grid's first dimension
  const dim3 grid((unsigned)kv_compact_blocks(p.c.hkv, p.c.d_qk, p.c.d_v, p.elem), (unsigned)(n < kMoveRows ? n : kMoveRows),
                  (unsigned)((n + kMoveRows - 1) / kMoveRows));
  void* args[] = {&p};
  return hipLaunchKernel(reinterpret_cast<const void*>(&fa_kv_compact_kernel), grid, dim3(kMoveThreads), args, 0, stream);
}

int64_t kv_copy_blocks(const PagedCache& c, int elem, int n) {
  const int64_t most = (int64_t)c.hkv * (1 << c.page_shift) * (c.d_qk > c.d_v ? c.d_qk : c.d_v) * elem / 16;
  if (most > INT32_MAX) return -1;
  return (most + kMoveThreads - 1) / kMoveThreads * n;
}

hipError_t launch_kv_copy(const PagedCache& c, int elem, const int* src, const int* dst, int n, hipStream_t stream) {
  CopyParams p{};
  const int slots = 1 << c.page_shift;
  p.side[0] = copy_side(c.k, c.k_page, c.k_head, c.k_slot, c.hkv, slots, c.d_qk, elem);
  p.side[1] = copy_side(c.v, c.v_page, c.v_head, c.v_slot, c.hkv, slots, c.d_v, elem);
  p.src = src, p.dst = dst, p.n_pages = c.n_pages;
  const int64_t blocks = kv_copy_blocks(c, elem, n);
  p.parts = (uint32_t)(blocks / n);
  const FastDiv f = make_fastdiv(p.parts);
  p.m_parts = f.m, p.sh_parts = f.sh;
  void* args[] = {&p};
  return hipLaunchKernel(reinterpret_cast<const void*>(&fa_kv_copy_kernel), dim3((unsigned)blocks, 2), dim3(kMoveThreads), args,
                         0, stream);
}

}  // namespace fa
