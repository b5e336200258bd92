// C ABI of the attention forward (declared in include/fa.h): host-side argument checks, then kernel
// launches on the caller's stream (fused forward, split mode, decode-shaped path, layer-by-layer
// operators). No allocation and no synchronisation; the only state is the per-device address of the
// static scratch array of fa_fwd_decode_noalloc.
#include <float.h>
#include <limits.h>
#include <math.h>
#include <stdint.h>

#include <atomic>
#include <mutex>

#include "fa.h"
#include "fa_internal.h"

// Static scratch of the allocation-free decode entry point: fa_fwd_decode_noalloc keeps its partial
// results in this file-scope device array instead of a caller workspace. Every device the library
// runs on holds its own copy (allocated with the code object, kept until the process ends). On the
// host, `scratch` names a host-side stand-in, not a device address: the device address is looked up
// once per device with hipGetSymbolAddress (with that device current, scratch_for_stream below) and
// only that address is passed to kernels.
static __device__ __align__(256) unsigned char scratch[FA_NOALLOC_SCRATCH_BYTES];

namespace {

bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

// Bytes of the split-mode workspace: partial O (fp32, d_v per row) and LSE (fp32) for every row and
// part; -1 if the count overflows.
int64_t split_workspace_bytes(int B, int Hq, int Sq, int d_v, int n_split) {
  if (B <= 0 || Hq <= 0 || Sq <= 0 || d_v <= 0 || n_split <= 0) return 0;
  const int64_t bh = static_cast<int64_t>(B) * Hq;  // < 2^62
  const int64_t per_row = (static_cast<int64_t>(d_v) + 1) * 4 * n_split;  // < 2^44
  if (bh > INT64_MAX / Sq) return -1;
  const int64_t rows = bh * Sq;
  if (rows > INT64_MAX / per_row) return -1;
  return rows * per_row;
}

// Checks shared by the fused entry points (fa_fwd_ex, fa_fwd_split, fa_fwd_decode and
// fa_fwd_decode_noalloc), in the order fa.h documents: sizes, head dimensions, pointers, scale,
// alignment, index ranges. On FA_OK, *cs holds scale * log2(e) as the kernels take it (magnitude at
// least FLT_MIN, so that a masked score stays infinite; negative when scale < 0).
fa_status_t check_fused(const void* Q, const void* K, const void* V, const void* O, const float* LSE, int B, int Hq,
                        int Hkv, int Sq, int Sk, int d_qk, int d_v, float scale, int causal, float* cs) {
  if (B < 0 || Hq < 0 || Hkv < 0 || Sq < 0 || Sk < 0) return FA_ERR_BAD_SHAPE;
  if (Hq > 0 && (Hkv <= 0 || Hq % Hkv != 0)) return FA_ERR_BAD_SHAPE;
  if (fa::block_rows(d_qk, d_v, causal != 0) == 0) return FA_ERR_UNSUPPORTED;
  // A pointer may be NULL only when the array it addresses has no element.
  const bool q_rows = static_cast<int64_t>(B) * Hq * Sq > 0;
  const bool kv_rows = static_cast<int64_t>(B) * Hkv * Sk > 0;
  if ((q_rows && (Q == nullptr || O == nullptr)) || (kv_rows && (K == nullptr || V == nullptr)))
    return FA_ERR_NULL_POINTER;
  if (!isfinite(scale)) return FA_ERR_BAD_SCALE;
  const double c = fabs(static_cast<double>(scale)) * 1.4426950408889634074;  // |scale| * log2(e)
  if (c > FLT_MAX) return FA_ERR_BAD_SCALE;
  if (!aligned(Q, 16) || !aligned(K, 16) || !aligned(V, 16) || !aligned(O, 16) || !aligned(LSE, 4))
    return FA_ERR_UNSUPPORTED;
  // Offsets inside one head are 32-bit in the kernels.
  const int64_t dmax = d_qk > d_v ? d_qk : d_v;
  if (static_cast<int64_t>(Sq) * dmax > INT_MAX || static_cast<int64_t>(Sk) * dmax > INT_MAX) return FA_ERR_BAD_SHAPE;
  const float cmag = c < FLT_MIN ? FLT_MIN : static_cast<float>(c);
  *cs = scale < 0.f ? -cmag : cmag;
  return FA_OK;
}

fa_status_t forward(const void* Q, const void* K, const void* V, void* O, float* LSE, int B, int Hq, int Hkv,
                    int Sq, int Sk, int d_qk, int d_v, float scale, int causal, hipStream_t stream, int n_split = 0,
                    void* workspace = nullptr, size_t workspace_bytes = 0) {
  float cs = 0.f;
  const fa_status_t st = check_fused(Q, K, V, O, LSE, B, Hq, Hkv, Sq, Sk, d_qk, d_v, scale, causal, &cs);
  if (st != FA_OK) return st;
  if (B == 0 || Hq == 0 || Sq == 0) return FA_OK;
  const int64_t n_wg = fa::forward_workgroups(B, Hq, Hkv, Sq);
  if (n_wg > INT_MAX || static_cast<int64_t>(B) * Hq > INT_MAX || static_cast<int64_t>(B) * Hkv > INT_MAX)
    return FA_ERR_BAD_SHAPE;
  if (n_split > 0) {
    if (n_wg * n_split > INT_MAX) return FA_ERR_BAD_SHAPE;
    if (static_cast<int64_t>(B) * Hq * Sq > INT_MAX) return FA_ERR_BAD_SHAPE;  // merge: a workgroup per row at most
    const int64_t need = split_workspace_bytes(B, Hq, Sq, d_v, n_split);
    if (need < 0 || workspace == nullptr || static_cast<uint64_t>(need) > workspace_bytes) return FA_ERR_WORKSPACE;
    if (!aligned(workspace, 16)) return FA_ERR_UNSUPPORTED;
  }

  fa::FwdParams p{};
  p.q = static_cast<const uint16_t*>(Q);
  p.k = static_cast<const uint16_t*>(K);
  p.v = static_cast<const uint16_t*>(V);
  p.o = static_cast<uint16_t*>(O);
  p.lse = LSE;
  p.batch = B;
  p.hq = Hq;
  p.hkv = Hkv;
  p.sq = Sq;
  p.sk = Sk;
  p.group = Hq / Hkv;
  p.cs = cs;
  hipError_t err;
  if (n_split > 0) {
    const int64_t rows = static_cast<int64_t>(B) * Hq * Sq;
    p.n_split = n_split;
    p.o_part = static_cast<float*>(workspace);
    p.lse_part = p.o_part + rows * n_split * d_v;
    err = fa::launch_forward_split(p, d_qk, d_v, causal != 0, stream);
  } else {
    err = fa::launch_forward(p, d_qk, d_v, causal != 0, stream);
  }
  return err == hipSuccess ? FA_OK : FA_ERR_HIP;
}

// Grid checks of the decode-shaped path (after check_fused and the degenerate sizes), and the bytes of
// partial results it stores (-1 if the count overflows).
fa_status_t decode_grid(int B, int Hq, int Hkv, int Sq, int d_v, int n_parts, int64_t* need) {
  const int64_t n_cb = (static_cast<int64_t>(Hq / Hkv) * Sq + 31) / 32;
  if (static_cast<int64_t>(B) * Hkv * n_cb * n_parts > INT_MAX || static_cast<int64_t>(B) * Hq * Sq > INT_MAX)
    return FA_ERR_BAD_SHAPE;
  *need = split_workspace_bytes(B, Hq, Sq, d_v, n_parts);
  return FA_OK;
}

hipError_t decode_launch(const void* Q, const void* K, const void* V, void* O, float* LSE, int B, int Hq, int Hkv,
                         int Sq, int Sk, int d_qk, int d_v, float cs, int causal, int n_parts, void* ws,
                         hipStream_t stream) {
  fa::DecodeParams p{};
  p.q = static_cast<const uint16_t*>(Q);
  p.k = static_cast<const uint16_t*>(K);
  p.v = static_cast<const uint16_t*>(V);
  p.o = static_cast<uint16_t*>(O);
  p.lse = LSE;
  p.batch = B;
  p.hq = Hq;
  p.hkv = Hkv;
  p.sq = Sq;
  p.sk = Sk;
  p.group = Hq / Hkv;
  p.causal = causal != 0;
  p.cs = cs;
  p.rows = p.group * Sq;
  p.n_parts = n_parts;
  const int64_t rows = static_cast<int64_t>(B) * Hq * Sq;
  p.o_part = static_cast<float*>(ws);
  p.lse_part = p.o_part + rows * n_parts * d_v;
  return fa::launch_decode(p, d_qk, d_v, stream);
}

// ---- per-device address of the static scratch (declared at the top of the file) -------------------

constexpr int kMaxDevices = 64;
std::atomic<void*> g_scratch[kMaxDevices];
std::mutex g_scratch_mu;

// Device address of `scratch` on the device `stream` belongs to (the current device for the null
// stream). The first call on a device looks it up; later calls read the cached address.
hipError_t scratch_for_stream(hipStream_t stream, void** out) {
  int cur = 0;
  hipError_t e = hipGetDevice(&cur);
  if (e != hipSuccess) return e;
  int dev = cur;
  if (stream != nullptr) {
    e = hipStreamGetDevice(stream, &dev);
    if (e != hipSuccess) return e;
  }
  if (dev < 0 || dev >= kMaxDevices) return hipErrorInvalidDevice;
  void* ptr = g_scratch[dev].load(std::memory_order_acquire);
  if (ptr != nullptr) {
    *out = ptr;
    return hipSuccess;
  }
  std::lock_guard<std::mutex> lock(g_scratch_mu);
  ptr = g_scratch[dev].load(std::memory_order_relaxed);
  if (ptr == nullptr) {
    if (dev != cur && (e = hipSetDevice(dev)) != hipSuccess) return e;
    e = hipGetSymbolAddress(&ptr, HIP_SYMBOL(scratch));
    if (dev != cur) {
      const hipError_t e2 = hipSetDevice(cur);
      if (e == hipSuccess) e = e2;
    }
    if (e != hipSuccess || ptr == nullptr) return e != hipSuccess ? e : hipErrorInvalidSymbol;
    g_scratch[dev].store(ptr, std::memory_order_release);
  }
  *out = ptr;
  return hipSuccess;
}

// ---- layer-by-layer operators ------------------------------------------------------------------

int64_t lbl_ld(int Sk) { return (static_cast<int64_t>(Sk) + fa::kLblKeys - 1) / fa::kLblKeys * fa::kLblKeys; }

// Shared checks of the layer-by-layer entry points, in the order documented in fa.h. d_qk / d_v are
// checked only where the operator uses them (0 = unused).
fa_status_t lbl_check_shape(int B, int Hq, int Hkv, int Sq, int Sk, int d_qk, int d_v) {
  if (B < 0 || Hq < 0 || Hkv < 0 || Sq < 0 || Sk < 0) return FA_ERR_BAD_SHAPE;
  if (Hq > 0 && (Hkv <= 0 || Hq % Hkv != 0)) return FA_ERR_BAD_SHAPE;
  if (Sk > fa::kLblMaxSk) return FA_ERR_BAD_SHAPE;
  const int64_t dmax = d_qk > d_v ? d_qk : d_v;
  if (static_cast<int64_t>(Sq) * dmax > INT_MAX || static_cast<int64_t>(Sk) * dmax > INT_MAX) return FA_ERR_BAD_SHAPE;
  const int64_t n_qb = (static_cast<int64_t>(Sq) + fa::kLblRows - 1) / fa::kLblRows;
  if (static_cast<int64_t>(B) * Hq * n_qb > INT_MAX) return FA_ERR_BAD_SHAPE;
  if (static_cast<int64_t>(B) * Hq * Sq > 4 * static_cast<int64_t>(INT_MAX)) return FA_ERR_BAD_SHAPE;
  if (static_cast<int64_t>(B) * Hkv > INT_MAX) return FA_ERR_BAD_SHAPE;
  if (d_qk != 0 && !fa::lbl_scores_supported(d_qk)) return FA_ERR_UNSUPPORTED;
  if (d_v != 0 && !fa::lbl_pv_supported(d_v)) return FA_ERR_UNSUPPORTED;
  return FA_OK;
}

// The whole problem as one chunk; spill buffers S and P.
fa::LblParams lbl_params(int B, int Hq, int Hkv, int Sq, int Sk, float scale, int causal) {
  fa::LblParams p{};
  p.batch = B;
  p.hq = Hq;
  p.hkv = Hkv;
  p.sq = Sq;
  p.sk = Sk;
  p.group = Hkv > 0 ? Hq / Hkv : 1;
  p.causal = causal != 0;
  p.ld = static_cast<int>(lbl_ld(Sk));
  p.scale = scale;
  p.bh0 = 0;
  p.nbh = B * Hq;
  p.qb0 = 0;
  p.nqb = (Sq + fa::kLblRows - 1) / fa::kLblRows;
  p.xgroup = p.group;
  p.rows = static_cast<int64_t>(B) * Hq * Sq;
  return p;
}

// ---- paged cache ---------------------------------------------------------------------------------

bool dims_supported(int d_qk, int d_v) { return fa::block_rows(d_qk, d_v, true) != 0; }

// Keys of one sequence: the kernels count keys in 32 bits, some tiles past the last.
constexpr int64_t kMaxPagedKeys = 1 << 30;

// Checks that both paged entry points begin with, in the order fa.h documents: sizes, then what is supported. Hq may be
// 0 (no queries). On FA_OK fills the kernels' view of the cache and the batch.
fa_status_t check_paged_shape(const fa_paged_cache_t* c, const fa_paged_batch_t* bt, int Hq) {
  if (bt->B < 0 || bt->T < 0 || bt->max_blocks < 0 || c->n_pages < 0 || c->page_size < 0 || c->Hkv < 0 || Hq < 0)
    return FA_ERR_BAD_SHAPE;
  if ((bt->T > 0 || Hq > 0) && (c->Hkv <= 0 || Hq % c->Hkv != 0)) return FA_ERR_BAD_SHAPE;
  if (bt->table_stride < 0 || static_cast<int64_t>(bt->max_blocks) * c->page_size > kMaxPagedKeys) return FA_ERR_BAD_SHAPE;
  const int64_t heads = Hq > c->Hkv ? Hq : c->Hkv;
  if (static_cast<int64_t>(bt->T) * heads > INT_MAX || bt->B == INT_MAX) return FA_ERR_BAD_SHAPE;
  return FA_OK;
}
fa_status_t check_paged_support(const fa_paged_cache_t* c) {
  if (!dims_supported(c->d_qk, c->d_v)) return FA_ERR_UNSUPPORTED;
  if (c->page_size < 16 || c->page_size > (1 << 20) || (c->page_size & (c->page_size - 1)) != 0) return FA_ERR_UNSUPPORTED;
  if (c->type != FA_CACHE_BF16 && c->type != FA_CACHE_E4M3) return FA_ERR_UNSUPPORTED;
  if (c->type == FA_CACHE_BF16 && (c->k_scale != nullptr || c->v_scale != nullptr)) return FA_ERR_UNSUPPORTED;
  return FA_OK;
}
bool paged_pointers(const fa_paged_cache_t* c, const fa_paged_batch_t* bt) {
  if (bt->kv_lens == nullptr || bt->q_starts == nullptr) return false;
  if (bt->max_blocks > 0 && bt->block_table == nullptr) return false;
  return c->n_pages == 0 || c->Hkv == 0 || (c->K != nullptr && c->V != nullptr);
}
bool paged_aligned(const fa_paged_cache_t* c, const fa_paged_batch_t* bt) {
  const long long m = c->type == FA_CACHE_E4M3 ? 15 : 7;  // elements of 16 bytes, less one
  return aligned(c->K, 16) && aligned(c->V, 16) && aligned(c->k_scale, 4) && aligned(c->v_scale, 4) &&
         aligned(bt->block_table, 4) && aligned(bt->kv_lens, 4) && aligned(bt->q_starts, 4) &&
         ((c->k_page | c->k_head | c->k_slot | c->v_page | c->v_head | c->v_slot) & m) == 0;
}
// Strides of K or V: not negative, slots apart by a row at least and close enough for the kernels' 32-bit offsets,
// the whole buffer addressable; `writes`: no element has two places in the index space.
bool paged_strides(long long page, long long head, long long slot, const fa_paged_cache_t* c, int d, bool writes) {
  const int64_t size = c->type == FA_CACHE_E4M3 ? 1 : 2;
  if (page < 0 || head < 0 || slot < d || slot > INT_MAX / (16 * size)) return false;
  const long long st[3] = {page, head, slot};
  const int64_t n[3] = {c->n_pages, c->Hkv, c->page_size};
  double last = d;
  for (int i = 0; i < 3; ++i)
    if (n[i] > 1) last += static_cast<double>(n[i] - 1) * static_cast<double>(st[i]);
  if (last * static_cast<double>(size) >= 1e15) return false;
  if (!writes) return true;
  // Innermost first: every dimension has to step over all that the smaller strides reach.
  bool done[3] = {false, false, false};
  int64_t reach = d;
  for (int k = 0; k < 3; ++k) {
    int at = -1;
    for (int i = 0; i < 3; ++i)
      if (!done[i] && n[i] > 1 && (at < 0 || st[i] < st[at])) at = i;
    if (at < 0) break;
    if (st[at] < reach) return false;
    reach += (n[at] - 1) * st[at];
    done[at] = true;
  }
  return true;
}
fa_status_t check_paged_strides(const fa_paged_cache_t* c, bool writes) {
  return paged_strides(c->k_page, c->k_head, c->k_slot, c, c->d_qk, writes) &&
                 paged_strides(c->v_page, c->v_head, c->v_slot, c, c->d_v, writes)
             ? FA_OK
             : FA_ERR_BAD_SHAPE;
}
void paged_view(const fa_paged_cache_t* c, const fa_paged_batch_t* bt, fa::PagedCache* v, fa::PagedBatch* w) {
  int shift = 0;
  while ((1 << shift) < c->page_size) ++shift;
  *v = fa::PagedCache{c->K,      c->V,      c->k_scale, c->v_scale, c->k_page, c->k_head, c->k_slot, c->v_page,
                      c->v_head, c->v_slot, c->n_pages, shift,      c->Hkv,    c->d_qk,   c->d_v};
  *w = fa::PagedBatch{bt->block_table, bt->kv_lens, bt->q_starts, bt->table_stride,
                      bt->B,           bt->T,       bt->max_blocks * c->page_size};
}
// Element strides of a packed input or output: multiples of 16 bytes, offsets within 64 bits.
bool token_strides(const long long* s, int n) {
  for (int i = 0; i < n; ++i)
    if (s[i] < 0 || (s[i] & 7) != 0 || s[i] > (1ll << 40)) return false;
  return true;
}
// What a call of fa_fwd_paged runs, and its workspace (sizes checked).
//  By path, or (FA_PAGED_AUTO) thus:
//  * The kernel for few rows reads K and V once per item of 32 or 64 row-heads of a key/value head, and starts fast; the
//    kernel for many rows computes at three times its rate, and takes some 10 us more to start. The former runs alone where
//    the host expects no sequence with more than 64 row-heads, or where the table holds too few keys for kManyUnits units
//    of work (items of 64 row-heads, 5 units each and one per 128 keys); the latter where no sequence can have as few as 64
//    row-heads if none has more than max_q tokens, and where even without cached keys they have kSureUnits (prompts of 4 096
//    and 3 001 tokens, 32/8 heads, d = 128: 200 us alone, 206 with the others' launches; 2 000 and 1 500: 61.5 against 65.5). Else both are launched and find from the lengths whether the sequences with more than
//    32 row-heads have kManyUnits together: if so the kernel for many rows takes these, else that for few takes all.
//    A call without max_q (0) is planned as if every other sequence had one token: mostly the lengths then decide. (The
//    mean in its place would be taken for a bound: 4 096 + 255 x 1 tokens, 2 heads a group, d = 128, ran in the kernel for few
//    rows alone, 440 us against 195. Where all tokens in one sequence would have fewer than kManyUnits, few alone: 16 x 9 over 2 000
//    keys, 32/8 heads, 37 us, launched with the other kernel 51.)
//    Few against many, us, one box (units): d = 128 32/8 heads 512 x 512 (1.8 K) 17.1 : 20.1, 128 x 2000 (1.3 K) 30.5 : 44.2,
//    4 x 200 x 200 (2.5 K) 22.6 : 16.9, 700 x 700 (2.8 K) 39.9 : 23.4, 4 x 128 x 2000 (5.4 K) 50.4 : 48.6, 300 x 4000 (5.5 K)
//    60.7 : 45.4; d = 64 16/16 4 x 128 x 2000 (2.7 K) 26.5 : 31.9, 300 x 4000 (2.9 K) 35.2 : 29.5, 4 x 512 x 512 (4.1 K)
//    16.7 : 16.0, 16 x 200 x 200 (6.1 K) 20.7 : 13.3; d_qk = 192 16/16 1024 x 1024 (2.6 K) 32.0 : 43.2, 300 x 4000 (2.9 K)
//    72.4 : 47.0, 4 x 512 x 512 (4.1 K) 39.7 : 33.8; e4m3 d = 128 32/8 512 x 512 17.2 : 26.9, 700 x 700 40.0 : 30.7.
//    The thresholds are the same for all head dimensions and types, and so are off for some. Where most (the better kernel :
//    what runs): d = 64 16/16 16 x 100 x 100 9.4 : 15.0, 700 x 700 15.8 : 20.8, 4 x 128 x 2000 26.5 : 35.0; d_qk = 192 16/16
//    1024 x 1024 32.0 : 43.3, 4 x 128 x 2000 44.7 : 61.5; e4m3 32/8 d = 128 4 x 128 x 2000 45.4 : 68.6; e4m3 14/2 d = 64
//    4 x 400 x 400 13.8 : 19.9, 4 x 512 x 512 14.3 : 21.2. A caller who knows better names the path.
//  * Items of 64 where sequences have more than 32 row-heads, so that K and V are read half as often (8 x 35 row-heads x 3 001
//    keys 13.4 us against 15.7), except where items of 32 are no more than the CUs and the keys few, or read several
//    times anyway (40 tokens x 40 keys of one sequence, 32/8 heads: 7.2 us in items of 32, 9.6 of 64; 16 of 128 x 128
//    56.0 and 42.7).
//  * Where the table has pages for at most kWholeKeys keys, the kernel for few rows takes whole items, without a join
//    (one token, 32/8 heads, 512 keys 9.9 us against 11.0 with the join; 1 000 keys 15.0 against 11.2).
constexpr int kFewCols = 64;
constexpr uint32_t kManyUnits = 2750, kSureUnits = 2000;
constexpr int kWholeKeys = 512, kWholeItems = 1 << 16;
// Whether the kernel for many rows may be launched: it has a workgroup of 256 threads per block, whole ones of 128 row-heads and
// a last one of every sequence, and one dimension of a grid holds fewer than 2^32 threads.
bool many_fits(int B, int T, int Hkv, int group) {
  const int64_t rows = static_cast<int64_t>(T) * group;
  return (rows / 128 + (B < rows ? B : rows)) * Hkv < 1 << 24;
}
struct PagedPlan {
  bool few, many;         // kernels to launch
  fa::PagedMany m;        // what that for many rows runs
  bool whole;             // whether that for few rows takes whole items
  int few_cols, col_blocks, n_wg, cols;
  int64_t usual;          // row-heads that a sequence is taken to have in the kernel for few rows
  uint32_t many_work;
  int64_t lse, desc, many_o, many_lse, many_desc, bytes;  // 16-byte aligned offsets
};
PagedPlan paged_plan(int B, int T, int max_keys, int Hkv, int group, int d_qk, int d_v, int type, int max_q,
                     int path) {
  PagedPlan w{};
  const bool known = max_q > 0;
  if (!known) max_q = T > B ? T - B + 1 : 1;
  const int64_t rows = static_cast<int64_t>(T) * group, most = static_cast<int64_t>(max_q) * group;
  w.usual = known ? most : (static_cast<int64_t>(T) + B - 1) / B * group;
  const bool e4m3 = type == FA_CACHE_E4M3;
  w.many_work = kManyUnits;
  // The most units that the call can have (without max_q: that its longest sequence can have), and the fewest (sequences of
  // equal length, without cached keys); the fewest row-heads of a sequence where none has more than max_q tokens (without
  // max_q: of one that has any).
  const double items64 = known ? static_cast<double>(rows) / 64 + B : static_cast<double>((most + 63) / 64);
  const double most_units = items64 * Hkv * (6 + max_keys / 128);
  const double least_units = static_cast<double>(rows) / 64 * Hkv * (6 + T / B / 256);
  const double least = known || B == 1 ? static_cast<double>(rows) - (B - 1.0) * static_cast<double>(most) : group;
  w.many = path == FA_PAGED_MANY || (path == FA_PAGED_AUTO && most > kFewCols && rows > kFewCols && most_units >= kManyUnits &&
                                      many_fits(B, T, Hkv, group));
  w.few = !w.many || (path == FA_PAGED_AUTO && (least <= kFewCols || least_units < kSureUnits));
  w.few_cols = !w.many ? INT_MAX : w.few ? 32 : 0;
  const int64_t items32 = (rows / 32 + (B < T ? B : T)) * Hkv;
  w.col_blocks = w.usual <= 32 || w.many || (items32 <= 256 && (w.usual > kFewCols || max_keys <= kWholeKeys)) ? 1 : 2;
  if (w.many) w.m = fa::paged_many(B, T, max_keys, Hkv, group, max_q, w.few_cols, d_qk, e4m3);
  auto place = [&](int64_t n) {
    const int64_t at = w.bytes;
    w.bytes += (n + 15) / 16 * 16;
    return at;
  };
  if (w.few) {
    const int cols = 32 * w.col_blocks;
    w.n_wg = fa::paged_workgroups(d_qk, e4m3, w.col_blocks);
    w.cols = rows < cols ? static_cast<int>(rows) : cols;
    const int64_t items = (rows / cols + (B < T ? B : T)) * Hkv;  // the most there can be
    w.whole = max_keys <= kWholeKeys && items <= kWholeItems;
    if (w.whole) w.n_wg = static_cast<int>(items);
  }
  if (w.few && !w.whole) {
    const int64_t places = 2ll * w.n_wg * w.cols;
    place(places * d_v * 4);
    w.lse = place(places * 4);
    w.desc = place(w.n_wg * static_cast<int64_t>(sizeof(fa::PagedItem)));
  }
  if (w.m.split) {
    const int64_t places = 2ll * w.m.n_wg * fa::many_place_cols(w.m.cols);
    w.many_o = place(places * d_v * 4);
    w.many_lse = place(places * 4);
    w.many_desc = place(w.m.n_wg * static_cast<int64_t>(sizeof(fa::PagedItem)));
  }
  return w;
}

}  // namespace

extern "C" {

fa_status_t fa_kv_append(const fa_paged_cache_t* cache, const fa_paged_batch_t* batch, const void* K, const void* V,
                         const void* Q, void* Q_out, int Hq, const long long* strides, const float* cos_sin, int n_pos,
                         int rot_begin, int rot_dim, int interleaved, hipStream_t stream) {
  if (cache == nullptr || batch == nullptr || strides == nullptr) return FA_ERR_NULL_POINTER;
  fa_status_t st = check_paged_shape(cache, batch, Hq);
  if (st != FA_OK) return st;
  if (rot_dim < 0 || rot_begin < 0 || static_cast<int64_t>(rot_begin) + rot_dim > cache->d_qk || n_pos < 0) return FA_ERR_BAD_SHAPE;
  if (rot_dim > 0 && n_pos < static_cast<int64_t>(batch->max_blocks) * cache->page_size) return FA_ERR_BAD_SHAPE;
  st = check_paged_support(cache);
  if (st != FA_OK) return st;
  if (rot_dim > 0 && (rot_begin % 8 != 0 || rot_dim % (interleaved != 0 ? 8 : 16) != 0)) return FA_ERR_UNSUPPORTED;
  if (batch->T == 0 || batch->B == 0) return FA_OK;
  if (!paged_pointers(cache, batch) || K == nullptr || V == nullptr || (Hq > 0 && (Q == nullptr || Q_out == nullptr)) ||
      (rot_dim > 0 && cos_sin == nullptr))
    return FA_ERR_NULL_POINTER;
  if (!paged_aligned(cache, batch) || !aligned(K, 16) || !aligned(V, 16) || !aligned(Q, 16) || !aligned(Q_out, 16) ||
      !aligned(cos_sin, 16) || !token_strides(strides, 8))
    return FA_ERR_UNSUPPORTED;
  st = check_paged_strides(cache, true);
  if (st != FA_OK) return st;
  fa::AppendParams p{};
  paged_view(cache, batch, &p.c, &p.bt);
  p.q = static_cast<const uint16_t*>(Q);
  p.q_out = static_cast<uint16_t*>(Q_out);
  p.k = static_cast<const uint16_t*>(K);
  p.v = static_cast<const uint16_t*>(V);
  p.cos_sin = cos_sin;
  p.q_token = strides[0], p.q_head = strides[1], p.qo_token = strides[2], p.qo_head = strides[3];
  p.k_token = strides[4], p.k_head = strides[5], p.v_token = strides[6], p.v_head = strides[7];
  p.hq = Hq;
  p.rot = rot_dim;
  p.begin = rot_dim > 0 ? rot_begin : 0;
  p.inter = rot_dim > 0 && interleaved != 0;
  return fa::launch_append(p, cache->type == FA_CACHE_E4M3, stream) == hipSuccess ? FA_OK : FA_ERR_HIP;
}

size_t fa_fwd_paged_workspace_bytes(int B, int T, int max_keys, int Hq, int Hkv, int d_qk, int d_v, int type, int max_q,
                                    int path) {
  if (B <= 0 || T <= 0 || max_keys < 0 || Hq <= 0 || Hkv <= 0 || Hq % Hkv != 0 || max_q < 0 || !dims_supported(d_qk, d_v) ||
      (type != FA_CACHE_BF16 && type != FA_CACHE_E4M3) || path < FA_PAGED_AUTO || path > FA_PAGED_MANY)
    return 0;
  return static_cast<size_t>(paged_plan(B, T, max_keys, Hkv, Hq / Hkv, d_qk, d_v, type, max_q, path).bytes);
}

fa_status_t fa_fwd_paged(const fa_paged_cache_t* cache, const fa_paged_batch_t* batch, const void* Q, void* O, float* LSE,
                         int Hq, const long long* strides, int max_q, int path, float scale, int causal, void* workspace,
                         size_t workspace_bytes, hipStream_t stream) {
  if (cache == nullptr || batch == nullptr || strides == nullptr) return FA_ERR_NULL_POINTER;
  fa_status_t st = check_paged_shape(cache, batch, Hq);
  if (st != FA_OK) return st;
  if (max_q < 0) return FA_ERR_BAD_SHAPE;
  if (Hq > 0) {
    // The kernel's line of work is counted in 32 bits.
    const int64_t blocks = (static_cast<int64_t>(batch->T) * (Hq / cache->Hkv) / 32 + batch->B) * cache->Hkv;  // < 2^58
    const int64_t tiles = static_cast<int64_t>(batch->max_blocks) * cache->page_size / 128 + 2;
    if (blocks > INT_MAX / tiles) return FA_ERR_BAD_SHAPE;
    if (path == FA_PAGED_MANY && !many_fits(batch->B, batch->T, cache->Hkv, Hq / cache->Hkv)) return FA_ERR_BAD_SHAPE;
  }
  st = check_paged_support(cache);
  if (st != FA_OK) return st;
  if (path < FA_PAGED_AUTO || path > FA_PAGED_MANY) return FA_ERR_UNSUPPORTED;
  if (batch->T == 0 || batch->B == 0 || Hq == 0) return FA_OK;
  if (!paged_pointers(cache, batch) || Q == nullptr || O == nullptr) return FA_ERR_NULL_POINTER;
  if (!isfinite(scale)) return FA_ERR_BAD_SCALE;
  const double c = static_cast<double>(scale) * 1.4426950408889634074;
  if (fabs(c) > FLT_MAX) return FA_ERR_BAD_SCALE;
  if (!paged_aligned(cache, batch) || !aligned(Q, 16) || !aligned(O, 16) || !aligned(LSE, 4) || !token_strides(strides, 4))
    return FA_ERR_UNSUPPORTED;
  st = check_paged_strides(cache, false);
  if (st != FA_OK) return st;
  const PagedPlan w = paged_plan(batch->B, batch->T, batch->max_blocks * cache->page_size, cache->Hkv, Hq / cache->Hkv,
                                 cache->d_qk, cache->d_v, cache->type, max_q, path);
  if (w.bytes > 0 && (workspace == nullptr || workspace_bytes < static_cast<size_t>(w.bytes))) return FA_ERR_WORKSPACE;
  if (!aligned(workspace, 16)) return FA_ERR_UNSUPPORTED;

  fa::PagedParams p{};
  paged_view(cache, batch, &p.c, &p.bt);
  p.q = static_cast<const uint16_t*>(Q);
  p.o = static_cast<uint16_t*>(O);
  p.lse = LSE;
  p.q_token = strides[0], p.q_head = strides[1], p.o_token = strides[2], p.o_head = strides[3];
  p.hq = Hq;
  p.group = Hq / cache->Hkv;
  p.causal = causal != 0;
  const float cmag = fabs(c) < FLT_MIN ? FLT_MIN : static_cast<float>(fabs(c));  // a masked score stays infinite
  p.cs = c < 0 ? -cmag : cmag;
  p.few_cols = w.few_cols;
  p.many_work = w.many_work;
  p.n_wg = w.n_wg;
  p.part_cols = w.cols;
  p.whole = w.whole;
  p.many_wg = w.m.n_wg;
  p.many_cols = w.m.cols;
  unsigned char* ws = static_cast<unsigned char*>(workspace);
  p.o_part = reinterpret_cast<float*>(ws);
  p.lse_part = reinterpret_cast<float*>(ws + w.lse);
  p.desc = reinterpret_cast<fa::PagedItem*>(ws + w.desc);
  p.many_o = reinterpret_cast<float*>(ws + w.many_o);
  p.many_lse = reinterpret_cast<float*>(ws + w.many_lse);
  p.many_desc = reinterpret_cast<fa::PagedItem*>(ws + w.many_desc);
  // A single item per sequence and head reads K and V once: they are then loaded past the caches.
  const bool stream_kv = w.usual <= 32 * w.col_blocks;
  // Beside the kernel for many rows the others are mostly single tokens.
  const int64_t usual = w.many ? p.group : w.usual;
  const int cols = usual < w.cols ? static_cast<int>(usual) : w.cols;
  hipError_t e = hipSuccess;
  if (w.many) e = fa::launch_paged_many(p, w.m, cache->d_qk, cache->type == FA_CACHE_E4M3, stream);
  if (e == hipSuccess && w.few) e = fa::launch_paged_few(p, cache->d_qk, cache->type == FA_CACHE_E4M3, w.col_blocks, stream_kv, stream);
  const bool few_joins = w.few && !w.whole;
  if (e == hipSuccess && (few_joins || w.m.split))
    e = fa::launch_paged_join(p, cache->d_v, few_joins ? cols : 0, w.m.split ? w.m.cols : 0, stream);
  return e == hipSuccess ? FA_OK : FA_ERR_HIP;
}

fa_status_t fa_fwd_ex(const void* Q, const void* K, const void* V, void* O, float* LSE, int B, int Hq, int Hkv,
                      int Sq, int Sk, int d_qk, int d_v, float scale, int causal, hipStream_t stream) {
  return forward(Q, K, V, O, LSE, B, Hq, Hkv, Sq, Sk, d_qk, d_v, scale, causal, stream);
}

fa_status_t fa_fwd(const void* Q, const void* K, const void* V, void* O, int B, int Hq, int Hkv, int Sq, int Sk,
                   int d, float scale, int causal, hipStream_t stream) {
  return forward(Q, K, V, O, nullptr, B, Hq, Hkv, Sq, Sk, d, d, scale, causal, stream);
}

fa_status_t fa_fwd_split(const void* Q, const void* K, const void* V, void* O, float* LSE, int B, int Hq, int Hkv,
                         int Sq, int Sk, int d_qk, int d_v, float scale, int causal, int n_split, void* workspace,
                         size_t workspace_bytes, hipStream_t stream) {
  if (n_split < 1) return FA_ERR_BAD_SHAPE;
  return forward(Q, K, V, O, LSE, B, Hq, Hkv, Sq, Sk, d_qk, d_v, scale, causal, stream, n_split, workspace,
                 workspace_bytes);
}

fa_status_t fa_fwd_decode(const void* Q, const void* K, const void* V, void* O, float* LSE, int B, int Hq, int Hkv,
                          int Sq, int Sk, int d_qk, int d_v, float scale, int causal, int n_parts, void* workspace,
                          size_t workspace_bytes, hipStream_t stream) {
  if (n_parts < 1) return FA_ERR_BAD_SHAPE;
  float cs = 0.f;
  fa_status_t st = check_fused(Q, K, V, O, LSE, B, Hq, Hkv, Sq, Sk, d_qk, d_v, scale, causal, &cs);
  if (st != FA_OK) return st;
  if (static_cast<int64_t>(B) * Hq * Sq == 0) return FA_OK;
  int64_t need = 0;
  st = decode_grid(B, Hq, Hkv, Sq, d_v, n_parts, &need);
  if (st != FA_OK) return st;
  if (need < 0 || workspace == nullptr || static_cast<uint64_t>(need) > workspace_bytes) return FA_ERR_WORKSPACE;
  if (!aligned(workspace, 16)) return FA_ERR_UNSUPPORTED;
  return decode_launch(Q, K, V, O, LSE, B, Hq, Hkv, Sq, Sk, d_qk, d_v, cs, causal, n_parts, workspace, stream) ==
                 hipSuccess
             ? FA_OK
             : FA_ERR_HIP;
}

fa_status_t fa_fwd_decode_noalloc(const void* Q, const void* K, const void* V, void* O, float* LSE, int B, int Hq,
                                  int Hkv, int Sq, int Sk, int d_qk, int d_v, float scale, int causal, int n_parts,
                                  hipStream_t stream) {
  if (n_parts < 1) return FA_ERR_BAD_SHAPE;
  float cs = 0.f;
  fa_status_t st = check_fused(Q, K, V, O, LSE, B, Hq, Hkv, Sq, Sk, d_qk, d_v, scale, causal, &cs);
  if (st != FA_OK) return st;
  if (static_cast<int64_t>(B) * Hq * Sq == 0) return FA_OK;
  int64_t need = 0;
  st = decode_grid(B, Hq, Hkv, Sq, d_v, n_parts, &need);
  if (st != FA_OK) return st;
  if (need < 0 || need > static_cast<int64_t>(FA_NOALLOC_SCRATCH_BYTES)) return FA_ERR_WORKSPACE;
  void* ws = nullptr;
  if (scratch_for_stream(stream, &ws) != hipSuccess) return FA_ERR_HIP;
  return decode_launch(Q, K, V, O, LSE, B, Hq, Hkv, Sq, Sk, d_qk, d_v, cs, causal, n_parts, ws, stream) ==
                 hipSuccess
             ? FA_OK
             : FA_ERR_HIP;
}

int fa_fwd_decode_parts(int n_cu, int B, int Hq, int Hkv, int Sq, int Sk) {
  if (n_cu <= 0 || B <= 0 || Hq <= 0 || Hkv <= 0 || Hq % Hkv != 0 || Sq <= 0 || Sk < 0) return 0;
  // One workgroup per CU in total (a workgroup holds two K+V tiles in LDS, so one fits a CU), but
  // no part shorter than 4 key tiles.
  const int64_t n_cb = (static_cast<int64_t>(Hq / Hkv) * Sq + 31) / 32;
  const int64_t items = static_cast<int64_t>(B) * Hkv * n_cb;
  const int64_t tiles = (static_cast<int64_t>(Sk) + fa::decode_tile_keys() - 1) / fa::decode_tile_keys();
  int64_t parts = (n_cu + items - 1) / items;
  const int64_t max_parts = (tiles + 3) / 4;
  if (parts > max_parts) parts = max_parts;
  return parts < 1 ? 1 : static_cast<int>(parts);
}

int fa_fwd_split_parts(int n_cu, int B, int Hq, int Sq, int Sk, int d_qk, int d_v, int causal) {
  const int bm = fa::block_rows(d_qk, d_v, causal != 0);
  if (bm == 0 || n_cu <= 0 || B <= 0 || Hq <= 0 || Sq <= 0 || Sk < 0) return 0;
  // Enough workgroups for about two per CU, but no part shorter than 8 key tiles (the fixed cost of
  // a workgroup and of the merge would dominate). The query block with the most keys sees all Sk.
  const int64_t items = static_cast<int64_t>(B) * Hq * ((static_cast<int64_t>(Sq) + bm - 1) / bm);
  const int64_t max_parts = (static_cast<int64_t>(Sk) + 64 * 8 - 1) / (64 * 8);
  int64_t parts = (2 * static_cast<int64_t>(n_cu)) / items;
  if (parts > max_parts) parts = max_parts;
  return parts < 1 ? 1 : static_cast<int>(parts);
}

size_t fa_fwd_split_workspace_bytes(int B, int Hq, int Sq, int d_v, int n_split) {
  const int64_t n = split_workspace_bytes(B, Hq, Sq, d_v, n_split);
  return n < 0 ? SIZE_MAX : static_cast<size_t>(n);
}

int fa_lbl_ld(int Sk) { return Sk < 0 || Sk > fa::kLblMaxSk ? -1 : static_cast<int>(lbl_ld(Sk)); }

size_t fa_lbl_workspace_bytes(int B, int Hq, int Sq, int Sk) {
  if (B <= 0 || Hq <= 0 || Sq <= 0 || Sk <= 0) return 0;
  if (Sk > fa::kLblMaxSk) return SIZE_MAX;
  const int64_t bh = static_cast<int64_t>(B) * Hq;
  const int64_t per_row = lbl_ld(Sk) * 2;  // < 2^24
  if (bh > INT64_MAX / Sq) return SIZE_MAX;
  const int64_t rows = bh * Sq;
  if (rows > INT64_MAX / per_row) return SIZE_MAX;
  return static_cast<size_t>(rows * per_row);
}

fa_status_t fa_lbl_scores(const void* Q, const void* K, void* S, int B, int Hq, int Hkv, int Sq, int Sk, int d_qk,
                          float scale, int causal, hipStream_t stream) {
  fa_status_t st = lbl_check_shape(B, Hq, Hkv, Sq, Sk, d_qk, 0);
  if (st != FA_OK) return st;
  const bool q_rows = static_cast<int64_t>(B) * Hq * Sq > 0;
  const bool kv_rows = static_cast<int64_t>(B) * Hkv * Sk > 0;
  if ((q_rows && Q == nullptr) || (kv_rows && K == nullptr) || (q_rows && Sk > 0 && S == nullptr))
    return FA_ERR_NULL_POINTER;
  if (!isfinite(scale)) return FA_ERR_BAD_SCALE;
  if (!aligned(Q, 16) || !aligned(K, 16) || !aligned(S, 16)) return FA_ERR_UNSUPPORTED;
  if (!q_rows || Sk == 0) return FA_OK;  // no score to write
  fa::LblParams p = lbl_params(B, Hq, Hkv, Sq, Sk, scale, causal);
  p.q = static_cast<const uint16_t*>(Q);
  p.k = static_cast<const uint16_t*>(K);
  p.s = static_cast<uint16_t*>(S);
  return fa::launch_lbl_scores(p, d_qk, stream) == hipSuccess ? FA_OK : FA_ERR_HIP;
}

fa_status_t fa_lbl_softmax(const void* S, void* P, float* LSE, int B, int Hq, int Sq, int Sk, int causal,
                           hipStream_t stream) {
  fa_status_t st = lbl_check_shape(B, Hq, Hq > 0 ? 1 : 0, Sq, Sk, 0, 0);
  if (st != FA_OK) return st;
  const bool rows = static_cast<int64_t>(B) * Hq * Sq > 0;
  if (rows && Sk > 0 && (S == nullptr || P == nullptr)) return FA_ERR_NULL_POINTER;
  if (!aligned(S, 16) || !aligned(P, 16) || !aligned(LSE, 4)) return FA_ERR_UNSUPPORTED;
  if (!rows) return FA_OK;
  fa::LblParams p = lbl_params(B, Hq, 1, Sq, Sk, 1.f, causal);
  p.s = const_cast<uint16_t*>(static_cast<const uint16_t*>(S));
  p.p = static_cast<uint16_t*>(P);
  p.lse = LSE;
  return fa::launch_lbl_softmax(p, stream) == hipSuccess ? FA_OK : FA_ERR_HIP;
}

fa_status_t fa_lbl_pv(const void* P, const void* V, void* O, int B, int Hq, int Hkv, int Sq, int Sk, int d_v,
                      int causal, hipStream_t stream) {
  fa_status_t st = lbl_check_shape(B, Hq, Hkv, Sq, Sk, 0, d_v);
  if (st != FA_OK) return st;
  const bool q_rows = static_cast<int64_t>(B) * Hq * Sq > 0;
  const bool kv_rows = static_cast<int64_t>(B) * Hkv * Sk > 0;
  if ((q_rows && O == nullptr) || (kv_rows && V == nullptr) || (q_rows && Sk > 0 && P == nullptr))
    return FA_ERR_NULL_POINTER;
  if (!aligned(P, 16) || !aligned(V, 16) || !aligned(O, 16)) return FA_ERR_UNSUPPORTED;
  if (!q_rows) return FA_OK;
  fa::LblParams p = lbl_params(B, Hq, Hkv, Sq, Sk, 1.f, causal);
  p.p = const_cast<uint16_t*>(static_cast<const uint16_t*>(P));
  p.v = static_cast<const uint16_t*>(V);
  p.o = static_cast<uint16_t*>(O);
  return fa::launch_lbl_pv(p, d_v, stream) == hipSuccess ? FA_OK : FA_ERR_HIP;
}

fa_status_t fa_fwd_unfused(const void* Q, const void* K, const void* V, void* O, float* LSE, int B, int Hq, int Hkv,
                           int Sq, int Sk, int d_qk, int d_v, float scale, int causal, void* workspace,
                           size_t workspace_bytes, hipStream_t stream) {
  fa_status_t st = lbl_check_shape(B, Hq, Hkv, Sq, Sk, d_qk, d_v);
  if (st != FA_OK) return st;
  const bool q_rows = static_cast<int64_t>(B) * Hq * Sq > 0;
  const bool kv_rows = static_cast<int64_t>(B) * Hkv * Sk > 0;
  if ((q_rows && (Q == nullptr || O == nullptr)) || (kv_rows && (K == nullptr || V == nullptr)))
    return FA_ERR_NULL_POINTER;
  if (!isfinite(scale)) return FA_ERR_BAD_SCALE;
  if (!aligned(Q, 16) || !aligned(K, 16) || !aligned(V, 16) || !aligned(O, 16) || !aligned(LSE, 4))
    return FA_ERR_UNSUPPORTED;
  if (!q_rows) return FA_OK;
  // Rows of spill buffer the workspace holds; one block of query rows (or all of Sq if shorter) is
  // the least a chunk needs.
  const int64_t row_bytes = lbl_ld(Sk) * 2;
  const int64_t min_rows = Sq < fa::kLblRows ? Sq : fa::kLblRows;
  const int64_t cap = row_bytes == 0 ? INT64_MAX : static_cast<int64_t>(workspace_bytes / row_bytes);
  if (row_bytes > 0 && (workspace == nullptr || cap < min_rows)) return FA_ERR_WORKSPACE;
  if (!aligned(workspace, 16)) return FA_ERR_UNSUPPORTED;

  fa::LblParams p = lbl_params(B, Hq, Hkv, Sq, Sk, scale, causal);
  p.q = static_cast<const uint16_t*>(Q);
  p.k = static_cast<const uint16_t*>(K);
  p.v = static_cast<const uint16_t*>(V);
  p.o = static_cast<uint16_t*>(O);
  p.lse = LSE;
  p.s = p.p = static_cast<uint16_t*>(workspace);  // probabilities overwrite the scores in place
  const int n_bh = B * Hq, n_qb = p.nqb;
  const hipStream_t s = stream;
  auto run = [&](int bh0, int nbh, int qb0, int nqb) {
    p.bh0 = bh0;
    p.nbh = nbh;
    p.qb0 = qb0;
    p.nqb = nqb;
    p.xgroup = (bh0 % p.group == 0 && nbh % p.group == 0) ? p.group : 1;
    const int64_t last = static_cast<int64_t>(qb0 + nqb) * fa::kLblRows;
    p.rows = static_cast<int64_t>(nbh - 1) * Sq + (last < Sq ? last : Sq) - static_cast<int64_t>(qb0) * fa::kLblRows;
    if (fa::launch_lbl_scores(p, d_qk, s) != hipSuccess) return false;
    if (fa::launch_lbl_softmax(p, s) != hipSuccess) return false;
    return fa::launch_lbl_pv(p, d_v, s) == hipSuccess;
  };
  if (cap >= static_cast<int64_t>(Sq)) {
    // Whole heads per chunk, a multiple of the group size when more than one group fits.
    int64_t heads = cap / Sq;
    if (heads > n_bh) heads = n_bh;
    if (heads >= p.group) heads -= heads % p.group;
    for (int64_t bh0 = 0; bh0 < n_bh; bh0 += heads) {  // 64-bit: bh0 + heads may pass INT_MAX
      const int nbh = static_cast<int>(n_bh - bh0 < heads ? n_bh - bh0 : heads);
      if (!run(static_cast<int>(bh0), nbh, 0, n_qb)) return FA_ERR_HIP;
    }
  } else {
    // Part of one head per chunk.
    const int blocks = static_cast<int>(cap / fa::kLblRows);
    for (int bh = 0; bh < n_bh; ++bh)
      for (int qb0 = 0; qb0 < n_qb; qb0 += blocks)
        if (!run(bh, 1, qb0, n_qb - qb0 < blocks ? n_qb - qb0 : blocks)) return FA_ERR_HIP;
  }
  return FA_OK;
}

const char* fa_status_str(fa_status_t s) {
  switch (s) {
    case FA_OK: return "FA_OK";
    case FA_ERR_NULL_POINTER: return "FA_ERR_NULL_POINTER";
    case FA_ERR_BAD_SHAPE: return "FA_ERR_BAD_SHAPE";
    case FA_ERR_UNSUPPORTED: return "FA_ERR_UNSUPPORTED";
    case FA_ERR_BAD_SCALE: return "FA_ERR_BAD_SCALE";
    case FA_ERR_HIP: return "FA_ERR_HIP";
    case FA_ERR_WORKSPACE: return "FA_ERR_WORKSPACE";
  }
  return "unknown status";
}

int fa_block_rows(int d_qk, int d_v, int causal) { return fa::block_rows(d_qk, d_v, causal != 0); }

int fa_fwd_rows(int B, int Hq, int Sq, int d_qk, int d_v, int causal) {
  return fa::instance_rows(B, Hq, Sq, d_qk, d_v, causal != 0);
}

fa_instance_t fa_fwd_instance(int B, int Hq, int Hkv, int Sq, int Sk, int d_qk, int d_v, int causal, int n_split) {
  static_assert(FA_INSTANCE_QUARTERS == 1 && FA_INSTANCE_HALVES == 2 && FA_INSTANCE_SHORT == 3 &&
                    FA_INSTANCE_SHORT_WIDE == 4 && FA_INSTANCE_LONG == 5,
                "launch_instance_id returns these values");
  return static_cast<fa_instance_t>(fa::launch_instance_id(B, Hq, Hkv, Sq, Sk, d_qk, d_v, causal != 0, n_split));
}

}  // extern "C"
