// Internal interface between the C-ABI layer (fa_api.hip) and the kernel launchers (fa_fwd_kernel.hip:
// fused forward and split mode; fa_decode_kernel.hip: decode; fa_lbl_kernel.hip: layer-by-layer operators;
// fa_paged_kernel.hip and fa_paged_fwd_kernel.hip: the paged cache). Not installed; callers use include/fa.h.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace fa {

// Arguments of one forward launch, after host-side validation.
struct FwdParams {
  const uint16_t* q;  // bf16 [B][Hq][Sq][d_qk]
  const uint16_t* k;  // bf16 [B][Hkv][Sk][d_qk]
  const uint16_t* v;  // bf16 [B][Hkv][Sk][d_v]
  uint16_t* o;        // bf16 [B][Hq][Sq][d_v]
  float* lse;         // fp32 [B][Hq][Sq] or nullptr
  int batch, hq, hkv, sq, sk;
  int group;          // Hq / Hkv
  float cs;           // scale * log2(e), magnitude at least FLT_MIN so that an infinite (masked)
                      // score stays infinite; negative when scale < 0
  int n_qtiles;       // ceil(Sq / block rows)
  int n_wg;           // work items (query blocks): batch * hq * n_qtiles
  // Work decomposition constants (host-computed): the items in whole spans of 8 groups, and the
  // multiply-high constants for dividing by group, hkv and batch, their shifts packed 6 bits apart.
  int full;
  int head_chunk, head_chunked;  // key/value heads per chunk, and how many of them run in whole chunks
  uint32_t m_group, m_hkv, m_batch, shifts;
  // Split mode only: number of key-range parts, and the partial results, in the caller's workspace:
  // o_part fp32 [n_split][B][Hq][Sq][d_v] (O of each part normalised by its own row sum), lse_part
  // fp32 [n_split][B][Hq][Sq].
  int n_split;
  float* o_part;
  float* lse_part;
};

// Arguments of the merge pass of split mode.
struct MergeParams {
  const float* o_part;
  const float* lse_part;
  uint16_t* o;      // bf16 [rows][d_v]
  float* lse;       // fp32 [rows] or nullptr
  int64_t rows;     // B * Hq * Sq
  int n_split;
};

// Query rows per workgroup of the long kernel instance for (d_qk, d_v, causal) when a workgroup holds
// one query head (split mode, every d_qk = 192 problem, and problems with more such blocks than the
// other instances take); 0 if not compiled in.
// With a GQA group size divisible by 2 or 4 a workgroup holds as many query heads, each with half or
// a quarter of these rows.
int block_rows(int d_qk, int d_v, bool causal);
// Query rows per block holding one query head of the instance that the grid alone selects for the fused
// forward (a launch with more than twice as many keys as query rows may run another one): the long instance's block_rows() (256), the short instance's 128 or the key-parts instances' 64 (the
// key quarters run such a block as two workgroups); 0 for unsupported head dimensions or negative sizes.
int instance_rows(int batch, int hq, int sq, int d_qk, int d_v, bool causal);
// The instance a launch runs (n_split == 0: the fused forward; else split mode), as fa_instance_t's values.
int launch_instance_id(int batch, int hq, int hkv, int sq, int sk, int d_qk, int d_v, bool causal, int n_split);
// Workgroups of the long instance's grid (one part per query block and packed heads).
int64_t forward_workgroups(int batch, int hq, int hkv, int sq);

// Enqueue the forward kernel for (d_qk, d_v, causal) on `stream`. Requires Sq > 0, B*Hq > 0 and a
// grid that fits; fills n_qtiles / n_wg itself. Returns the launch status of the HIP runtime.
hipError_t launch_forward(FwdParams p, int d_qk, int d_v, bool causal, hipStream_t stream);

// Split mode: the forward kernel over n_split parts of every query block's key range, writing the
// partial results, then the merge pass into O / LSE, both on `stream`. Same requirements as
// launch_forward plus n_split >= 1 and the partial buffers.
hipError_t launch_forward_split(FwdParams p, int d_qk, int d_v, bool causal, hipStream_t stream);

// The merge pass alone (d_v 64 or 128), on `stream`.
hipError_t launch_merge(MergeParams m, int d_v, hipStream_t stream);

// ---- decode-shaped problems (fa_decode_kernel.hip) -----------------------------------------------
//
// The group's query heads and their Sq rows form the columns of 32-column MFMA blocks; workgroup t
// takes part t % n_parts of column block (t / n_parts) % n_cb of (batch, key/value head)
// t / (n_parts * n_cb), and the parts are
// merged by the merge pass of split mode (same partial-result layout: o_part fp32
// [n_parts][B][Hq][Sq][d_v], lse_part fp32 [n_parts][B][Hq][Sq]).
struct DecodeParams {
  const uint16_t* q;
  const uint16_t* k;
  const uint16_t* v;
  uint16_t* o;
  float* lse;
  float* o_part;
  float* lse_part;
  int batch, hq, hkv, sq, sk, group, causal;
  float cs;           // scale * log2(e), as in FwdParams
  int rows;           // group * Sq (columns)
  int n_parts;
  int n_tiles, per;   // filled by launch_decode: key tiles, tiles per part
  int n_cb;           // filled by launch_decode: 32-column blocks
  int64_t total_rows; // B * Hq * Sq, filled by launch_decode
};

// Keys per tile of the decode kernel.
int decode_tile_keys();
// Enqueue the decode kernel and the merge pass on `stream`; (d_qk, d_v) in {(64,64), (128,128), (192,128)}.
hipError_t launch_decode(DecodeParams p, int d_qk, int d_v, hipStream_t stream);

// ---- layer-by-layer (unfused) operators --------------------------------------------------------
//
// A work unit is one block of kLblRows query rows of one (batch, query head); bh = b * Hq + h. A chunk
// is a rectangle of units, query heads bh0 .. bh0+nbh-1 times query blocks qb0 .. qb0+nqb-1, that is
// either whole heads (qb0 = 0, all blocks) or part of one head (nbh = 1). Row r of the chunk, i.e.
// (bh - bh0) * Sq + (qb - qb0) * kLblRows + row in block, is row r of the spill buffers S and P
// (stride ld elements). Key extents are multiples of kLblKeys: the rows of block qb use keys
// [0, lbl_extent(qb)), the visible keys of the block's last row rounded up.
constexpr int kLblRows = 128;
constexpr int kLblKeys = 64;
// Largest Sk of the layer-by-layer operators: keeps every byte offset inside one block's rows of the
// spill buffer (kLblRows * ld * 2) below 2^30.
constexpr int kLblMaxSk = 1 << 22;

struct LblParams {
  const uint16_t* q;  // bf16 [B][Hq][Sq][d_qk]
  const uint16_t* k;  // bf16 [B][Hkv][Sk][d_qk]
  const uint16_t* v;  // bf16 [B][Hkv][Sk][d_v]
  uint16_t* s;        // bf16 scores of the chunk, row stride ld
  uint16_t* p;        // bf16 probabilities of the chunk, row stride ld (may equal s)
  uint16_t* o;        // bf16 [B][Hq][Sq][d_v]
  float* lse;         // fp32 [B][Hq][Sq] or nullptr
  int batch, hq, hkv, sq, sk, group, causal;
  int ld;             // Sk rounded up to kLblKeys
  float scale;
  int bh0, nbh, qb0, nqb;
  int xgroup;         // query heads placed together on one XCD: group if the chunk is aligned to it, else 1
  int64_t rows;       // rows of the chunk
};

bool lbl_scores_supported(int d_qk);
bool lbl_pv_supported(int d_v);
// Each enqueues one kernel over the chunk on `stream` and returns the launch status.
hipError_t launch_lbl_scores(const LblParams& p, int d_qk, hipStream_t stream);
hipError_t launch_lbl_softmax(const LblParams& p, hipStream_t stream);
hipError_t launch_lbl_pv(const LblParams& p, int d_v, hipStream_t stream);

// ---- paged key/value cache (fa_paged_kernel.hip) -------------------------------------------------

// The cache: strides in elements (2 bytes each, or 1 for e4m3); a page holds 1 << page_shift slots.
struct PagedCache {
  void* k;
  void* v;
  const float* k_scale;  // fp32 [Hkv] or nullptr (1): an e4m3 element stands for itself times the scale
  const float* v_scale;
  int64_t k_page, k_head, k_slot, v_page, v_head, v_slot;
  int n_pages, page_shift, hkv, d_qk, d_v;
};

// The batch; all arrays are device data.
struct PagedBatch {
  const int* block_table;  // [n_seq], rows table_stride apart: page numbers
  const int* kv_lens;      // [n_seq]
  const int* q_starts;     // [n_seq + 1]
  int64_t table_stride;
  int n_seq, n_tokens;
  int max_keys;            // keys that a row of the table has pages for
};

// Where a token's rows of the table of angles come from, if not from its place: device arrays.
struct Positions {
  const int* positions;            // token t's position on axis a at t * token + a * axis (batch: the rotation alone)
  const unsigned char* pair_axes;  // [rot / 2]: the axis of each pair; nullptr: the first
  int64_t batch, token, axis;
  int n_axes, n_pos;
};

struct AppendParams {
  PagedCache c;
  PagedBatch bt;
  const uint16_t* q;
  uint16_t* q_out;
  const uint16_t* k;
  const uint16_t* v;
  const float* cos_sin;  // fp32 [positions][rot]: cosines, then sines
  int64_t q_token, q_head, qo_token, qo_head, k_token, k_head, v_token, v_head;
  int hq;                // 0: no queries
  int rot, begin, inter; // rotated dims (0: none), the first of them, neighbouring pairs
  Positions pos;         // positions nullptr: the row of a token is its place among its sequence's keys
};

// Columns of a place of the kernel for many rows. One more than a block has: with places 128 KiB apart the workgroups that
// write and read the same column of theirs at one time would all meet in the same memory channels.
__host__ __device__ constexpr int many_place_cols(int cols) { return cols + 1; }

// An item of the attention that several workgroups share, written by the first of them for the join kernel.
struct PagedItem {
  int n_parts;  // 0 or 1: nothing to join
  int q0;       // first packed token of the sequence
  int n_cols, c0, g;
  int first;    // that workgroup's index on the line of work: its places and those of the next ones hold the parts
  int pad[2];
};

// How scores are changed and keys hidden, beyond causal masking (fa_paged_scores_t).
struct PagedForms {
  float cap_a, cap_r;        // cap * log2(e), 2 / cap; 0: no cap
  const float* slopes;       // [Hq] or nullptr
  const int* prefix_lens;    // [n_seq] or nullptr
  const uint32_t* mask;      // [n_tokens], rows mask_stride apart: the new tokens that a token sees; or nullptr
  int64_t mask_stride;
  int mask_words;
  int window;                // 0: none; below 2^30
  int causal;                // PagedParams::causal
};

struct PagedParams {
  PagedCache c;
  PagedBatch bt;
  const uint16_t* q;
  uint16_t* o;
  float* lse;            // fp32 [n_tokens][Hq] or nullptr
  int64_t q_token, q_head, o_token, o_head;
  int hq, group, causal;
  float cs;              // scale * log2(e)
  int n_wg, min_units;   // workgroups (a power of two), fewest units of work of one
  int wg_log;            // log2 of n_wg, filled by launch_paged_few
  int whole;             // nonzero: a workgroup takes one whole item, n_wg covers the most there can be; no join
  int part_cols;         // columns of a place in the workspace
  float* o_part;         // fp32 [2 * n_wg][part_cols][d_v]
  float* lse_part;       // fp32 [2 * n_wg][part_cols]
  PagedItem* desc;       // [n_wg]
  // Sequences with more than few_cols row-heads per key/value head run in the kernel for many rows if all of them together
  // have many_work units of work (big_work in fa_paged_device.h), else in that for few rows. few_cols INT32_MAX: only the
  // latter is launched; 0: only the former. It has work units, places and items of its own (the latter three only
  // where it splits blocks).
  int few_cols;
  uint32_t many_work;
  int many_wg, many_min_units, many_cols;  // many_wg: a power of two; many_cols: columns of a block
  int many_log;          // log2 of many_wg, filled by launch_paged_many
  float* many_o;         // fp32 [2 * many_wg][many_place_cols(many_cols)][d_v]
  float* many_lse;       // fp32 [2 * many_wg][many_place_cols(many_cols)]
  PagedItem* many_desc;  // [many_wg]
  uint32_t m_group, sh_group;  // division by group, filled by the launchers
  PagedForms f;            // used by the kernels with forms alone
};

// ---- rotation alone (fa_rotate_kernel.hip) --------------------------------------------------------

struct RotateParams {
  const uint16_t* x;
  uint16_t* y;
  const float* cos_sin;
  Positions pos;          // positions nullptr: the row of token s is s
  int64_t x_b, x_h, x_s, y_b, y_h, y_s;
  int batch, h, s, d, rot, begin, inter, in_place;
  float sign;             // of the angles
  int per, n_blocks, heads;  // filled by launch_rotate: blocks of tokens of a batch and in all, heads of a workgroup
  uint32_t m_per, sh_per;
};
hipError_t launch_rotate(RotateParams p, hipStream_t stream);

// ---- around the paged cache (fa_paged_moves_kernel.hip) --------------------------------------------

struct TreeParams {
  PagedBatch bt;          // block_table unused
  const int* parents;     // [n_tokens]
  uint32_t* mask;         // [n_tokens], rows mask_stride apart
  int64_t mask_stride;
  int words;
  int* positions;         // [n_tokens]
};
hipError_t launch_tree_mask(TreeParams p, hipStream_t stream);

// Sequences of one row of the grid (its second dimension; the third counts rows).
constexpr int kMoveRows = 65535;
struct CompactParams {
  PagedCache c;
  PagedBatch bt;
  const int* kept;        // [n_seq], rows kept_stride apart
  const int* n_kept;      // [n_seq]
  int64_t kept_stride;
  int max_kept, elem;     // entries of a row, bytes of an element
  int* lens_out;          // [n_seq]
  uint32_t k_chunks, v_chunks, m_k, sh_k, m_v, sh_v;  // filled by launch_kv_compact: 16-byte chunks of a row
};
// Workgroups of a sequence, one at least.
int64_t kv_compact_blocks(int hkv, int d_qk, int d_v, int elem);
hipError_t launch_kv_compact(CompactParams p, hipStream_t stream);

// K or V of a page as heads of rows of `run` 16-byte chunks; strides in bytes.
struct CopySide {
  unsigned char* base;
  int64_t page, head, row;
  uint32_t chunks, rows, run, m_run, sh_run, m_rows, sh_rows;
};
struct CopyParams {
  CopySide side[2];
  const int* src;
  const int* dst;
  int n_pages;
  uint32_t parts, m_parts, sh_parts;  // workgroups of a pair of pages
};
// Workgroups of a copy of n pages (of K, and as many of V); -1 where a page is too large.
int64_t kv_copy_blocks(const PagedCache& c, int elem, int n);
hipError_t launch_kv_copy(const PagedCache& c, int elem, const int* src, const int* dst, int n, hipStream_t stream);

hipError_t launch_append(AppendParams p, bool fp8, hipStream_t stream);
// Workgroups of the attention kernel (as many as the chip holds at once).
int paged_workgroups(int d_qk, bool fp8, int col_blocks);
// The kernels below run on `stream`; (d_qk, d_v) as for the other paths. Few rows: every sequence with at most few_cols
// row-heads per key/value head, in items of 32 * col_blocks of them (1 or 2). stream_kv: K and V are loaded past the
// caches (items of 32 always are).
hipError_t launch_paged_few(PagedParams p, int d_qk, bool fp8, int col_blocks, bool stream_kv, hipStream_t stream);
// Join of split items of the kernel for few rows and of that for many: the columns that an item of each is expected to have, 0
// where there is nothing to join.
hipError_t launch_paged_join(PagedParams p, int d_v, int few_cols, int many_cols, hipStream_t stream);
// Many rows (fa_paged_fwd_kernel.hip): all other sequences, in blocks of `cols` row-heads of a key/value head. Where `split`,
// n_wg workgroups share the blocks, which are split if the lengths make it worth it, and a join follows; else a workgroup
// takes a block, of which there are at most `blocks` per key/value head. max_q, as the host expects it, helps to choose the
// instance.
struct PagedMany {
  bool is_short, split;
  int cols, n_wg;
  int64_t blocks;
};
PagedMany paged_many(int n_seq, int n_tokens, int max_keys, int hkv, int group, int max_q, int few_cols, int d_qk, bool e4m3,
                     bool forms);
hipError_t launch_paged_many(const PagedParams& p, const PagedMany& m, int d_qk, bool e4m3, hipStream_t stream);
// The same kernels with forms (fa_paged_forms_few_kernel.hip; fa_paged_masked_kernel.hip, fa_paged_capped_kernel.hip,
// fa_paged_biased_kernel.hip: scores as they are, capped, or with slopes).
hipError_t launch_paged_few_forms(PagedParams p, int d_qk, bool fp8, int col_blocks, hipStream_t stream);
hipError_t launch_paged_many_masked(const PagedParams& p, const PagedMany& m, int d_qk, bool e4m3, hipStream_t stream);
hipError_t launch_paged_many_capped(const PagedParams& p, const PagedMany& m, int d_qk, bool e4m3, hipStream_t stream);
hipError_t launch_paged_many_biased(const PagedParams& p, const PagedMany& m, int d_qk, bool e4m3, hipStream_t stream);

}  // namespace fa
