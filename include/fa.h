/*
 * fa.h -- C ABI of the attention forward for AMD Instinct MI355X (gfx950): the fused kernel, its
 * split mode, the unfused layer-by-layer operators it is measured against, and a paged key/value cache: appending to
 * it, attention over it (also with other masks and scores), drafted trees, and moves in it.
 *
 * Operation (the paper's scaled dot-product attention, Eq. (1), Sec. 2.1, replicated over heads):
 *
 *     O[b,h] = softmax(scale * Q[b,h] * K[b,g]^T) * V[b,g],   g = h / (Hq / Hkv)
 *
 * computed in one kernel launch: the score tile S = Q K^T never leaves the chip; an online softmax
 * keeps a running row max and row sum and rescales the partial P V accumulation (Alg. 1, Sec. 2.1).
 * The query heads h of one group share key/value head g (grouped-query attention, Sec. 4.4 and
 * Sec. 6.5). With causal masking, key j is visible to query i iff j <= i + (Sk - Sq) (bottom-right
 * alignment; the usual j <= i when Sq == Sk).
 *
 * Element types: Q, K, V and O are IEEE bfloat16 bit patterns (torch.bfloat16). LSE is float32.
 * Arithmetic: bf16 x bf16 products with fp32 accumulation for both contractions; softmax statistics
 * and the output accumulator in fp32; P is rounded to bf16 (round-to-nearest-even) only as the
 * operand of the P V product; O is rounded to bf16 (RNE) once, at the end.
 *
 * Layout: every tensor is a contiguous row-major BHSD array in device memory, no strides:
 *     Q   [B][Hq ][Sq][d_qk]      K [B][Hkv][Sk][d_qk]      V [B][Hkv][Sk][d_v]
 *     O   [B][Hq ][Sq][d_v ]      LSE (optional) float32 [B][Hq][Sq]
 * LSE[b,h,i] = ln( sum over visible j of exp(scale * q_i . k_j) ), natural log; -inf for a row with
 * no visible key (that row's O is 0).
 *
 * Ownership: the caller owns every buffer. The library allocates nothing, frees nothing, and is
 * reentrant and thread-safe; its only state is the static scratch array of fa_fwd_decode_noalloc
 * (below) and that array's per-device address. Q, K, V are only read; O and
 * LSE are only written, every element exactly once per call.
 *
 * Asynchrony: the work is enqueued on `stream` (NULL is the null stream of the current device);
 * FA_OK means "enqueued". The library never synchronises. Faults
 * during execution surface at the caller's next synchronisation.
 *
 * Errors: every argument check runs on the host before any HIP call. On any error return nothing is
 * launched and O / LSE are untouched, so the checks are usable on a machine without a GPU. Checks run
 * in this order and the first failing one is reported: sizes (FA_ERR_BAD_SHAPE), head dimensions
 * (FA_ERR_UNSUPPORTED), pointers (FA_ERR_NULL_POINTER), scale (FA_ERR_BAD_SCALE), alignment
 * (FA_ERR_UNSUPPORTED), index ranges (FA_ERR_BAD_SHAPE).
 *
 * Degenerate sizes: B == 0, Hq == 0 or Sq == 0 is a no-op returning FA_OK (no HIP call). Sk == 0
 * is valid: every row gets O = 0 and LSE = -inf.
 *
 * Supported head dimensions: (d_qk, d_v) in {(64, 64), (128, 128), (192, 128)}; others return
 * FA_ERR_UNSUPPORTED.
 */
#ifndef FA_MI355X_FA_H
#define FA_MI355X_FA_H

#include <stddef.h>

/* HIP's stream handle, the same declaration as in hip/hip_runtime_api.h, so that this header needs
 * no HIP include (C callers may include either header first). */
typedef struct ihipStream_t* hipStream_t;

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  FA_OK = 0,
  FA_ERR_NULL_POINTER = 1, /* Q or O is NULL with B*Hq*Sq > 0, or K or V is NULL with B*Hkv*Sk > 0 */
                           /* (LSE may always be NULL)                                            */
  FA_ERR_BAD_SHAPE = 2,    /* a size < 0; Hkv <= 0 or Hq % Hkv != 0 with Hq > 0; Sq*d or Sk*d of  */
                           /* one head >= 2^31 elements; more than 2^31-1 workgroups              */
  FA_ERR_UNSUPPORTED = 3,  /* (d_qk, d_v) not compiled in; Q/K/V/O not 16-byte aligned, or LSE   */
                           /* not 4-byte aligned                                                  */
  FA_ERR_BAD_SCALE = 4,    /* scale is NaN or +-inf, or |scale| * log2(e) overflows float32       */
  FA_ERR_HIP = 5,          /* the HIP runtime reported an error when enqueuing the kernel         */
  FA_ERR_WORKSPACE = 6     /* split mode: workspace NULL or smaller than                          */
                           /* fa_fwd_split_workspace_bytes(B, Hq, Sq, d_v, n_split); for          */
                           /* fa_fwd_decode_noalloc: that size exceeds FA_NOALLOC_SCRATCH_BYTES   */
} fa_status_t;

/*
 * fa_fwd -- attention forward with one head dimension d = d_qk = d_v and no LSE output.
 * Same contract as fa_fwd_ex(Q, K, V, O, NULL, B, Hq, Hkv, Sq, Sk, d, d, scale, causal, stream).
 */
fa_status_t fa_fwd(const void* Q, const void* K, const void* V, void* O, int B, int Hq, int Hkv,
                   int Sq, int Sk, int d, float scale, int causal, hipStream_t stream);

/*
 * fa_fwd_ex -- general entry point.
 *   Q, K, V   device pointers to bf16 inputs (layout above), 16-byte aligned
 *   O         device pointer to the bf16 output, 16-byte aligned
 *   LSE       device pointer to the float32 log-sum-exp output, 4-byte aligned, or NULL to skip it
 *   B, Hq, Hkv, Sq, Sk   batch, query heads, key/value heads, query length, key length (>= 0)
 *   d_qk, d_v head dimension of Q/K and of V/O
 *   scale     multiplier of the scores (the paper uses 1/sqrt(d_k)); any finite value, including
 *             0 (uniform weights over the visible keys) and negative values
 *   causal    nonzero for bottom-right causal masking
 *   stream    the HIP stream to enqueue on
 */
fa_status_t fa_fwd_ex(const void* Q, const void* K, const void* V, void* O, float* LSE, int B,
                      int Hq, int Hkv, int Sq, int Sk, int d_qk, int d_v, float scale, int causal,
                      hipStream_t stream);

/*
 * fa_fwd_split -- the same operation with every query block's key range cut into n_split parts that
 * run as separate workgroups, for shapes with too few query blocks to fill the GPU (short or few
 * query rows against long keys). This is the paper's tile-to-tile level (Alg. 2, Sec. 2.1): each
 * part runs the per-tile online softmax (Alg. 1) over its contiguous run of 64-key tiles and yields a
 * partial result; a second kernel merges the parts of every row with the log-sum-exp combination
 * (u = max over parts of u_c; each part's accumulator and row sum rescaled by exp(u_c - u) before
 * they are added), then normalises. Results agree with fa_fwd_ex within floating-point rounding.
 *
 *   Q .. stream  as in fa_fwd_ex
 *   n_split      parts per query block (>= 1). Each query block's visible key tiles are divided into
 *                n_split runs of ceil(tiles / n_split) tiles; parts left without a tile contribute
 *                nothing.
 *   workspace    device buffer owned by the caller, 16-byte aligned, at least
 *                fa_fwd_split_workspace_bytes(B, Hq, Sq, d_v, n_split) bytes; overwritten by the call
 *                (fp32 partial outputs [n_split][B][Hq][Sq][d_v], then partial LSE
 *                [n_split][B][Hq][Sq]); the caller must not touch it until the call's work on
 *                `stream` has completed. NULL is allowed only when no byte is needed.
 *   workspace_bytes  its size in bytes
 *
 * Enqueues two kernels on `stream`. Errors: n_split < 1 first (FA_ERR_BAD_SHAPE), then the checks of
 * fa_fwd_ex in their order (a degenerate size still returns FA_OK without touching the workspace),
 * then more than 2^31-1 workgroups in total or more than 2^31-1 rows B*Hq*Sq (FA_ERR_BAD_SHAPE),
 * workspace NULL or too small (FA_ERR_WORKSPACE), workspace not 16-byte aligned (FA_ERR_UNSUPPORTED).
 */
fa_status_t fa_fwd_split(const void* Q, const void* K, const void* V, void* O, float* LSE, int B,
                         int Hq, int Hkv, int Sq, int Sk, int d_qk, int d_v, float scale, int causal,
                         int n_split, void* workspace, size_t workspace_bytes, hipStream_t stream);

/* Workspace bytes fa_fwd_split needs: n_split * B * Hq * Sq * (d_v + 1) * 4; 0 when B, Hq, Sq, d_v
 * or n_split is <= 0 (nothing to store); SIZE_MAX if the count overflows. */
size_t fa_fwd_split_workspace_bytes(int B, int Hq, int Sq, int d_v, int n_split);

/*
 * fa_fwd_decode -- the same operation for decode-shaped problems, where each key/value head has few
 * query rows (one to a few new tokens per query head; best when (Hq / Hkv) * Sq <= 32). The Hq / Hkv
 * query heads that share a key/value head and their Sq rows are computed together as the columns of
 * 32-column matrix-core blocks, so K and V are read once per key/value head and block of 32 rows.
 * The key range of every (batch, key/value head, block) is cut into n_parts contiguous runs of
 * 128-key tiles that run as separate
 * workgroups (the tile-to-tile level, Alg. 2, Sec. 2.1), each running the per-tile online softmax
 * (Alg. 1); a second kernel merges the parts with the log-sum-exp combination, as fa_fwd_split does.
 * Results agree with fa_fwd_ex within floating-point rounding.
 *
 *   Q .. stream  as in fa_fwd_ex
 *   n_parts      key-range parts per (batch, key/value head, block), >= 1; parts left without a tile
 *                contribute nothing. fa_fwd_decode_parts suggests a count.
 *   workspace    device buffer owned by the caller, 16-byte aligned, at least
 *                fa_fwd_split_workspace_bytes(B, Hq, Sq, d_v, n_parts) bytes, with the layout of
 *                fa_fwd_split's workspace; overwritten by the call and not to be touched until the
 *                call's work on `stream` has completed. NULL only when no byte is needed.
 *   workspace_bytes  its size in bytes
 *
 * Enqueues two kernels on `stream` (with n_parts == 1 only the first, which writes O and LSE itself
 * and leaves the workspace untouched). Errors: n_parts < 1 (FA_ERR_BAD_SHAPE); then sizes
 * (FA_ERR_BAD_SHAPE), head dimensions (FA_ERR_UNSUPPORTED), pointers
 * (FA_ERR_NULL_POINTER), scale (FA_ERR_BAD_SCALE), alignment (FA_ERR_UNSUPPORTED), index ranges
 * (FA_ERR_BAD_SHAPE); B*Hq*Sq == 0 returns FA_OK without touching the workspace; then more than
 * 2^31-1 workgroups or 2^31-1 rows B*Hq*Sq (FA_ERR_BAD_SHAPE), workspace NULL or too small
 * (FA_ERR_WORKSPACE), workspace not 16-byte aligned (FA_ERR_UNSUPPORTED).
 */
fa_status_t fa_fwd_decode(const void* Q, const void* K, const void* V, void* O, float* LSE, int B,
                          int Hq, int Hkv, int Sq, int Sk, int d_qk, int d_v, float scale, int causal,
                          int n_parts, void* workspace, size_t workspace_bytes, hipStream_t stream);

/* Bytes of the static scratch array behind fa_fwd_decode_noalloc (32 MiB per device). */
#define FA_NOALLOC_SCRATCH_BYTES (32u << 20)

/*
 * fa_fwd_decode_noalloc -- fa_fwd_decode for callers that cannot allocate device memory (code under
 * HIP graph capture, tight serving loops, harnesses that forbid hipMalloc): the same kernels and
 * results, bit for bit, as fa_fwd_decode with the same n_parts, but the partial results live in a
 * static device array of FA_NOALLOC_SCRATCH_BYTES that the library holds on every device it runs on
 * until the process ends, instead of a caller workspace. The call allocates and frees nothing.
 *
 *   Q .. causal, n_parts   as in fa_fwd_decode
 *   stream                 the HIP stream to enqueue on; the scratch of the stream's device is used
 *                          (the current device's for the NULL stream)
 *
 * The first call on a device looks up that device's scratch address (hipGetSymbolAddress), once.
 * Every call on one device shares its scratch, and every element a call reads there it has written
 * itself first (nothing needs to start at zero). Calls that overlap in time on one device -- on two
 * streams, or from two threads without ordering -- race on the scratch and give undefined results;
 * calls ordered on one stream do not.
 *
 * Errors: n_parts < 1 (FA_ERR_BAD_SHAPE); then the checks of fa_fwd_decode in their order up to the
 * grid size (B*Hq*Sq == 0 returns FA_OK with no HIP call); then partial results of
 * fa_fwd_split_workspace_bytes(B, Hq, Sq, d_v, n_parts) > FA_NOALLOC_SCRATCH_BYTES bytes
 * (FA_ERR_WORKSPACE: fewer parts, or fa_fwd_decode with a workspace, is the remedy); a failed lookup
 * of the scratch address or a failed launch (FA_ERR_HIP).
 */
fa_status_t fa_fwd_decode_noalloc(const void* Q, const void* K, const void* V, void* O, float* LSE, int B,
                                  int Hq, int Hkv, int Sq, int Sk, int d_qk, int d_v, float scale,
                                  int causal, int n_parts, hipStream_t stream);

/* Suggested n_parts for fa_fwd_decode on a device with n_cu compute units: about one workgroup per
 * CU in total, no part shorter than 4 key tiles (512 keys), at least 1. Host arithmetic only.
 * Returns 0 if n_cu, B, Hq, Hkv or Sq <= 0, Hq % Hkv != 0 or Sk < 0. */
int fa_fwd_decode_parts(int n_cu, int B, int Hq, int Hkv, int Sq, int Sk);

/* Suggested n_split for fa_fwd_split on a device with n_cu compute units: about two workgroups per
 * CU over all parts, no part shorter than 8 key tiles (512 keys), at least 1 (1 means the single
 * pass fa_fwd_ex is the better call). Host arithmetic only, no HIP call. Returns 0 for unsupported
 * head dimensions or n_cu, B, Hq, Sq <= 0 or Sk < 0. */
int fa_fwd_split_parts(int n_cu, int B, int Hq, int Sq, int Sk, int d_qk, int d_v, int causal);

/*
 * Layer-by-layer (unfused) attention -- the paper's diagnostic baseline mapping (Sec. "Diagnostic
 * Baseline: Unfused Layer-by-Layer Attention"): the same operation as three operators dispatched
 * one after another, each reading its input from device memory and writing its result back, with
 * the intermediates in bfloat16 (Table 3 lists the score matrix QK^T and the probability matrix
 * among what this mapping spills):
 *
 *   fa_lbl_scores:   S[b,h,i,j] = bf16(scale * q_i . k_j)                (fp32 accumulation, RNE)
 *   fa_lbl_softmax:  LSE[b,h,i] = ln sum over visible j of exp(S[b,h,i,j]);
 *                    P[b,h,i,j] = bf16(exp(S[b,h,i,j] - LSE[b,h,i])) for visible j, 0 for masked j
 *   fa_lbl_pv:       O[b,h,i,:] = bf16(sum over j of P[b,h,i,j] * V[b,g,j,:])  (fp32 accumulation)
 *
 * It exists to measure what fusion saves; fa_fwd_ex is the operation's fast path. Results differ
 * from fa_fwd_ex by the roundings of S and P: per output row at most
 * max|V| * ((1 + u)^2 * exp(2 u M) - 1) with u = 2^-8 and M the row's largest visible |score|, plus
 * fp32 accumulation error.
 *
 * Spill buffers S and P: bf16 [B][Hq][Sq][ld] with row stride ld = fa_lbl_ld(Sk) (Sk rounded up to
 * 64), 16-byte aligned, owned by the caller. Row extents: query rows are taken in blocks of 128
 * (rows 128*c .. 128*c+127 of a head); let n be the number of keys visible to the last row of the
 * block (Sk without causal masking); the block's extent is E = 64 * ceil(n / 64) <= ld.
 *   - fa_lbl_scores writes S[i][j] for j < E (unmasked values, also past the diagonal) and nothing
 *     else of S;
 *   - fa_lbl_softmax reads S[i][j] for visible j (j < ld otherwise unread), writes P[i][j] for every
 *     j < E (0 for masked j) and nothing else of P; P may be the same buffer as S (in place) or
 *     disjoint from it, but must not partly overlap it;
 *   - fa_lbl_pv reads P[i][j] and V rows j for j < E only (V rows j >= Sk count as zeros).
 * Causal masking and GQA as for fa_fwd_ex. Supported dimensions: d_qk in {64, 128, 192} for the
 * scores, d_v in {64, 128} for P V; Sk <= 2^22.
 *
 * Errors (host checks, in this order; on error nothing is launched): sizes as for fa_fwd_ex or
 * Sk > 2^22 (FA_ERR_BAD_SHAPE), head dimension not supported (FA_ERR_UNSUPPORTED), a NULL buffer
 * that has elements (FA_ERR_NULL_POINTER; LSE may be NULL), scale not finite (FA_ERR_BAD_SCALE), a
 * pointer not 16-byte aligned or LSE not 4-byte aligned (FA_ERR_UNSUPPORTED). B*Hq*Sq == 0 returns
 * FA_OK without a launch. Each operator enqueues one kernel on `stream`.
 */
fa_status_t fa_lbl_scores(const void* Q, const void* K, void* S, int B, int Hq, int Hkv, int Sq, int Sk,
                          int d_qk, float scale, int causal, hipStream_t stream);
fa_status_t fa_lbl_softmax(const void* S, void* P, float* LSE, int B, int Hq, int Sq, int Sk, int causal,
                           hipStream_t stream);
fa_status_t fa_lbl_pv(const void* P, const void* V, void* O, int B, int Hq, int Hkv, int Sq, int Sk, int d_v,
                      int causal, hipStream_t stream);

/* Row stride ld (elements) of the spill buffers: Sk rounded up to 64; -1 if Sk < 0 or Sk > 2^22. */
int fa_lbl_ld(int Sk);

/* Bytes of spill buffer for the whole problem, B * Hq * Sq * ld * 2; 0 if B, Hq, Sq or Sk <= 0;
 * SIZE_MAX if Sk > 2^22 or the count overflows. */
size_t fa_lbl_workspace_bytes(int B, int Hq, int Sq, int Sk);

/*
 * fa_fwd_unfused -- the three layer-by-layer operators in sequence on `stream`, producing O and
 * (optionally) LSE like fa_fwd_ex. The score matrix and then, in place, the probabilities of a
 * chunk of the problem live in `workspace` (caller-owned device memory, 16-byte aligned,
 * overwritten; not to be touched until the work on `stream` has completed). A chunk is as many whole
 * query heads as fit (a multiple of Hq / Hkv heads when more than that many fit) or, when one head
 * does not fit, as many blocks of 128 query rows of one head as fit; each chunk is three launches.
 * workspace_bytes >= fa_lbl_workspace_bytes(B, Hq, Sq, Sk) runs the whole problem as one chunk;
 * the least accepted is min(Sq, 128) * fa_lbl_ld(Sk) * 2. Supported dimensions: d_qk in
 * {64, 128, 192}, d_v in {64, 128}.
 *
 * Errors: as for the operators (sizes, head dimensions, pointers, scale, alignment of Q, K, V, O,
 * LSE), then workspace NULL or smaller than the least size (FA_ERR_WORKSPACE), then workspace not
 * 16-byte aligned (FA_ERR_UNSUPPORTED). B*Hq*Sq == 0 returns FA_OK without touching the workspace.
 * With Sk == 0 no workspace is needed and every row gets O = 0, LSE = -inf.
 */
fa_status_t fa_fwd_unfused(const void* Q, const void* K, const void* V, void* O, float* LSE, int B, int Hq,
                           int Hkv, int Sq, int Sk, int d_qk, int d_v, float scale, int causal,
                           void* workspace, size_t workspace_bytes, hipStream_t stream);

/*
 * Paged key/value cache. A serving program keeps the keys and values of its sequences in pages of page_size
 * tokens that lie anywhere in two buffers; a block table names the pages of every sequence in order: key j of
 * sequence b is slot j % page_size of page block_table[b][j / page_size]. The T new tokens of a call are packed, those
 * of sequence b being tokens q_starts[b] .. q_starts[b + 1] - 1, and are the last of its kv_lens[b] keys: token i of
 * n new ones is at position kv_lens[b] - n + i. fa_kv_append writes the keys and values of new tokens to the cache (and
 * turns keys and queries by their positions); fa_fwd_paged is their attention over it.
 *
 * Block table, kv_lens, q_starts and scales are device arrays that the host does not read. The kernels read and
 * write inside the buffers whatever is in them:
 *   - kv_lens[b] counts as clamped to [0, max_blocks * page_size], q_starts[b] to [0, T]; q_starts must not
 *     decrease (else the results of the call are undefined); q_starts[b] == q_starts[b + 1] is a sequence without
 *     new tokens; tokens before q_starts[0] or from q_starts[B] on belong to no sequence, and their rows of every
 *     output are left as they were;
 *   - entries of the table behind a sequence's last key are not used; a page number outside [0, n_pages) is a page
 *     that is not there: nothing is written to it, and its keys are not visible;
 *   - slots behind a sequence's last key are not read into any result (whatever bits they hold).
 * Pages may be shared for reading; a page that the new tokens of two sequences are written to (or the same table
 * entry twice in one sequence's written range) gets one of the two tokens in each 16 bytes, whichever comes last.
 */
typedef enum {
  FA_CACHE_BF16 = 0, /* bf16 */
  FA_CACHE_E4M3 = 1  /* 8-bit floats (OCP e4m3), times a scale per key/value head */
} fa_cache_type_t;

/* The cache: K is [n_pages][Hkv][page_size][d_qk] and V the same with d_v, in any order of the first three
 * dimensions: element (page, head, slot, 0) lies at page * k_page + head * k_head + slot * k_slot, its d elements one
 * after the other. Strides are in elements, not negative, a multiple of 16 bytes; k_slot >= d_qk, v_slot >= d_v, and a
 * slot stride times 16 is below 2^31 bytes. page_size is a power of two from 16 to 2^20. An element of an e4m3 cache
 * stands for its value times k_scale[head] (v_scale[head]); NULL stands for ones, and bf16 caches take NULL. */
typedef struct {
  void* K;
  void* V;
  const float* k_scale;
  const float* v_scale;
  long long k_page, k_head, k_slot, v_page, v_head, v_slot;
  int n_pages, page_size, Hkv, d_qk, d_v;
  int type; /* fa_cache_type_t */
} fa_paged_cache_t;

/* The batch: int32 arrays block_table [B][max_blocks] (rows table_stride elements apart), kv_lens [B] and q_starts
 * [B + 1], and the number of packed tokens T. */
typedef struct {
  const int* block_table;
  long long table_stride;
  const int* kv_lens;
  const int* q_starts;
  int B, max_blocks, T;
} fa_paged_batch_t;

/*
 * fa_kv_append -- write the keys and values of the new tokens to the cache, turning keys (and queries) by the
 * position rotation on the way.
 *   cache, batch     as above; kv_lens counts the new tokens already
 *   K, V             bf16 [T][Hkv][d_qk], [T][Hkv][d_v]; element (t, h, 0) at t * k_token + h * k_head
 *   Q, Q_out, Hq     bf16 [T][Hq][d_qk] likewise, or Hq = 0 for none; Q_out is Q itself (same strides) or does not
 *                    overlap it
 *   strides          {q_token, q_head, qo_token, qo_head, k_token, k_head, v_token, v_head}, in elements, multiples of 8
 *   cos_sin          float32 [n_pos][rot_dim], 16-byte aligned: the cosines of a position's rot_dim / 2 angles, then
 *                    their sines; NULL with rot_dim = 0 for no rotation
 *   rot_begin, rot_dim  the dims that turn. interleaved == 0: dim rot_begin + c pairs with rot_begin + rot_dim / 2 + c
 *                    (rot_dim a multiple of 16); else 2c with 2c + 1 (a multiple of 8). rot_begin is a multiple of 8.
 * A pair (x, y) becomes (x cos - y sin, y cos + x sin), computed in fp32 and rounded once, to bf16 or, for an
 * e4m3 cache, after division by the head's scale to e4m3 (nearest even; what passes +-448 becomes +-448, NaN
 * stays NaN). V, and dims that do not turn, are copied (or divided and rounded). n_pos >= max_blocks * page_size, so that
 * every position has its row. A token before position 0 (more new tokens than keys) is left out, and nothing is
 * written for it. Neither inputs nor Q_out may overlap the cache, nor Q_out K
 * or V. Enqueues one kernel.
 *
 * Errors, in this order: cache, batch, strides or cos_sin description NULL (FA_ERR_NULL_POINTER); sizes (FA_ERR_BAD_SHAPE:
 * negative (table_stride too), Hkv <= 0 with T > 0, Hq not a multiple of Hkv, max_blocks * page_size > 2^30, T * Hq >= 2^31,
 * B > 2^31 - 65, n_pos too small, the rotated dims outside [0, d_qk)); head dimensions, page size, type or rotation not supported
 * (FA_ERR_UNSUPPORTED); a NULL buffer that has elements (FA_ERR_NULL_POINTER); alignment (FA_ERR_UNSUPPORTED: 16 bytes for
 * buffers and strides, 4 for the int and scale arrays); cache strides negative, too large, or letting two elements of the cache
 * overlap (FA_ERR_BAD_SHAPE). T == 0 or B == 0 returns FA_OK without a launch.
 */
fa_status_t fa_kv_append(const fa_paged_cache_t* cache, const fa_paged_batch_t* batch, const void* K, const void* V,
                         const void* Q, void* Q_out, int Hq, const long long* strides, const float* cos_sin, int n_pos,
                         int rot_begin, int rot_dim, int interleaved, hipStream_t stream);

/*
 * Positions by device arrays: token t stands at positions[t * token + a * axis] on axis a of n_axes (int32), for images and
 * video (time, height, width) and for drafted tokens, whose place in the cache is not their position. pair_axes
 * (uint8, 4-byte aligned, one for each of the rot_dim / 2 pairs) names the axis whose position turns a pair; NULL: the first.
 * Strides in elements, 0 to 2^40; `batch` is that of the batch in fa_rotate, and unused elsewhere. The device clamps: an axis
 * behind the last counts as the last, a position outside the table of angles as its first or last row.
 */
typedef struct {
  const int* positions;
  const unsigned char* pair_axes;
  long long batch, token, axis;
  int n_axes;
} fa_positions_t;

/*
 * fa_kv_append_at -- fa_kv_append with the angles by `positions` (token t: the packed one) instead of the tokens' places
 * among their sequences' keys. What it writes where is the same. n_pos >= 1 rows of angles with rot_dim > 0.
 * Errors: positions NULL (FA_ERR_NULL_POINTER), then as fa_kv_append, with n_axes < 1 and strides out of range among the
 * sizes, NULL arrays and alignment (4 bytes) of the positions among the others.
 */
fa_status_t fa_kv_append_at(const fa_paged_cache_t* cache, const fa_paged_batch_t* batch, const void* K, const void* V,
                            const void* Q, void* Q_out, int Hq, const long long* strides, const fa_positions_t* positions,
                            const float* cos_sin, int n_pos, int rot_begin, int rot_dim, int interleaved, hipStream_t stream);

/*
 * fa_rotate -- the position rotation of fa_kv_append for queries or keys that are in no cache (bf16): Y[b,h,s] is X[b,h,s] with
 * the pairs of its dims rot_begin .. rot_begin + rot_dim - 1 turned, its other dims copied. inverse != 0 turns by the negative
 * angles, which takes a rotation back and is its gradient.
 *   X, Y        element (b, h, s, 0) at b * strides[0] + h * strides[1] + s * strides[2], of Y likewise by strides[3 .. 5]; in
 *               elements, multiples of 8. Y is X itself with the same strides, or does not overlap it
 *   d           a multiple of 8, up to 1024
 *   positions   of token (b, s); NULL, or positions->positions NULL: token s stands at s (n_pos >= S)
 *   cos_sin, n_pos, rot_begin, rot_dim, interleaved   as in fa_kv_append
 * Enqueues one kernel. Errors, in this order: strides NULL (FA_ERR_NULL_POINTER); sizes (FA_ERR_BAD_SHAPE: negative,
 * B * H * S >= 2^31, rotated dims outside [0, d), n_pos, positions as above); d or rotation not supported
 * (FA_ERR_UNSUPPORTED); NULL buffers (FA_ERR_NULL_POINTER); alignment (FA_ERR_UNSUPPORTED: 16 bytes for buffers, strides and cos_sin, 4
 * for the positions). No element returns FA_OK without a launch.
 */
fa_status_t fa_rotate(const void* X, void* Y, int B, int H, int S, int d, const long long* strides,
                      const fa_positions_t* positions, const float* cos_sin, int n_pos, int rot_begin, int rot_dim,
                      int interleaved, int inverse, hipStream_t stream);

/* Most 32-bit words of a row of a tree's mask (2048 drafted tokens), and most tokens of a tree of fa_tree_mask. */
#define FA_TREE_WORDS 64
#define FA_TREE_TOKENS 4096

/*
 * fa_tree_mask -- mask and positions of trees of drafted tokens, as fa_fwd_paged_ex and fa_kv_append_at take them. The new tokens
 * of sequence b (by q_starts and kv_lens as above, kv_lens counting them, clamped to max_keys) are a tree: token i's
 * parent is token parents[t] of the same sequence, one before it; anything else (-1) makes it a root, whose
 * parent is the last cached key. Bit j % 32 of word j / 32 of mask[t] is set where token j is token t itself or an ancestor (those
 * from 32 * words on have no bit); positions[t] = kv_lens[b] - n + its number of ancestors, for the n new ones.
 *   parents, mask, positions   int32 [T], 32-bit words [T] in rows mask_stride apart, int32 [T]; the outputs overlap neither each other
 *               nor an input
 * Rows of tokens that belong to no sequence, or to one of more than FA_TREE_TOKENS new tokens, are left as they were. Enqueues
 * one kernel.
 * Errors: sizes (FA_ERR_BAD_SHAPE: negative, max_keys > 2^30, words outside [1, FA_TREE_WORDS], mask_stride < words), NULL
 * arrays (FA_ERR_NULL_POINTER), alignment of 4 bytes (FA_ERR_UNSUPPORTED). T == 0 or B == 0 returns FA_OK without a launch.
 */
fa_status_t fa_tree_mask(const int* parents, const int* q_starts, const int* kv_lens, int B, int T, int max_keys, void* mask,
                         int words, long long mask_stride, int* positions, hipStream_t stream);

/*
 * fa_kv_compact -- close up the new tokens that a sequence keeps (of drafted ones those that were accepted): of the n new tokens
 * of sequence b, which are in the cache, number kept[b][i] moves to the i-th place behind its cached keys, key kv_lens[b] - n + i, for
 * i < n_kept[b]; kv_lens_out[b] = kv_lens[b] - n + n_kept[b]. Keys keep the rotation that they were written with.
 *   cache, batch    as above (T is not used: there are no packed tokens here)
 *   kept            int32 [B][max_kept], rows kept_stride apart: numbers of new tokens, which increase (else the moved keys hold
 *                   what any of the sequence's new tokens held); one outside [0, n) moves nothing
 *   n_kept          int32 [B], clamped to [0, min(max_kept, n)]
 *   kv_lens_out     int32 [B], apart from all inputs
 * Nothing moves to or from a page that is not there. A cache whose layers lie in one buffer, [n_pages][layers][Hkv] .., closes up in
 * one call with layers * Hkv heads. Enqueues one kernel. Errors: as fa_kv_append's of cache and batch, in that order (sizes
 * also: max_kept or kept_stride < 0, Hkv >= 2^25; behind what is supported: B * ceil(Hkv * (d_qk + d_v) * element bytes /
 * 4096) >= 2^24). B == 0 returns FA_OK without a launch.
 */
fa_status_t fa_kv_compact(const fa_paged_cache_t* cache, const fa_paged_batch_t* batch, const int* kept, long long kept_stride,
                          int max_kept, const int* n_kept, int* kv_lens_out, hipStream_t stream);

/*
 * fa_kv_copy -- copy pages: keys and values of all heads and slots of page src[i] to page dst[i], i < n (int32 device arrays), for
 * sequences that fork and write on in pages of their own. A pair with a page number outside [0, n_pages) or of one page
 * does nothing. A page that is copied to twice, or copied to and from, holds afterwards, 16 bytes by 16 bytes, what any order of
 * the copies could leave. The scales of an e4m3 cache are per head and stay. Layers in one buffer count as heads, as above.
 * Enqueues one kernel. Errors: cache NULL (FA_ERR_NULL_POINTER); sizes (FA_ERR_BAD_SHAPE); head dimensions, page size or type
 * not supported (FA_ERR_UNSUPPORTED); NULL buffers (FA_ERR_NULL_POINTER); alignment (FA_ERR_UNSUPPORTED); cache strides, or
 * n * ceil(Hkv * page_size * max(d_qk, d_v) * element bytes / 4096) >= 2^24 (FA_ERR_BAD_SHAPE). n == 0 returns FA_OK
 * without a launch.
 */
fa_status_t fa_kv_copy(const fa_paged_cache_t* cache, const int* src, const int* dst, int n, hipStream_t stream);

/* The kernels of fa_fwd_paged: one reads K and V once per 32 or 64 row-heads of a key/value head (query rows times the
 * heads that share it) and splits every sequence over the chip, for single tokens, draft tokens and short prompts; one computes
 * in blocks of 128 or 256 row-heads, for longer prompts and chunks. Each is right for any lengths. */
typedef enum {
  FA_PAGED_AUTO = 0, /* chosen by max_q, the sizes and, on the device, the lengths */
  FA_PAGED_FEW = 1,
  FA_PAGED_MANY = 2
} fa_paged_path_t;

/*
 * fa_fwd_paged -- attention of the new tokens over the paged cache: for token t of sequence b at position p,
 *     O[t,h] = softmax over visible j of (scale * q[t,h] . K[b,g,j]) * V[b,g,j],   g = h / (Hq / Hkv),
 * j <= p when causal, j < kv_lens[b] else. Arithmetic as for fa_fwd_ex (e4m3 caches: K and V are widened exactly, P is
 * rounded to fp16, by 2^-11 of it or 2^-32 of the row's largest at most). A row with no visible key, or whose sum is no
 * number, gets O = 0, LSE = -inf. An infinity or a NaN in a key reaches only the rows that see the key; one in a value may
 * reach other rows of its sequence.
 *   Q, O        bf16 [T][Hq][d_qk], [T][Hq][d_v]; element (t, h, 0) at t * q_token + h * q_head
 *   LSE         float32 [T][Hq] (contiguous), or NULL
 *   strides     {q_token, q_head, o_token, o_head}, in elements, multiples of 8. O and LSE overlap neither each other nor
 *               an input (O may be Q itself with the same strides, where d_qk = d_v)
 *   max_q       the most new tokens of one sequence, as far as the host knows, 0 if it does not: it helps to choose the
 *               kernels, the results are right for any
 *   path        fa_paged_path_t
 *   workspace   16-byte aligned, at least fa_fwd_paged_workspace_bytes(...) bytes, overwritten; nothing needs to be in
 *               it before, and it must not be used elsewhere until the call's work has completed. NULL only when no
 *               byte is needed.
 * The work is cut on the device by the lengths found there, so one captured call serves whatever lengths the arrays
 * hold at a replay.
 *
 * Errors, in this order: cache, batch or strides NULL (FA_ERR_NULL_POINTER); sizes (FA_ERR_BAD_SHAPE: as for fa_kv_append, max_q < 0,
 * Hkv * (T * Hq / Hkv / 32 + B) * (max_blocks * page_size / 128 + 2) >= 2^31, with FA_PAGED_MANY also
 * Hkv * (rows / 128 + min(B, rows)) >= 2^24 for rows = T * Hq / Hkv); head dimensions, page size, type, path
 * (FA_ERR_UNSUPPORTED); NULL buffers (FA_ERR_NULL_POINTER); scale (FA_ERR_BAD_SCALE); alignment (FA_ERR_UNSUPPORTED); cache
 * strides (FA_ERR_BAD_SHAPE); workspace NULL or too small (FA_ERR_WORKSPACE), not aligned (FA_ERR_UNSUPPORTED). T == 0, B == 0 or
 * Hq == 0 returns FA_OK without a launch.
 */
fa_status_t fa_fwd_paged(const fa_paged_cache_t* cache, const fa_paged_batch_t* batch, const void* Q, void* O, float* LSE,
                         int Hq, const long long* strides, int max_q, int path, float scale, int causal, void* workspace,
                         size_t workspace_bytes, hipStream_t stream);

/* Workspace bytes of a fa_fwd_paged call with these sizes, max_keys = max_blocks * page_size, this max_q and this path (they do
 * not depend on the lengths; 0 is possible). Host arithmetic only; 0 for sizes <= 0 (max_keys, max_q: < 0), Hq not a multiple of
 * Hkv, or an unsupported type, path or head dimension. */
size_t fa_fwd_paged_workspace_bytes(int B, int T, int max_keys, int Hq, int Hkv, int d_qk, int d_v, int type, int max_q,
                                    int path);

/* The largest cap of scores. */
#define FA_MAX_SOFTCAP 1024.0f

/*
 * How fa_fwd_paged_ex changes scores and hides keys. For the token at position p (its place among its sequence's kv_lens[b] keys)
 * and key j, with x = scale * q . k:
 *   softcap      > 0: x becomes softcap * tanh(x / softcap), up to FA_MAX_SOFTCAP; 0: none
 *   slopes       float32 [Hq] or NULL: then slopes[h] * |p - j| is taken off (a slope beyond +-2^96 / log2(e), 5e28, counts as that)
 *   window       > 0: key j is hidden where |p - j| >= window (the token itself counts); 0: none
 *   prefix_lens  int32 [B] or NULL: keys j < prefix_lens[b] (clamped to [0, kv_lens[b]]) are visible to all tokens of the
 *                sequence, whatever window and causal masking say: a bidirectional prefix, or first tokens kept beside a window
 *   tree_mask    32-bit words [T][mask_words], rows mask_stride >= mask_words apart, up to FA_TREE_WORDS words; or NULL. The new tokens
 *                are drafted ones: token t sees all cached keys j < kv_lens[b] - n, and the sequence's i-th new token where
 *                bit i % 32 of word i / 32 is set (new tokens from 32 * mask_words on are hidden). Only causal calls, and not with
 *                slopes, a window or a prefix, whose distances would be those of places in the cache.
 */
typedef struct {
  float softcap;
  int window;
  const float* slopes;
  const int* prefix_lens;
  const void* tree_mask;
  long long mask_stride;
  int mask_words;
} fa_paged_scores_t;

/*
 * fa_fwd_paged_ex -- fa_fwd_paged with `scores` (NULL, or nothing in it set: fa_fwd_paged). Keys that no token of a block sees,
 * such as those before its window, are mostly not read. Keys that are hidden from a row reach neither its O nor its LSE, except that,
 * as in fa_fwd_paged, an infinity or a NaN in a value may. A capped score is off by up to 2^-22 softcap, which is
 * why caps are bounded. The workspace has fa_fwd_paged_ex_workspace_bytes(...) bytes.
 * Errors: as fa_fwd_paged, with a negative window, mask_words and mask_stride out of range among the sizes, the combinations
 * above FA_ERR_UNSUPPORTED among what is supported, a softcap that is negative, no number or too large FA_ERR_BAD_SCALE behind the
 * scale, and an alignment of 4 bytes of the arrays.
 */
fa_status_t fa_fwd_paged_ex(const fa_paged_cache_t* cache, const fa_paged_batch_t* batch, const fa_paged_scores_t* scores,
                            const void* Q, void* O, float* LSE, int Hq, const long long* strides, int max_q, int path,
                            float scale, int causal, void* workspace, size_t workspace_bytes, hipStream_t stream);

/* Workspace bytes of a fa_fwd_paged_ex call with these sizes, whatever its scores; as fa_fwd_paged_workspace_bytes. */
size_t fa_fwd_paged_ex_workspace_bytes(int B, int T, int max_keys, int Hq, int Hkv, int d_qk, int d_v, int type, int max_q,
                                       int path);

/* Static, human-readable name of a status code ("FA_OK", ...); "unknown status" otherwise. */
const char* fa_status_str(fa_status_t s);

/* Query rows per workgroup of the fused kernel's long instance for the given head dimensions when a
 * workgroup holds one query head (256); 0 if unsupported. It runs every (192, 128) problem, and at
 * (d_qk, d_v) = (64, 64) or (128, 128) problems with more such blocks (B * Hq * ceil(Sq / rows)) than
 * the other instances take (fa_fwd_rows) and split mode where blocks of half the rows would neither pad
 * fewer rows nor fill more compute units (fa_fwd_instance). When Hq / Hkv is divisible
 * by 2 or 4 a workgroup holds that many query heads of one key/value head with a half or a quarter of
 * these rows each. Host arithmetic only. */
int fa_block_rows(int d_qk, int d_v, int causal);

/* Query rows per block holding one query head of the fused-kernel instance that the grid alone (B
 * batches, Hq query heads, Sq query rows) selects for fa_fwd and fa_fwd_ex without split mode:
 * 256 (long instance: one workgroup per compute unit, two at d = 64), 128 (short instance: two per
 * compute unit, at most 1024 blocks at d = 64 and 256 at d = 128, i.e. blocks of the long instance's
 * rows) or 64 (key parts: the wave sets of a workgroup take the parts of every key tile and merge their
 * results at the end; causal problems of at most 320 blocks at d = 64 and 192 at d = 128, others of at
 * most 64 and 128). A call with more than twice as many keys as query rows may run another one, which
 * this function, having no Sk, cannot tell: fa_fwd_instance does. 0 for unsupported head dimensions or
 * negative sizes. Host arithmetic only. */
int fa_fwd_rows(int B, int Hq, int Sq, int d_qk, int d_v, int causal);

/* The fused kernel's instances. Each computes the same function (Eq. (1) by Alg. 1); which one runs
 * follows from the sizes alone. */
typedef enum {
  FA_INSTANCE_NONE = 0,        /* unsupported or invalid sizes, or no query row */
  FA_INSTANCE_QUARTERS = 1,    /* 32-row workgroups, four waves on the quarters of every 128-key tile */
  FA_INSTANCE_HALVES = 2,      /* 64 row-heads per workgroup, two wave sets on the halves of every 64-key tile */
  FA_INSTANCE_SHORT = 3,       /* 128 row-heads per workgroup */
  FA_INSTANCE_SHORT_WIDE = 4,  /* the same with 128-key tiles (d = 64) */
  FA_INSTANCE_LONG = 5         /* 256 row-heads per workgroup */
} fa_instance_t;

/* The instance that fa_fwd and fa_fwd_ex (n_split == 0) or fa_fwd_split (n_split >= 1) launch for these
 * sizes, decided by the code that launches it. Host arithmetic only. */
fa_instance_t fa_fwd_instance(int B, int Hq, int Hkv, int Sq, int Sk, int d_qk, int d_v, int causal, int n_split);

#ifdef __cplusplus
}
#endif

#endif /* FA_MI355X_FA_H */
