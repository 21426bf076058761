/*
 * msa.h -- C ABI of libmsa.so, the MI355X (gfx950) inference hot path of
 * MiniMax Sparse Attention (MSA).
 *
 * The paper factors sparse attention into an indexer that picks which keys a
 * query attends to and an exact attention over the picked keys (Sec. 2.2,
 * two-stage equation).  MSA's indexer is block- and GQA-group-granular
 * (Sec. 2.3; Sec. 3.1 "Index Branch"); its attention runs only over the
 * selected blocks (Sec. 3.1 "Main Branch").  The library exports one call per
 * stage and per inference phase:
 *
 *   msa_index_topk           Index Branch: block scores + Top-k (prefill and decode)
 *   msa_block_topk           the Top-k operator alone, on a score matrix the caller holds
 *   msa_sparse_attn_prefill  Main Branch for many query rows per sequence
 *   msa_sparse_attn_decode   Main Branch for one query row per sequence
 *   msa_sparse_attn_*_fp8    Main Branch on e4m3 queries and KV cache
 *   msa_dense_attn           dense causal GQA attention (the comparison baseline)
 *   msa_sparse_attn_backward training: Main Branch gradients dQ, dK, dV
 *   msa_sparse_kl_backward   training: sparse KL loss and its index-projection gradients
 *
 * and what a layer needs around them:
 *
 *   msa_qk_norm_rope(_fp8)   RMS norm of each query and key head and the rotation by position
 *   msa_qk_norm_rope_backward   its gradients
 *   msa_kv_append(_fp8)      new keys, values and index keys into the (paged) cache
 *   msa_dense_attn_paged(_fp8)   dense causal attention over a paged cache
 *
 * and the same for layers whose keys and values come from one latent vector per token:
 *
 *   msa_latent_append(_fp8)  latents and shared key parts into the (paged) cache
 *   msa_latent_attn_paged(_fp8)   attention on that cache (absorbed form)
 *   msa_latent_attn          attention on per-head keys and values (expanded form)
 *   msa_latent_attn_backward its gradients
 *
 * Conventions shared by every call
 * --------------------------------
 * - Every tensor argument is a DEVICE pointer to contiguous row-major memory
 *   that the caller allocates, owns and keeps alive until the stream has
 *   executed the call.  bf16 tensors hold IEEE bfloat16 bit patterns.
 * - Calls are asynchronous on `stream` (0 = the null stream): they validate
 *   their arguments on the host, launch kernels and return.  Results are
 *   valid once the stream has reached them.  Nothing is launched when a call
 *   returns an error.  No call synchronises the host with the device.
 * - No call allocates device memory.  Calls that need scratch space take a
 *   caller-provided `workspace` of at least the size returned by the matching
 *   *_workspace_size() query; the workspace is free again once the stream has
 *   executed the call.  Calls that share a workspace must be ordered on one
 *   stream.  (msa_index_topk_noalloc uses the library's static device array
 *   instead, see below.)
 * - Global state: the opt-in kernel timing at the end of this header, the
 *   grid size of each persistent kernel (derived from the device's occupancy
 *   on first use and cached in an atomic), and msa_index_topk_noalloc's
 *   file-scope device scratch array with its per-device address table.
 *   Concurrent calls from several host threads are safe when they use
 *   distinct outputs and workspaces (msa_index_topk_noalloc calls on one GPU
 *   share its scratch array and must not overlap).
 * - NaN or Inf inputs give unspecified (but memory-safe) results.  In the sparse
 *   forward calls they stay local: a row that does not list a key block is not
 *   touched by what the block holds.
 *
 * Sequence layout (struct msa_seqs)
 * ---------------------------------
 * A batch holds `num_seqs` sequences.  Sequence s owns the packed query rows
 * q_offsets[s] .. q_offsets[s+1]-1 of the query-side tensors (index_q, q, o,
 * lse, block_ids) and key rows kv_starts[s] .. kv_starts[s]+kv_lens[s]-1 of
 * the key-side tensors (index_k, k, v).  Query row t of sequence s (t counted
 * from 0 inside the sequence) sits at absolute position
 *     p = kv_lens[s] - (q_offsets[s+1] - q_offsets[s]) + t,
 * i.e. its own key is already in the cache.  This covers prefill
 * (q rows == kv_len), chunked prefill (rows appended to a cached context) and
 * decode (one row per sequence; kv_starts may then point into a padded cache,
 * e.g. s * max_len).  Key block b of a sequence holds its keys
 * b*block_size .. min((b+1)*block_size, kv_len)-1 (Sec. 2.3, block equation);
 * the local block of position p is p / block_size.  Rows of several tokens per
 * sequence after a cached context (speculative / multi-token decode) are the
 * chunked-prefill case with a few rows.
 *
 * Paged key side (optional): with block_table != NULL the key-side tensors
 * (index_k, k, v) are a pool of pages of page_size rows; key j of sequence s
 * is row page * page_size + j % page_size with
 * page = block_table[s * block_table_stride + j / page_size] (kv_starts is
 * then ignored and may be NULL).  page_size must be block_size times 1, 2, 4,
 * ... or 64 for the call's block_size; kv_lens[s] <= block_table_stride *
 * page_size.  Page ids outside [0, total_kv_rows /
 * page_size) are clamped into it (results unspecified, memory safe).  This
 * is a serving layout, not part of the paper.  Every call accepts it except
 * msa_dense_attn, which returns MSA_ERR_UNSUPPORTED for a paged layout
 * (msa_dense_attn_paged takes it; that call and msa_kv_append, which have no
 * block size, accept any power of two from 16 to 8192 as page_size; so do
 * msa_latent_append and msa_latent_attn_paged, while msa_latent_attn and its
 * backward are for a contiguous key side); the
 * training calls then write dK, dV and d index_k in the pool's rows (rows of
 * pages no sequence lists get zero; keys in pages shared by several
 * sequences get the sum of their gradients).
 */
#ifndef MSA_H_
#define MSA_H_

#include <stddef.h>
#include <stdint.h>

#include <hip/hip_runtime_api.h>

#ifdef __cplusplus
extern "C" {
#endif

/* Status codes returned by every int-valued call. */
#define MSA_OK 0
#define MSA_ERR_INVALID (-1)     /* null pointer, negative or inconsistent size, H_q % H_kv != 0 ... */
#define MSA_ERR_UNSUPPORTED (-2) /* a valid shape the library has no kernel for */
#define MSA_ERR_WORKSPACE (-3)   /* workspace smaller than the *_workspace_size() value */
#define MSA_ERR_HIP (-4)         /* a HIP launch failed (the HIP error is consumed) */

typedef struct msa_seqs {
  int32_t num_seqs;          /* host: number of sequences, >= 1 */
  int64_t total_q_rows;      /* host: rows of the query-side tensors (= q_offsets[num_seqs]) */
  int64_t total_kv_rows;     /* host: rows of the key-side tensors; every key access is
                                kept below this bound */
  int32_t max_q_rows;        /* host: upper bound of q_offsets[s+1]-q_offsets[s] */
  int32_t max_kv_len;        /* host: upper bound of kv_lens[s] */
  const int32_t* q_offsets;  /* device [num_seqs+1], non-decreasing, q_offsets[0] == 0 */
  const int64_t* kv_starts;  /* device [num_seqs], >= 0 (unused when paged) */
  const int32_t* kv_lens;    /* device [num_seqs], >= the sequence's query rows */
  const int32_t* block_table;   /* device [num_seqs, block_table_stride] page ids, or NULL
                                   (contiguous key side) */
  int32_t block_table_stride;   /* host: entries (pages) per sequence of block_table */
  int32_t page_size;            /* host: key rows per page (block_size x 2^j, j <= 6) */
} msa_seqs;

/* Human-readable text of a status code (static storage). */
const char* msa_strerror(int status);

/* ------------------------------------------------------------------------
 * Index Branch: msa_index_topk
 *
 * Sec. 3.1, index-score equation: for query position i of group r and key j,
 * S_ij = q_idx[i, r, :] . k_idx[j, :] / sqrt(d_idx); a key block scores the
 * maximum of S over its causally visible tokens (j <= i).  Sec. 3.1, top-k
 * equation and Sec. 3.2 "Local Block": each (query row, group) keeps the
 * local block i / block_size plus the top-k-1 other causal blocks.  Selection
 * ranks the raw dot products (Sec. 4.1 "Exp-free selection": neither the
 * softmax nor the positive scale changes the order); equal scores keep the
 * lower block id.
 *
 *   index_q   bf16 [total_q_rows, num_kv_heads, d_idx]   one index-query head per group
 *   index_k   bf16 [total_kv_rows, d_idx]                the single shared index-key head
 *   block_ids int32 [total_q_rows, num_kv_heads, topk]   OUTPUT: the min(topk, lb+1) selected
 *             block ids of each (row, group) in ascending order, then -1 padding.
 *
 * Supported: d_idx in {64, 128}; block_size in {64, 128}; 1 <= topk <= 64;
 * num_kv_heads a power of two <= 64.
 * ------------------------------------------------------------------------ */
size_t msa_index_topk_workspace_size(const msa_seqs* seqs, int num_kv_heads, int d_idx,
                                     int block_size, int topk);
int msa_index_topk(const void* index_q, const void* index_k, const msa_seqs* seqs,
                   int num_kv_heads, int d_idx, int block_size, int topk, int32_t* block_ids,
                   void* workspace, size_t workspace_bytes, hipStream_t stream);

/* ------------------------------------------------------------------------
 * msa_index_topk_noalloc -- msa_index_topk without a workspace argument, for
 * callers that cannot allocate device memory: code under HIP graph capture,
 * serving loops that must not call hipMalloc, harnesses that forbid it.
 *
 * Arguments, outputs (block_ids, caller-allocated), results and errors are
 * those of msa_index_topk.  The scratch space lives in a device array of the
 * library of MSA_INDEX_TOPK_NOALLOC_MAX_BYTES bytes; each GPU the call runs on
 * holds its own copy until the process ends.  The call runs on the current
 * device, and `stream` must belong to it.  It allocates nothing (no hipMalloc,
 * hipFree or allocating library routine); its first call on a device looks
 * the array's address up once.  A problem whose smallest workspace (four bytes
 * per sequence plus one unit of rows, the quantum msa_index_topk chunks by)
 * exceeds the array returns MSA_ERR_WORKSPACE and launches nothing; problems
 * larger than the array but within that bound run in several chunks.
 * Every call on a GPU shares that GPU's array: calls that overlap on one GPU
 * (several streams or host threads) race and must be serialised by the
 * caller.  Nothing in the array needs to start at zero.
 * ------------------------------------------------------------------------ */
#define MSA_INDEX_TOPK_NOALLOC_MAX_BYTES ((size_t)64 << 20)
int msa_index_topk_noalloc(const void* index_q, const void* index_k, const msa_seqs* seqs,
                           int num_kv_heads, int d_idx, int block_size, int topk,
                           int32_t* block_ids, hipStream_t stream);

/* ------------------------------------------------------------------------
 * msa_block_topk -- the Top-k operator of the Index Branch on its own, for a
 * score matrix the caller already holds (Sec. 3.1 top-k equation; Sec. 4.1
 * "Per-thread register top-k" and its latency table, which times this
 * operator on fp32 inputs of shape (N, B) with rows processed independently).
 *
 *   scores  fp32 [n_rows, ld]: columns 0 .. n_cols-1 of each row are ranked;
 *           the buffer spans n_rows * ld floats.
 *   ids     int32 [n_rows, k]  OUTPUT: the min(k, n_cols) columns of largest
 *           score of each row in ascending order, then -1 padding.  Equal
 *           scores keep the lower column; -0 equals +0; -inf ranks below
 *           every finite score like any other value.
 *
 * No block is forced and no causal limit applies (msa_index_topk adds both).
 * Supported: 1 <= k <= 64; 0 <= n_cols <= 2^30; ld >= n_cols.  NaN
 * scores give unspecified (memory-safe) ids.  No workspace.  Rows that are
 * 16-byte aligned (scores aligned, ld % 4 == 0) are read four columns per
 * lane and load; others one column per lane.
 * ------------------------------------------------------------------------ */
int msa_block_topk(const float* scores, int64_t n_rows, int n_cols, int64_t ld, int k,
                   int32_t* ids, hipStream_t stream);

/* ------------------------------------------------------------------------
 * Main Branch: msa_sparse_attn_prefill / msa_sparse_attn_decode
 *
 * Sec. 3.1, sparse-attention equation: for query row i and query head h of
 * group r = h / (num_q_heads / num_kv_heads), softmax attention with scale
 * `softmax_scale` (the paper uses 1/sqrt(head_dim); any finite value, zero and
 * negative ones included, in every call that takes one) over the causally visible
 * tokens (j <= i) of the blocks listed in block_ids[i, r, :], using key/value
 * head r.  Entries < 0 are padding; the ids of a row must be distinct; ids
 * past the local block select no token.  Every row must list a block with a
 * visible token (its local block, as msa_index_topk guarantees); a row without
 * one gets O = 0 and LSE = -inf.
 *
 *   q          bf16 [total_q_rows, num_q_heads, head_dim]
 *   k, v       bf16 [total_kv_rows, num_kv_heads, head_dim]
 *   block_ids  int32 [total_q_rows, num_kv_heads, topk]   (msa_index_topk's output)
 *   o          bf16 [total_q_rows, num_q_heads, head_dim]  OUTPUT
 *   lse        fp32 [total_q_rows, num_q_heads]            OUTPUT, natural log of the
 *              softmax denominator including the scale (Sec. 4.2 combine)
 *
 * The prefill call is built for many query rows per sequence; the decode call
 * for one query row per sequence (it accepts any layout, and gives the same
 * result as the prefill call up to rounding).  Which kernel computes a prefill
 * row follows the sizes of its call (num_seqs, total_q_rows, max_q_rows,
 * max_kv_len, heads, block_size, topk), so a row's result is bit-reproducible
 * between calls of equal sizes and may differ by rounding between others.  A
 * prefill call whose sizes send every row to the query tiles leaves the
 * workspace untouched and requires it all the same.
 *
 * Supported: head_dim == 128; block_size in {64, 128}; 1 <= topk <= 64;
 * 1 <= num_q_heads / num_kv_heads <= 16; num_kv_heads <= 64.
 * ------------------------------------------------------------------------ */
size_t msa_sparse_attn_prefill_workspace_size(const msa_seqs* seqs, int num_q_heads,
                                              int num_kv_heads, int head_dim, int block_size,
                                              int topk);
int msa_sparse_attn_prefill(const void* q, const void* k, const void* v,
                            const int32_t* block_ids, const msa_seqs* seqs, int num_q_heads,
                            int num_kv_heads, int head_dim, int block_size, int topk,
                            float softmax_scale, void* o, float* lse, void* workspace,
                            size_t workspace_bytes, hipStream_t stream);

size_t msa_sparse_attn_decode_workspace_size(const msa_seqs* seqs, int num_q_heads,
                                             int num_kv_heads, int head_dim, int block_size,
                                             int topk);
int msa_sparse_attn_decode(const void* q, const void* k, const void* v,
                           const int32_t* block_ids, const msa_seqs* seqs, int num_q_heads,
                           int num_kv_heads, int head_dim, int block_size, int topk,
                           float softmax_scale, void* o, float* lse, void* workspace,
                           size_t workspace_bytes, hipStream_t stream);

/* ------------------------------------------------------------------------
 * msa_sparse_attn_prefill_fp8 / msa_sparse_attn_decode_fp8 -- the Main Branch
 * on 8-bit queries and KV cache.
 *
 * Sec. 4.2 notes that the kernels also take fp8 inputs, which rescales the IO
 * volume of the Main Branch.  q, k and v hold OCP 8-bit floating point E4M3
 * ("e4m3fn": sign, 4 exponent bits with bias 7, 3 mantissa bits; no
 * infinities; S.1111.111 is NaN) codes, one byte per element, in the layouts
 * of the bf16 calls.  Element values are code * q_scale, code * k_scale and
 * code * v_scale (per-tensor fp32 scales, finite and > 0).  The result is the
 * attention of those values: logits use softmax_scale * q_scale * k_scale and
 * O is scaled by v_scale.  Block ids, the bf16 O and fp32 LSE outputs, the
 * workspace (the *_workspace_size queries of the bf16 calls apply), stream and
 * error behaviour are those of msa_sparse_attn_prefill / _decode; a scale that
 * is not finite and positive returns MSA_ERR_INVALID.  The kernels widen e4m3
 * to bf16 exactly on load and compute as the bf16 calls do.
 * ------------------------------------------------------------------------ */
int msa_sparse_attn_prefill_fp8(const void* q, const void* k, const void* v, float q_scale,
                                float k_scale, float v_scale, const int32_t* block_ids,
                                const msa_seqs* seqs, int num_q_heads, int num_kv_heads,
                                int head_dim, int block_size, int topk, float softmax_scale,
                                void* o, float* lse, void* workspace, size_t workspace_bytes,
                                hipStream_t stream);
int msa_sparse_attn_decode_fp8(const void* q, const void* k, const void* v, float q_scale,
                               float k_scale, float v_scale, const int32_t* block_ids,
                               const msa_seqs* seqs, int num_q_heads, int num_kv_heads,
                               int head_dim, int block_size, int topk, float softmax_scale,
                               void* o, float* lse, void* workspace, size_t workspace_bytes,
                               hipStream_t stream);

/* ------------------------------------------------------------------------
 * msa_dense_attn -- dense causal GQA attention, the baseline MSA is measured
 * against (no block selection).
 *
 * Every query row attends to all keys of its sequence at positions <= p: the
 * softmax attention that the sparse-attention equation of Sec. 3.1 becomes
 * when the selected set covers every causal block (Sec. 2.2, full attention
 * with GQA sharing of K and V across the G query heads of a group).
 *
 * Arguments, layouts, ownership, outputs and errors are those of
 * msa_sparse_attn_prefill without block ids: q [total_q_rows, H_q, 128],
 * k and v [total_kv_rows, H_kv, 128] (bf16), o [total_q_rows, H_q, 128] bf16,
 * lse [total_q_rows, H_q] fp32 natural log (-inf for rows with no visible
 * key).  Sequences with at most 4 query rows (decode) run a split row kernel
 * whose partials need the workspace; longer ones run a FlashAttention-style
 * tiled kernel, which leaves the workspace of its query (a few bytes per
 * sequence, required all the same) untouched.
 *
 * Supported: head_dim == 128; 1 <= num_q_heads / num_kv_heads <= 16;
 * num_kv_heads <= 64.
 * ------------------------------------------------------------------------ */
size_t msa_dense_attn_workspace_size(const msa_seqs* seqs, int num_q_heads, int num_kv_heads,
                                     int head_dim);
int msa_dense_attn(const void* q, const void* k, const void* v, const msa_seqs* seqs,
                   int num_q_heads, int num_kv_heads, int head_dim, float softmax_scale, void* o,
                   float* lse, void* workspace, size_t workspace_bytes, hipStream_t stream);

/* ------------------------------------------------------------------------
 * msa_dense_attn_paged / msa_dense_attn_paged_fp8 -- dense causal GQA attention
 * of each sequence's new rows over its paged keys: the layers and phases
 * without block selection, on the cache that the sparse calls read.
 *
 * Arguments, layouts, outputs and errors are those of msa_dense_attn (and, for
 * E4M3, the codes and scales of msa_sparse_attn_prefill_fp8), with a paged
 * seqs: block_table != NULL, page_size a power of two from 16 to 8192 (a
 * contiguous key side returns MSA_ERR_UNSUPPORTED).  Any number of new rows per
 * sequence, from one (decode) to a whole prompt, mixed in a batch.  A row
 * without a visible key gets O = 0 and LSE = -inf; rows of o and lse behind the
 * last sequence are left as they are.  What the cache holds behind a sequence's
 * last key (the rest of its last page, other pages) does not matter, NaN
 * included; a NaN or infinity among a sequence's own new keys may reach rows
 * before it.  How keys are split over the chip follows the sizes in seqs and
 * the lengths on the device: a result is bit-reproducible for equal inputs.
 *
 * Supported: head_dim == 128; 1 <= num_q_heads / num_kv_heads <= 16;
 * num_kv_heads <= 64; total_kv_rows < 2^31; q, k, v, o and the workspace 16-byte
 * aligned (else MSA_ERR_UNSUPPORTED).
 * ------------------------------------------------------------------------ */
size_t msa_dense_attn_paged_workspace_size(const msa_seqs* seqs, int num_q_heads, int num_kv_heads,
                                           int head_dim);
int msa_dense_attn_paged(const void* q, const void* k, const void* v, const msa_seqs* seqs,
                         int num_q_heads, int num_kv_heads, int head_dim, float softmax_scale,
                         void* o, float* lse, void* workspace, size_t workspace_bytes,
                         hipStream_t stream);
int msa_dense_attn_paged_fp8(const void* q, const void* k, const void* v, float q_scale,
                             float k_scale, float v_scale, const msa_seqs* seqs, int num_q_heads,
                             int num_kv_heads, int head_dim, float softmax_scale, void* o,
                             float* lse, void* workspace, size_t workspace_bytes,
                             hipStream_t stream);

/* ------------------------------------------------------------------------
 * Rotation by position (struct msa_rope)
 *
 * The first rot_dim elements of a head are turned in pairs: pair i, at position
 * p, by the angle p * inv_freq[i], cosine and sine both times `scale`; the rest
 * of the head passes unchanged.  Pair i is elements (i, i + rot_dim / 2), or,
 * interleaved, (2i, 2i + 1):
 *     y_a = x_a cos - x_b sin,  y_b = x_b cos + x_a sin.
 * Frequencies are the caller's, so that every scaling for long contexts is a
 * choice of them (and of `scale`).  Angles are formed in 64 bits.  rot_dim == 0
 * (or a NULL msa_rope) is no rotation.
 *
 * Supported: rot_dim a multiple of 8, at most the head's size; scale finite.
 * ------------------------------------------------------------------------ */
typedef struct msa_rope {
  int32_t rot_dim;          /* host */
  int32_t interleaved;      /* host: 0 = pairs (i, i + rot_dim / 2), else (2i, 2i + 1) */
  float scale;              /* host: factor of cosine and sine, 1 if none */
  const double* inv_freq;   /* device [rot_dim / 2]: radians per position */
} msa_rope;

/* ------------------------------------------------------------------------
 * msa_qk_norm_rope / msa_qk_norm_rope_fp8 -- RMS norm of each head of the new
 * rows' queries and keys, and their rotation, in one pass:
 *     n = x / sqrt(mean(x^2) + eps) * weight  over each head's head_dim elements,
 *     y = rotation of n by the row's position (Sequence layout above).
 * A NULL weight leaves that tensor without the norm (the rotation alone).
 * Queries and keys of the Main Branch, or index queries and index keys.
 *
 *   q      bf16 rows [total_q_rows], q_stride elements apart, each num_q_heads
 *          heads of head_dim, e.g. columns of a joint projection's output
 *   k      bf16 rows [total_q_rows], k_stride apart, num_kv_heads heads
 *   q_weight, k_weight   fp32 [head_dim], or NULL
 *   q_out  bf16 (fp8: E4M3 codes of the fp32 quotient y / q_scale, to nearest even,
 *          at most 448 in size) [total_q_rows, num_q_heads, head_dim] contiguous   OUTPUT
 *   k_out  the same with num_kv_heads, k_scale                      OUTPUT
 *
 * Either tensor is left out with 0 heads.  fp32 in between, one rounding.  The
 * bf16 outputs may be the inputs themselves where those are contiguous; other
 * overlaps are not allowed.  Rows behind the last sequence are left as they are.
 * With eps 0 a head of zeros gives NaN, and one whose mean square is below fp32's
 * normal range (elements of about 2^-63) is unspecified; sums of squares beyond
 * fp32 (elements of about 2^60) give 0.  bf16 elements that neither a norm nor the rotation
 * applies to keep their bits.  A scale is from 2^-126 to 2^126 (else
 * MSA_ERR_INVALID).  No workspace.
 *
 * Supported: head_dim 64 or 128; up to 1024 heads each; strides a multiple of 4
 * elements, tensors 8-byte aligned (else MSA_ERR_UNSUPPORTED).
 * ------------------------------------------------------------------------ */
int msa_qk_norm_rope(const void* q, int64_t q_stride, const void* k, int64_t k_stride,
                     const msa_seqs* seqs, int num_q_heads, int num_kv_heads, int head_dim,
                     const float* q_weight, const float* k_weight, float eps,
                     const msa_rope* rope, void* q_out, void* k_out, hipStream_t stream);
int msa_qk_norm_rope_fp8(const void* q, int64_t q_stride, const void* k, int64_t k_stride,
                         float q_scale, float k_scale, const msa_seqs* seqs, int num_q_heads,
                         int num_kv_heads, int head_dim, const float* q_weight,
                         const float* k_weight, float eps, const msa_rope* rope, void* q_out,
                         void* k_out, hipStream_t stream);

/* ------------------------------------------------------------------------
 * msa_qk_norm_rope_backward -- gradients of msa_qk_norm_rope.
 *
 * For upstream gradients g of q_out and k_out, h = g turned back (the transposed
 * rotation, times the same scale) and u = x / sqrt(mean(x^2) + eps):
 *     d weight = sum over rows and heads of h * u,
 *     d x      = (h * weight - u * mean(h * weight * u)) / sqrt(mean(x^2) + eps);
 * without the norm d x = h.
 *
 *   q, k, weights, eps, rope   as passed to the forward call (q or k of a tensor
 *              without weight is not read and may be NULL)
 *   d_q_out, d_k_out   bf16, contiguous, as the outputs
 *   d_q, d_k   bf16 rows d_q_stride / d_k_stride elements apart   OUTPUT (each may
 *              be the contiguous gradient it is formed from)
 *   d_q_weight, d_k_weight   fp32 [head_dim]   OUTPUT, or NULL to skip; written,
 *              not added to (zeros for a tensor with 0 heads, or without rows)
 *
 * fp32 in between.  Every output is bit-reproducible: the weight gradients add
 * rows in an order that the sizes fix.  Rows behind the last sequence are left
 * as they are and take no part.  The workspace, 8-byte aligned, is needed where a
 * weight is given.
 * Supported sizes as for msa_qk_norm_rope.
 * ------------------------------------------------------------------------ */
size_t msa_qk_norm_rope_backward_workspace_size(const msa_seqs* seqs, int num_q_heads,
                                                int num_kv_heads, int head_dim);
int msa_qk_norm_rope_backward(const void* q, int64_t q_stride, const void* k, int64_t k_stride,
                              const void* d_q_out, const void* d_k_out, const msa_seqs* seqs,
                              int num_q_heads, int num_kv_heads, int head_dim,
                              const float* q_weight, const float* k_weight, float eps,
                              const msa_rope* rope, void* d_q, int64_t d_q_stride, void* d_k,
                              int64_t d_k_stride, float* d_q_weight, float* d_k_weight,
                              void* workspace, size_t workspace_bytes, hipStream_t stream);

/* ------------------------------------------------------------------------
 * msa_kv_append / msa_kv_append_fp8 -- the new rows' keys, values and index keys
 * into the cache, keys and index keys with norm and rotation on the way.
 *
 * Row t of sequence s goes to the cache row of its position (Sequence layout
 * above; kv_lens count the new rows already): kv_starts[s] + p, or its row in
 * the page that the block table lists.  A row whose page id lies outside the
 * pool (a table filled with -1, say) or whose position lies outside the cache
 * is not stored; nothing else in the cache is written.  Cache rows must not be
 * shared between new rows (two sequences listing the same page for new
 * positions): what such a row holds is unspecified.
 *
 *   k, v       bf16 rows [total_q_rows], k_stride / v_stride elements apart, each
 *              num_kv_heads heads of head_dim
 *   index_k    bf16 rows, index_k_stride apart, of d_idx elements; NULL together
 *              with index_k_cache: no index keys (d_idx, its stride, weight and
 *              rope are then ignored)
 *   k_weight, index_k_weight, eps, rope, index_rope   as in msa_qk_norm_rope
 *   k_cache, v_cache   bf16 (fp8: E4M3 codes of the fp32 quotients y / k_scale and
 *              v / v_scale, to nearest even, at most 448 in size)
 *              [total_kv_rows, num_kv_heads, head_dim]   UPDATED
 *   index_k_cache      bf16 [total_kv_rows, d_idx]        UPDATED
 *
 * Values are stored bit for bit (bf16) or as codes; scales as for
 * msa_qk_norm_rope_fp8.  No workspace.
 * Supported: head_dim == 128; num_kv_heads <= 64; d_idx 64 or 128; contiguous, or
 * pages of a power of two from 16 to 8192 rows; strides and alignment as for
 * msa_qk_norm_rope.
 * ------------------------------------------------------------------------ */
int msa_kv_append(const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                  const void* index_k, int64_t index_k_stride, const msa_seqs* seqs,
                  int num_kv_heads, int head_dim, int d_idx, const float* k_weight,
                  const float* index_k_weight, float eps, const msa_rope* rope,
                  const msa_rope* index_rope, void* k_cache, void* v_cache, void* index_k_cache,
                  hipStream_t stream);
int msa_kv_append_fp8(const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                      float k_scale, float v_scale, const void* index_k, int64_t index_k_stride,
                      const msa_seqs* seqs, int num_kv_heads, int head_dim, int d_idx,
                      const float* k_weight, const float* index_k_weight, float eps,
                      const msa_rope* rope, const msa_rope* index_rope, void* k_cache,
                      void* v_cache, void* index_k_cache, hipStream_t stream);

/* ------------------------------------------------------------------------
 * Latent attention
 *
 * Token j has one latent vector c_j of latent_dim elements, from which every
 * head's key and value are products, and one rotated key part r_j of 64 elements
 * that the heads share.  With a head's query of two parts, n_i (128) and the
 * rotated e_i (64), its key matrix A and its value matrix B (128 x latent_dim):
 *     S_ij = softmax_scale (n_i . A c_j + e_i . r_j),   P = softmax over j <= i,
 *     O_i = sum_j P_ij B c_j.
 * Expanded form (msa_latent_attn): the products A c_j, B c_j are made for every
 * token and head before the call.  Absorbed form (msa_latent_attn_paged): the
 * query is A^T n_i (latent_dim elements), the cache holds c_j and r_j alone, and
 * the call returns sum_j P_ij c_j, to be multiplied by B.  Both give the same O
 * and LSE; the products are the caller's.  softmax_scale is that of the expanded
 * head (1 / sqrt(128 + 64), say) in both.
 * ------------------------------------------------------------------------ */

/* ------------------------------------------------------------------------
 * msa_latent_append / msa_latent_append_fp8 -- the new rows' latents and shared
 * key parts into the cache:
 *     row = [ c / sqrt(mean(c^2) + eps) * weight,  rotation of k_rope by position ]
 * Row t of sequence s goes to the cache row of its position, as in msa_kv_append
 * (contiguous or paged; rows without a place in the cache are not stored).
 *
 *   latent     bf16 rows [total_q_rows], latent_stride elements apart, of latent_dim
 *              elements, e.g. columns of a joint projection's output
 *   k_rope     bf16 rows, k_rope_stride apart, of 64 elements
 *   weight     fp32 [latent_dim], or NULL: no norm
 *   rope       the rotation of k_rope (rot_dim at most 64), or NULL
 *   cache      bf16 (fp8: E4M3 codes of the fp32 quotients by cache_scale, to nearest
 *              even, at most 448 in size) [total_kv_rows, latent_dim + 64]   UPDATED
 *
 * fp32 in between, one rounding; bf16 elements that neither the norm nor the
 * rotation applies to keep their bits.  eps, weights and scales as for
 * msa_qk_norm_rope(_fp8).  No workspace.
 * Supported: latent_dim 256 or 512; pages of a power of two from 16 to 8192 rows;
 * strides a multiple of 4 elements, tensors 8-byte aligned (else
 * MSA_ERR_UNSUPPORTED).
 * ------------------------------------------------------------------------ */
int msa_latent_append(const void* latent, int64_t latent_stride, const void* k_rope, int64_t k_rope_stride,
                      const msa_seqs* seqs, int latent_dim, const float* weight, float eps, const msa_rope* rope,
                      void* cache, hipStream_t stream);
int msa_latent_append_fp8(const void* latent, int64_t latent_stride, const void* k_rope, int64_t k_rope_stride,
                          float cache_scale, const msa_seqs* seqs, int latent_dim, const float* weight, float eps,
                          const msa_rope* rope, void* cache, hipStream_t stream);

/* ------------------------------------------------------------------------
 * msa_latent_attn_paged / msa_latent_attn_paged_fp8 -- latent attention, absorbed
 * form, of each sequence's new rows over its paged cache; one token per sequence,
 * draft rows and chunks, mixed in a batch.
 *
 *   q          bf16 [total_q_rows, num_heads, latent_dim], rows q_stride and heads
 *              q_head_stride elements apart (a product made head by head is
 *              [num_heads, total_q_rows, latent_dim]: strides latent_dim and
 *              total_q_rows * latent_dim)
 *   q_rope     bf16 [total_q_rows, num_heads, 64], with strides of its own
 *   cache      bf16 (fp8: E4M3 codes of value / cache_scale) [total_kv_rows, latent_dim + 64]
 *   o          bf16 [total_q_rows, num_heads, latent_dim]   OUTPUT: sum_j P_ij c_j
 *   lse        fp32 [total_q_rows, num_heads]               OUTPUT, natural log
 *
 * A row without a visible key gets O = 0 and LSE = -inf; rows of o and lse behind
 * the last sequence are left as they are.  What the cache holds behind a
 * sequence's last key does not matter, NaN included; a NaN or infinity among a
 * sequence's own new keys may reach rows before it.  The weights P are rounded to
 * bf16 for the second product, their sums are of the unrounded ones.  Results are
 * bit-reproducible for equal inputs.  cache_scale is finite and positive (else
 * MSA_ERR_INVALID).  A contiguous key side returns MSA_ERR_UNSUPPORTED.
 *
 * Supported: latent_dim 256 or 512; num_heads <= 1024; pages of a power of two from
 * 16 to 8192 rows; total_kv_rows < 2^31; strides a multiple of 8 elements; q, q_rope,
 * cache, o and the workspace 16-byte aligned (else MSA_ERR_UNSUPPORTED).
 * ------------------------------------------------------------------------ */
size_t msa_latent_attn_paged_workspace_size(const msa_seqs* seqs, int num_heads, int latent_dim);
int msa_latent_attn_paged(const void* q, int64_t q_stride, int64_t q_head_stride, const void* q_rope,
                          int64_t q_rope_stride, int64_t q_rope_head_stride, const void* cache,
                          const msa_seqs* seqs, int num_heads, int latent_dim, float softmax_scale, void* o,
                          float* lse, void* workspace, size_t workspace_bytes, hipStream_t stream);
int msa_latent_attn_paged_fp8(const void* q, int64_t q_stride, int64_t q_head_stride, const void* q_rope,
                              int64_t q_rope_stride, int64_t q_rope_head_stride, const void* cache,
                              float cache_scale, const msa_seqs* seqs, int num_heads, int latent_dim,
                              float softmax_scale, void* o, float* lse, void* workspace,
                              size_t workspace_bytes, hipStream_t stream);

/* ------------------------------------------------------------------------
 * msa_latent_attn -- latent attention, expanded form: causal attention of prompts,
 * training batches, and chunks whose context was expanded for them.
 *
 *   q          bf16 [total_q_rows, num_heads, 128], rows q_stride and heads
 *              q_head_stride elements apart
 *   q_rope     bf16 [total_q_rows, num_heads, 64], with strides of its own
 *   kv         bf16 [total_kv_rows, num_heads, 256] contiguous: a head's own key part
 *              (128), then its values (128), as one up-projection of the latents gives them
 *   k_rope     bf16 rows [total_kv_rows], k_rope_stride elements apart, of 64 elements: the
 *              shared key part, e.g. columns of a contiguous latent cache
 *   o          bf16 [total_q_rows, num_heads, 128]   OUTPUT
 *   lse        fp32 [total_q_rows, num_heads]        OUTPUT, natural log
 *
 * Rows without a visible key get O = 0 and LSE = -inf; rows behind the last sequence
 * are left as they are.  A NaN or infinity among a sequence's own new keys may reach
 * rows before it.  The weights are rounded to bf16 for the second product, their sums
 * are of the unrounded ones.  Results are bit-reproducible for equal inputs.
 *
 * Supported: num_heads <= 256; contiguous key side; total_q_rows * num_heads < 2^31;
 * strides a multiple of 8 elements, k_rope_stride at most 2^20; tensors 16-byte
 * aligned; (total_q_rows / 32 + 8 num_seqs) num_heads < 2^26, a grid's limit (else
 * MSA_ERR_UNSUPPORTED).  The query may give 0: then the workspace is
 * not read and may be NULL.
 * ------------------------------------------------------------------------ */
size_t msa_latent_attn_workspace_size(const msa_seqs* seqs, int num_heads);
int msa_latent_attn(const void* q, int64_t q_stride, int64_t q_head_stride, const void* q_rope,
                    int64_t q_rope_stride, int64_t q_rope_head_stride, const void* kv, const void* k_rope,
                    int64_t k_rope_stride, const msa_seqs* seqs, int num_heads, float softmax_scale, void* o,
                    float* lse, void* workspace, size_t workspace_bytes, hipStream_t stream);

/* ------------------------------------------------------------------------
 * msa_latent_attn_backward -- gradients of msa_latent_attn.
 *
 * For the upstream gradient dO of O, with P_ij = exp(S_ij - LSE_i), D_i = dO_i . O_i
 * and dS_ij = P_ij (dO_i . v_j - D_i), for each head
 *   dq_i = scale sum_j dS_ij k_j,   dq_rope_i = scale sum_j dS_ij k_rope_j,
 *   dk_j = scale sum_i dS_ij q_i,   dv_j = sum_i P_ij dO_i,
 * and, summed over the heads that share it,
 *   dk_rope_j = scale sum_h sum_i dS_ij q_rope_i.
 *
 *   q .. k_rope, strides, seqs, num_heads, softmax_scale   as passed to the forward call
 *   o, lse     the forward's outputs;  d_o  bf16 as o, the upstream gradient
 *   d_q, d_q_rope   bf16 as q and q_rope, with strides of their own (rows and heads that
 *              do not overlap; e.g. columns of a joint gradient)   OUTPUT
 *   d_kv       bf16 [total_kv_rows, num_heads, 256]   OUTPUT: dk, then dv
 *   d_k_rope   bf16 rows d_k_rope_stride elements apart, of 64 elements   OUTPUT
 *
 * Every key row is written (zeros where no query attends); a query row without a
 * visible key gets zeros, also where there is no key row at all; query rows behind the
 * last sequence are left as they are and take no part.  P and dS are rounded to bf16 for
 * the products, everything else is fp32 with one rounding of each result; the heads'
 * shares of d_k_rope are added in fp32 in the heads' order.  Every output is
 * bit-reproducible.  Key ranges of different sequences must not overlap (the call
 * cannot tell; d_kv and d_k_rope are then unspecified, of other rows too).  No output
 * may alias an input.
 *
 * Supported: as msa_latent_attn, with total_kv_rows * num_heads < 2^31, (the larger of
 * total_q_rows / 256 and total_kv_rows / 128, + num_seqs) num_heads < 2^24, q_stride,
 * q_rope_stride and k_rope_stride at most 2^24, d_q and d_q_rope 8-byte aligned with
 * strides a multiple of 4 elements.
 * ------------------------------------------------------------------------ */
size_t msa_latent_attn_backward_workspace_size(const msa_seqs* seqs, int num_heads);
int msa_latent_attn_backward(const void* q, int64_t q_stride, int64_t q_head_stride, const void* q_rope,
                             int64_t q_rope_stride, int64_t q_rope_head_stride, const void* kv,
                             const void* k_rope, int64_t k_rope_stride, const void* o, const float* lse,
                             const void* d_o, const msa_seqs* seqs, int num_heads, float softmax_scale,
                             void* d_q, int64_t d_q_stride, int64_t d_q_head_stride, void* d_q_rope,
                             int64_t d_q_rope_stride, int64_t d_q_rope_head_stride, void* d_kv, void* d_k_rope,
                             int64_t d_k_rope_stride, void* workspace, size_t workspace_bytes,
                             hipStream_t stream);

/* ------------------------------------------------------------------------
 * msa_sparse_attn_backward -- training backward of the Main Branch.
 *
 * Alg. 1 trains through the sparse attention of Sec. 3.1.  For an upstream
 * gradient dO of the output O, with P_ij = exp(softmax_scale q_i.k_j - LSE_i)
 * over the tokens row i attended and D_i = dO_i . O_i:
 *   dV_j = sum_i P_ij dO_i,  dS_ij = P_ij (dO_i . v_j - D_i),
 *   dQ_i = softmax_scale sum_j dS_ij k_j,  dK_j = softmax_scale sum_i dS_ij q_i,
 * each sum running over the (row, head, token) triples of the forward.
 *
 *   q, k, v, block_ids, seqs, heads, block_size, topk, softmax_scale: exactly
 *              as passed to the forward call (msa_sparse_attn_prefill/_decode)
 *   o          bf16 [total_q_rows, num_q_heads, head_dim]   the forward's O
 *   lse        fp32 [total_q_rows, num_q_heads]             the forward's LSE
 *   d_o        bf16 [total_q_rows, num_q_heads, head_dim]   upstream gradient
 *   d_q        bf16 [total_q_rows, num_q_heads, head_dim]   OUTPUT
 *   d_k, d_v   bf16 [total_kv_rows, num_kv_heads, head_dim] OUTPUT; every row is
 *              written, key rows no query attended get 0
 *
 * Work runs key-block-outer with fp32 accumulation.  Every output is
 * bit-reproducible: d_q adds its partials in slot order, and d_k and d_v add a
 * key block's contributions in ascending (query row, slot) order (the
 * reverse index is sorted into that order).  Workspace, stream and
 * error behaviour as for msa_sparse_attn_prefill.  Supported: head_dim == 128;
 * block_size 64 or 128 with 1 <= topk <= 64; 1 <= num_q_heads / num_kv_heads
 * <= 16; num_kv_heads <= 64.
 * ------------------------------------------------------------------------ */
size_t msa_sparse_attn_backward_workspace_size(const msa_seqs* seqs, int num_q_heads,
                                               int num_kv_heads, int head_dim, int block_size,
                                               int topk);
int msa_sparse_attn_backward(const void* q, const void* k, const void* v, const void* o,
                             const float* lse, const void* d_o, const int32_t* block_ids,
                             const msa_seqs* seqs, int num_q_heads, int num_kv_heads,
                             int head_dim, int block_size, int topk, float softmax_scale,
                             void* d_q, void* d_k, void* d_v, void* workspace,
                             size_t workspace_bytes, hipStream_t stream);

/* ------------------------------------------------------------------------
 * msa_sparse_kl_backward -- the sparse KL loss that trains the Index Branch.
 *
 * Sec. 3.2 ("KL Loss"), per query row i and group r, over the causally
 * visible tokens T of the selected blocks: the student
 * P_idx_j = softmax_j(q_idx[i,r] . k_idx[j] / sqrt(d_idx)) and the detached
 * teacher P_j = (1/G) sum over the group's query heads h of
 * exp(softmax_scale q[i,h] . k[j,r] - lse[i,h]) (Alg. 1: the Main Branch
 * attention over the same tokens; lse is the forward's LSE, Sec. 4.3 "LSE
 * fusion").  Outputs, with Delta_j = P_idx_j - P_j:
 *   kl[i, r]        = sum_j P_j (ln P_j - ln P_idx_j)          (optional)
 *   d_index_q[i, r] = grad_scale / sqrt(d_idx) sum_j Delta_j k_idx[j]
 *   d_index_k[j]    = grad_scale / sqrt(d_idx) sum_{i,r} Delta_ij q_idx[i, r]
 * i.e. grad_scale times the gradients of sum_{i,r} kl[i, r]; the paper's
 * per-layer loss is the mean over rows and groups, so a training loop passes
 * grad_scale = lambda / (total_q_rows * num_kv_heads).  Nothing flows into q
 * or k (the gradient detach of Sec. 3.2).
 *
 *   index_q    bf16 [total_q_rows, num_kv_heads, d_idx]
 *   index_k    bf16 [total_kv_rows, d_idx]
 *   q, k       bf16 as for msa_sparse_attn_prefill; lse fp32 [total_q_rows, num_q_heads]
 *   block_ids  int32 [total_q_rows, num_kv_heads, topk]   the selection the forward used
 *   d_index_q  bf16 [total_q_rows, num_kv_heads, d_idx]   OUTPUT
 *   d_index_k  bf16 [total_kv_rows, d_idx]                OUTPUT; every row written
 *   kl         fp32 [total_q_rows, num_kv_heads]          OUTPUT, or NULL to skip
 *
 * Workspace, stream and error behaviour as for msa_sparse_attn_prefill.
 * d_index_q, d_index_k and kl are bit-reproducible (d_index_k adds a key
 * block's queries in ascending (row, slot) order).  Supported: d_idx in {64, 128};
 * head_dim == 128; block_size 64 or 128 with 1 <= topk <= 64;
 * num_q_heads / num_kv_heads in {1, 2, 4, 8, 16}; num_kv_heads <= 64.
 * ------------------------------------------------------------------------ */
size_t msa_sparse_kl_backward_workspace_size(const msa_seqs* seqs, int num_q_heads,
                                             int num_kv_heads, int d_idx, int head_dim,
                                             int block_size, int topk);
int msa_sparse_kl_backward(const void* index_q, const void* index_k, const void* q, const void* k,
                           const float* lse, const int32_t* block_ids, const msa_seqs* seqs,
                           int num_q_heads, int num_kv_heads, int d_idx, int head_dim,
                           int block_size, int topk, float softmax_scale, float grad_scale,
                           void* d_index_q, void* d_index_k, float* kl, void* workspace,
                           size_t workspace_bytes, hipStream_t stream);

/* ------------------------------------------------------------------------
 * Kernel timing (a measurement aid; no part of the attention path)
 *
 * While enabled, every kernel a call launches is bracketed by a pair of HIP
 * events recorded on the call's stream, filed under the kernel's name (e.g.
 * "kvo_attn_kernel", "index_block_max_lds_kernel"; all variants of a template
 * under one name, the query-tile attention kernel under "dense_prefill_kernel"
 * or "tile_attn_kernel" by the call that runs it).  The events are created
 * on first use and kept for reuse (global state of the timer alone).
 *
 *   msa_profile_enable(on)   on != 0 starts recording for later calls, 0 stops.
 *   msa_profile_reset()      forgets the launches recorded so far.
 *   msa_profile_kernel_name(i)  name of the i-th kernel seen since load, or
 *                            NULL past the last one; the string stays valid
 *                            until the library is unloaded.
 *   msa_profile_read(name, &launches, &total_ms)  launches of `name` since the
 *                            last reset and their summed event-to-event time;
 *                            waits for those events; unknown names read 0.
 *
 * Timing adds two event records per launch, so enable it only for runs that
 * read it.  Calls on several host threads must not interleave with reset or
 * read.  Errors: MSA_ERR_INVALID for null output pointers, MSA_ERR_HIP when
 * an event cannot be read.
 * ------------------------------------------------------------------------ */
int msa_profile_enable(int on);
int msa_profile_reset(void);
const char* msa_profile_kernel_name(int i);
int msa_profile_read(const char* kernel, int64_t* launches, double* total_ms);

#ifdef __cplusplus
}
#endif

#endif /* MSA_H_ */
