/*
 * sdllm_paged.h -- the paged key / value cache of the sdllm library: sequences of different lengths that share one pool of
 * pages, and the calls that a serving loop makes on it.  Conventions, dtypes, status codes and error text are those of sdllm.h.
 *
 *   sdllm_paged_extend      pages for the step's new rows: stack of free pages, block tables and slots, on the device
 *   sdllm_qk_norm_rope      per-head norms of queries and keys with the position rotation in the same pass; the keys (and
 *                           values) optionally straight into their pages
 *   sdllm_paged_kv_append   copy a finished block's K/V rows of every layer into their slots
 *   sdllm_paged_attention   attention of K query rows per sequence over the cached rows and, optionally, the block's own
 *
 * The cache of a layer is two tensors k_pages, v_pages [n_pages, Hkv, page_size, D].  Row t of sequence b lies in page
 * block_table[b][t / page_size] at row t % page_size; page * page_size + row is the row's slot.  page_size is a power of two,
 * 16 .. 1024; n_pages * page_size < 2^31.  One block table serves every layer.
 *
 * Lengths, tables and slots are device data and are not checked on the host.  They are bounded on the device instead: no
 * value of theirs makes a call read or write outside the tensors it was given.  What each call makes of a value out of range
 * is stated with it.
 */
#ifndef SDLLM_PAGED_H
#define SDLLM_PAGED_H

#include "sdllm.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---------------------------------------------------------------------------------------
 * Block tables and slots from request lengths.  free_pages[0 .. n_free) is a stack of page ids (top at n_free - 1).
 *  1. In batch order every sequence with release[b] != 0 pushes the pages of its kv_lens[b] rows, in table order, and its
 *     length becomes 0 (a finished request makes room for the next one in its batch slot).  Entries outside [0, n_pages) are no
 *     pages and are not pushed: a page that was given back before (behind a window) and its entry set to -1 does not come back again.
 *  2. Sequence b asks for n = clamp(new_lens[b], 0, K) rows (new_lens NULL: K; do_append[b] == 0: none), that is for
 *     ceil((len + n) / page_size) - ceil(len / page_size) pages.  In batch order the pages are popped off the stack, top first,
 *     into the table entries behind the ones in use.  A sequence gets all of its rows or none: none if len + n exceeds
 *     max_pages * page_size (then it does not count below), or if it needs pages and its need together with that of all
 *     sequences before it exceeds the stack.
 *  3. granted[b] = n or 0; kv_lens_out[b] = len + granted[b]; n_free_out = what is left on the stack;
 *     slots[b][t] = slot of row len + t for t < granted[b], -1 for the other t < K.
 * Entries of block_table that no new page goes to are left as they were, and so is the stack apart from pushed entries.
 *
 *   B 1..65536, K >= 1, max_pages (entries of a table row) >= 1, n_pages (pool size, capacity of free_pages) >= 1;
 *   max_pages * page_size <= 2^30, B * K < 2^31, B * max_pages < 2^30
 * Out of range: kv_lens is clamped to [0, max_pages * page_size], n_free to [0, n_pages]; pushes past n_pages are dropped; a
 * row whose page id is outside [0, n_pages) gets slot -1.
 * --------------------------------------------------------------------------------------- */
typedef struct sdllm_paged_extend_params {
  int32_t B, K;
  int32_t page_size, max_pages, n_pages;
} sdllm_paged_extend_params;

size_t sdllm_paged_extend_workspace_bytes(const sdllm_paged_extend_params* p);

/*
 *   block_table [B,max_pages] int32 in/out     kv_lens [B] int32      kv_lens_out [B] int32 out (may be kv_lens)
 *   new_lens [B] int32 or NULL    do_append [B] uint8 or NULL         release [B] uint8 or NULL
 *   free_pages [n_pages] int32 in/out          n_free [1] int32       n_free_out [1] int32 out (may be n_free)
 *   slots [B,K] int32 out         granted [B] int32 out
 * Apart from kv_lens_out == kv_lens and n_free_out == n_free no two arrays may overlap.
 * Errors: INVALID_ARG, UNSUPPORTED, WORKSPACE, HIP.
 */
int sdllm_paged_extend(const sdllm_paged_extend_params* p,
                       int32_t* block_table, const int32_t* kv_lens, const int32_t* new_lens,
                       const uint8_t* do_append, const uint8_t* release,
                       int32_t* free_pages, const int32_t* n_free,
                       int32_t* kv_lens_out, int32_t* n_free_out,
                       int32_t* slots, int32_t* granted,
                       void* workspace, size_t workspace_bytes, void* stream);

/* ---------------------------------------------------------------------------------------
 * Norms of queries and keys for each head and the position rotation, in one pass over the rows.  For a row x of D elements
 *     y = x / sqrt(mean(x^2) + eps) * w     (w: q_weight for queries, k_weight for keys; NULL: y = x)
 * and the first rotary_dim elements of y are turned in pairs by the angle position * f_i, i = 0 .. rotary_dim / 2 - 1, and
 * multiplied by `amplitude`; the others stay as they are.  Pairs are (i, i + rotary_dim / 2), or (2i, 2i + 1) if interleaved.
 *     f_i = theta_base^(-2i / rotary_dim), and for longer contexts than a model was trained on (scale_factor s > 1):
 *     original_len == 0:  f_i / s for every pair
 *     original_len  > 0:  u f_i + (1 - u) f_i / s, where r = f_i * original_len / (2 pi) is the number of turns of pair i in the
 *                         original context and u = clamp((r - low_turns) / (high_turns - low_turns), 0, 1)
 * Position of row t of sequence b: positions[b] + t (which may pass 2^31), or positions[b * K + t] if positions_per_row.  The angle is formed in
 * double precision and reduced there, cos / sin, norm and products are fp32, the result is rounded once.
 *
 *   dtype, B, K >= 1 (B * K < 2^24), Hq, Hkv 1..65535, D (multiple of 16, <= 256), rotary_dim (multiple of 16, 0..D; 0: no rotation)
 *   *_stride: distances in elements between sequences, heads and rows of a tensor [B, H, K, D] with D contiguous, in this
 *   order; all zero: dense.  Each a multiple of 16 bytes.
 *   page_size, n_pages: only used with pages
 * --------------------------------------------------------------------------------------- */
typedef struct sdllm_qk_norm_rope_params {
  int32_t dtype;
  int32_t B, K, Hq, Hkv, D;
  int32_t rotary_dim, interleaved, positions_per_row;
  int32_t page_size, n_pages;
  float eps, theta_base;
  float scale_factor, low_turns, high_turns, amplitude;
  int32_t original_len;
  int64_t q_stride[3], k_stride[3], v_stride[3], q_out_stride[3], k_out_stride[3];
} sdllm_qk_norm_rope_params;

/*
 *   q [B,Hq,K,D], k [B,Hkv,K,D] read      positions [B] or [B,K] int32 on the device
 *   q_weight, k_weight [D] of the same dtype, or NULL
 *   q_out [B,Hq,K,D] written entirely (may be q, same strides)
 *   Keys: either k_out [B,Hkv,K,D] (may be k), written entirely, with v, k_pages, v_pages, slots NULL;
 *   or k_out NULL and v [B,Hkv,K,D] read, k_pages, v_pages [n_pages,Hkv,page_size,D], slots [B,K] int32: row t of sequence b
 *   of k (normed, rotated) and of v (bit for bit) goes to slot slots[b][t]; a slot outside [0, n_pages * page_size) is skipped.
 *   Slots must be distinct.  Nothing else in the pages is written.
 * Apart from exact in-place use outputs must not overlap inputs.  No workspace.  Errors: INVALID_ARG, UNSUPPORTED, HIP.
 */
int sdllm_qk_norm_rope(const sdllm_qk_norm_rope_params* p,
                       const void* q, const void* k, const void* v, const int32_t* positions,
                       const void* q_weight, const void* k_weight,
                       void* q_out, void* k_out, void* k_pages, void* v_pages, const int32_t* slots,
                       void* stream);

/* ---------------------------------------------------------------------------------------
 * KV append into pages: the paged form of sdllm_kv_append.  For every layer, K and V, bit for bit:
 *     pages[l][slots[b][t] / page_size, h, slots[b][t] % page_size, :] <- block[l][b,h,t,:]
 * Rows whose slot lies outside [0, n_pages * page_size) are skipped (a sequence whose block is not finished has slots -1).
 * Slots must be distinct.  Nothing else in the pages is written.
 *
 *   n_layers, B, Hkv, K >= 1; D * sizeof(element) % 16 == 0;
 *   pages_layer_stride / block_layer_stride: distance between layers in ELEMENTS (0 = dense)
 * --------------------------------------------------------------------------------------- */
typedef struct sdllm_paged_append_params {
  int32_t dtype;
  int32_t n_layers, B, Hkv, D, K;
  int32_t page_size, n_pages;
  int64_t pages_layer_stride, block_layer_stride;
} sdllm_paged_append_params;

/*
 *   k_pages, v_pages [n_layers][n_pages,Hkv,page_size,D] in/out      k_blocks, v_blocks [n_layers][B,Hkv,K,D] read only
 *   slots [B,K] int32 on the device
 */
int sdllm_paged_kv_append(const sdllm_paged_append_params* p,
                          void* k_pages, void* v_pages, const void* k_blocks, const void* v_blocks,
                          const int32_t* slots, void* stream);

/* ---------------------------------------------------------------------------------------
 * Attention over the paged cache.  Sequence b has n = kv_lens[b] cached rows and q = q_lens[b] query rows; with a block its
 * own K/V rows 0..q-1 follow the cached ones, so that there are N = n + q keys, without one N = n.  The queries are the last q
 * of the N positions: row r is at position p = N - q + r.  Key j < N is visible to it if
 *     j <= p                     (causal != 0)       and
 *     p - j < window or j < sinks      (window > 0: a sliding window, with the first `sinks` keys kept visible)
 * and its page id is valid.  out row = softmax over the visible keys of scale * q k, times their values; a row that sees no
 * key is zero, and what is stored for hidden keys, or behind the last one in a page, does not matter, NaN included.
 * A value of a visible key that is infinite or NaN reaches its column of the rows that see it, and nothing else.
 * One token per sequence (K = 1), the rows of a block and the pieces of prompts are the same call.
 *
 *   B, Hq, Hkv, D   as for sdllm_block_attention; D in {64, 128} for both dtypes; B * Hkv < 2^22,
 *                   B * Hq * K < 2^28
 *   K               query rows per sequence of q, out and the block (>= 1)
 *   page_size, n_pages, max_pages (entries of a table row, > 0); a page of all heads below 2 GiB
 *   max_kv_len      upper bound of kv_lens, <= max_pages * page_size: the launch plan is made for it (the lengths themselves are
 *                   device data); max_kv_len + K <= 2^30
 *   scale           softmax scale, at most 1e38; <= 0 selects 1/sqrt(D)
 *   kv_splits       0 = choose automatically; n >= 1: a sequence of max_kv_len keys is cut into about n parts, unless
 *                   batch or sequences are so large that keys are not shared out
 *   *_stride        as for sdllm_qk_norm_rope; the rows of q and of the block may overlap
 * Out of range: kv_lens is clamped to [0, max_kv_len], q_lens to [0, K]; the keys of a page id outside [0, n_pages) are hidden
 * (a page that has left the window may be given back and its entry set to -1).
 * --------------------------------------------------------------------------------------- */
typedef struct sdllm_paged_attn_params {
  int32_t dtype;
  int32_t B, Hq, Hkv, D, K;
  int32_t page_size, n_pages, max_pages, max_kv_len;
  int32_t causal, window, sinks;
  float scale;
  int32_t kv_splits;
  int64_t q_stride[3], out_stride[3], k_block_stride[3], v_block_stride[3];
} sdllm_paged_attn_params;

/* Bytes of device workspace for these parameters (0 if none); (size_t)-1 if they are invalid.  with_block: whether the call is
 * given k_block / v_block (its keys count towards the plan). */
size_t sdllm_paged_attention_workspace_bytes(const sdllm_paged_attn_params* p, int32_t with_block);

/*
 *   q [B,Hq,K,D] read    k_pages, v_pages [n_pages,Hkv,page_size,D] read    block_table [B,max_pages] int32, kv_lens [B] int32
 *   k_block, v_block [B,Hkv,K,D] read, both or neither      q_lens [B] int32 or NULL (= K)
 *   out [B,Hq,K,D]: rows r < q_lens[b] are written, the others left as they were
 * Inputs are only read; out and workspace overlap none of them.  Errors: INVALID_ARG, UNSUPPORTED, WORKSPACE, HIP.
 */
int sdllm_paged_attention(const sdllm_paged_attn_params* p,
                          const void* q, const void* k_pages, const void* v_pages,
                          const int32_t* block_table, const int32_t* kv_lens,
                          const void* k_block, const void* v_block, const int32_t* q_lens,
                          void* out, void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* SDLLM_PAGED_H */
