/*
 * libamxfp4 — a paged key / value cache of FP4 codes for batches of conversations of different lengths, and the attention
 * that reads it.
 *
 * The paper's setting is inference with everything cast without calibration (Sec. 4, 5.1); its long-context discussion
 * (Sec. 5.2) is about caches. It defines no cache: pages, tables and the operators here are this library's. Keys and values
 * are cast PER TOKEN, in groups of 32 along the head dimension (Algorithm 1, Eq. 1), so that a token can be appended without
 * touching its neighbours; queries and probabilities stay BF16. (amxfp4_attention and amxfp4_attention_decode cast all four
 * operands, V along the keys, on caches of one length without pages.)
 *
 * Conventions as in amxfp4.h: data pointers are DEVICE pointers owned by the caller, `fmt` and `pool` are HOST structures
 * read during the call; nothing is allocated, retained or synchronised; arguments are validated on the host before any
 * launch, the return value is an amx_status_t, the message is available from amxfp4_last_error().
 * What lies on the device cannot be validated there. The calls never access memory outside the buffers that they are given,
 * whatever the lengths, tables, slots and queues say: a page id or slot outside the pool is not dereferenced, lengths and
 * row numbers are taken as if cut to what the buffers hold. Outputs and workspaces share no memory with anything else of a call.
 *
 * Layout of the pool, for each layer of a model its own (tables, slots and lengths are shared by the layers):
 *   codes    [pages][kv_heads][page_size][head_dim / 2] bytes, as amxfp4_quantize writes a row of head_dim elements;
 *   scales   [pages][kv_heads][head_dim / 32][page_size]([2]) bytes: the scales of one group of all tokens of the page side
 *            by side (a lane of the attention reads those of 16 keys at once), (S_p, S_n) pairs when asymmetric.
 *   slot     of a token: page * page_size + its place in the page. Token i of sequence b lies in page
 *            table[b][i / page_size] at place i % page_size.
 */
#ifndef AMXFP4_PAGED_H
#define AMXFP4_PAGED_H

#include <stddef.h>
#include <stdint.h>

#include "amxfp4.h" /* amx_format_t, status codes */

#ifdef __cplusplus
extern "C" {
#endif

typedef struct {
  int64_t pages;     /* >= 1; pages * page_size <= 2^30 */
  int32_t page_size; /* tokens to a page: a power of two, 16 to 1024 (AMX_ERR_UNSUPPORTED otherwise) */
  int32_t kv_heads;  /* 1 to 1024 */
  int32_t head_dim;  /* 64 or 128 (AMX_ERR_UNSUPPORTED otherwise) */
  int32_t reserved;  /* 0 */
  uint8_t* k_codes;  /* all four: 16-byte aligned */
  uint8_t* k_scales;
  uint8_t* v_codes;
  uint8_t* v_scales;
} amx_paged_pool_t;

/* Bytes of the codes (of K, and of V again) and of the scales of such a pool; the pointers are not looked at. 0 on invalid
 * arguments. */
size_t amxfp4_paged_codes_bytes(const amx_format_t* fmt, const amx_paged_pool_t* pool);
size_t amxfp4_paged_scales_bytes(const amx_format_t* fmt, const amx_paged_pool_t* pool);

/*
 * One step's bookkeeping, on the device: which rows of the packed batch belong to which sequence, where their keys and
 * values go, and which pages are taken or given back for it. In the order of the sequences b = 0 .. seqs - 1:
 *   new_rows[b] > 0    the sequence has lens[b] tokens and gets that many more, its rows starts[b] .. starts[b + 1] - 1 of the
 *                      batch (starts[b] = the sum of the new_rows before it, cut to `rows`). It takes the pages that they need
 *                      beyond those it has from the head of the queue, puts their ids into its row of the table, and
 *                      lens_out[b] = lens[b] + new_rows[b]; row starts[b] + i gets position lens[b] + i and its slot.
 *                      REFUSED are: one that would not fit its row of the table or the `rows` of the batch, and, in the
 *                      order of the sequences, from the first one on whose pages the queue no longer holds, all that need
 *                      pages. A refused sequence keeps its length; its rows get position -1 and slot -1.
 *   new_rows[b] == 0   nothing changes (an idle sequence).
 *   new_rows[b] < 0    it has ended: its pages go to the queue's end, lens_out[b] = 0.
 * Rows behind the last sequence's get position -1 and slot -1.
 *   queue     [pages] int32, a ring: `count` free page ids from entry `head` on (modulo pages). Read and written in place:
 *             pages given back are entered behind the last one; taken ones are not erased.
 *   state     int32[4] = {head, count, -, -}; state_out int32[4] = {head, count, sequences refused, rows of all sequences (cut to
 *             `rows`)}.
 *   table     [seqs][max_pages] int32, read and written in place: entries of new pages only.
 *   lens, new_rows, lens_out [seqs], starts [seqs + 1], slots, positions [rows]: int32.
 * The outputs are buffers of their own: lens_out must not be lens, state_out not state (AMX_ERR_INVALID_ARG): the call has no
 * order between reading and writing them. The same inputs give the same outputs and entries, so that a call may be repeated.
 * A program keeps two sets of lens and state and uses them in turn.
 * A sequence grows or ends, it does not shrink: lens are 0 or what an earlier call wrote. Behind a length that the caller lowers, pages
 * are lost: the sequence takes new ones for tokens whose pages it had, and gives back only those that the lower length counts.
 * Rows that turn out not to be wanted (of a draft) are taken back by planning the step again: as nothing that the call reads has
 * changed, the same lens, state, queue and table with the numbers of accepted rows give what they would have given without the
 * draft. Pages may be others then, so that the accepted rows are written again, at the second plan's slots.
 *   limits    seqs <= 4096; rows <= 2^30; max_pages * page_size <= 2^30; pages * page_size <= 2^30; page_size as in the pool.
 */
int amxfp4_paged_plan(const int32_t* lens, const int32_t* new_rows, int64_t seqs, int64_t rows, int64_t page_size,
                      int64_t pages, int64_t max_pages, const int32_t* state, int32_t* queue, int32_t* table,
                      int32_t* lens_out, int32_t* starts, int32_t* slots, int32_t* positions, int32_t* state_out,
                      void* stream);

/*
 * The new rows' queries, keys and values out of the fused projection: in [rows][ld] FP32 with q_heads heads of queries, then
 * kv_heads of keys, then kv_heads of values side by side, head_dim columns each.
 *   queries   rotated to positions[row] and rounded to BF16 as by amxfp4_split_heads_rope, written token-major: q_out
 *             [rows][q_heads][head_dim]. Rows of negative position are left as they were.
 *   keys      the same rotation and rounding, cast along head_dim as by amxfp4_quantize and stored at slots[row];
 *   values    rounded, cast and stored, not rotated. Bit for bit what the separate calls would give.
 *             Rows whose slot lies outside the pool (-1 of amxfp4_paged_plan) are not stored. Two rows with one slot: one of the
 *             two, or parts of both, are stored.
 *   fmt       group_size 32 (AMX_ERR_UNSUPPORTED otherwise).
 *   in        16-byte aligned, ld a multiple of 4; q_out 16-byte aligned. 1 <= q_heads <= 1024, theta > 1, rows <= 2^24.
 */
int amxfp4_paged_write(const amx_format_t* fmt, const amx_paged_pool_t* pool, const float* in, int64_t rows, int64_t ld,
                       int64_t q_heads, const int32_t* slots, const int32_t* positions, double theta, void* q_out_bf16,
                       void* stream);

/*
 * What the cache holds at `rows` slots, dequantized (Eq. 1; exact in both types, but 2^128, which a rounded power-of-two scale can give,
 * is infinite): k_out, v_out [rows][kv_heads][head_dim], 16-byte aligned, out_dtype 0 = float32, 1 = BF16 bit patterns. A slot outside
 * the pool gives a row of zeros. rows <= 2^24.
 */
int amxfp4_paged_read(const amx_format_t* fmt, const amx_paged_pool_t* pool, const int32_t* slots, int64_t rows,
                      int32_t out_dtype, void* k_out, void* v_out, void* stream);

/*
 * Attention of the new rows over everything their sequences hold, for the few rows to a sequence of decoding (one new token,
 * a draft being verified, a short chunk; right for any number). Row t of sequence b (starts[b] <= t < starts[b + 1]) and
 * query head h, which reads key / value head h / (q_heads / kv_heads):
 *     s_j = scale * sum_d q[t][h][d] K_hat[j][d]          for tokens j <= positions[t], j < lens[b]
 *     out[t][h][:] = bf16( sum_j exp(s_j - max s) V_hat[j][:] / sum_j exp(s_j - max s) )
 * FP32 throughout, but the weights exp(s_j - running max), each times a scale of V, are rounded to BF16 for the matrix
 * instructions; sums that leave FP32's range (of exp(s_j - max) |V_hat| too, before the division) are infinite. A row that sees no key (position -1) gets zeros; rows behind the last sequence's are left as they were. Keys in
 * pages whose id lies outside the pool are not seen. Tokens from lens[b] on may hold anything, infinite scales too. The
 * least power-of-two scale (byte 0, 2^-127) counts as 0.
 *   q_bf16     [rows][q_heads][head_dim], 16-byte aligned, finite in rows that see a key; out_bf16 [rows][q_heads * head_dim], 16-byte aligned.
 *   table      [seqs][max_pages]; lens [seqs], starts [seqs + 1] (ascending), positions [rows]: as amxfp4_paged_plan wrote
 *              them (its lens_out). A position from lens[b] on, up to 2^31 - 1, sees all that the sequence holds.
 *   max_keys   at least the largest of lens, or 0 if not known (max_pages * page_size then). Work is divided by it; a sequence
 *              that is longer all the same costs time only.
 *   workspace  at least amxfp4_paged_attention_workspace_bytes() bytes, 256-byte aligned (AMX_ERR_WORKSPACE otherwise); partial
 *              results of this call alone: calls that may run at the same time need one each.
 *   limits     group_size 32; q_heads a multiple of kv_heads, at most 1024; rows <= 2^24, rows * q_heads <= 2^31; seqs <= 4096;
 *              max_pages * page_size <= 2^30; 0 < scale <= 2^127.
 * The split of the work, and with it the order of the FP32 sums, depends on all sequences of the call: a sequence's result
 * is not bit for bit the same in another batch. The same call gives the same bits.
 */
size_t amxfp4_paged_attention_workspace_bytes(const amx_format_t* fmt, const amx_paged_pool_t* pool, int64_t rows,
                                              int64_t q_heads, int64_t seqs, int64_t max_keys);
int amxfp4_paged_attention(const amx_format_t* fmt, const amx_paged_pool_t* pool, const void* q_bf16, int64_t rows,
                           int64_t q_heads, const int32_t* table, int64_t seqs, int64_t max_pages, const int32_t* lens,
                           const int32_t* starts, const int32_t* positions, float scale, int64_t max_keys, void* out_bf16,
                           void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* AMXFP4_PAGED_H */
