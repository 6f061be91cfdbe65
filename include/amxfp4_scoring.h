/*
 * libamxfp4 — scoring text with a quantized model: attention whose rows see a range of keys each (documents packed into one
 * pass, prefixes that are read in both directions, windows, padding), scores that are capped by a tanh or fall with distance,
 * and the log probabilities of tokens.
 *
 * The paper evaluates by perplexity and by the likelihood of given answers (Sec. 5); the models it does so on need none of the
 * masks, caps and biases here, and it defines no operator for the logits. All of it is this library's.
 *
 * Conventions as in amxfp4.h: data pointers are DEVICE pointers owned by the caller, `fmt`, `pool` and `scores` are HOST
 * structures read during the call; nothing is allocated, retained or synchronised; arguments are validated on the host before
 * any launch, the return value is an amx_status_t, the message is available from amxfp4_last_error(). What lies on the device
 * cannot be validated there: the calls access no memory outside the buffers that they are given, whatever the ranges, targets
 * and tables say. Outputs and workspaces share no memory with anything else of a call; calls that may run at the same time need a workspace each.
 */
#ifndef AMXFP4_SCORING_H
#define AMXFP4_SCORING_H

#include <stddef.h>
#include <stdint.h>

#include "amxfp4.h"       /* amx_format_t, status codes */
#include "amxfp4_paged.h" /* amx_paged_pool_t */

#ifdef __cplusplus
extern "C" {
#endif

/*
 * What becomes of a score s = scale * q . k of a query at position p and a key at position j, before the softmax:
 *     cap > 0:         s = cap * tanh(s / cap)
 *     slopes != NULL:  s = s - slopes[h] * |p - j|        (h: the query head)
 * in this order. Both in FP32. The tanh is right to about 2^-22 of cap, absolutely (1 - 2 / (1 + exp 2x)). Scores up to 0.45 of the cap (from a cap of
 * 4096 scale on, and of scales up to 2^-20, up to 0.02 of it, from 2^30 scale on 2^-12) are right to 2^-21 of themselves (a polynomial): over the paged cache each by itself, in a prompt
 * where those of 32 neighbouring rows and 32 or 64 neighbouring keys all are so small. Raw products above 2^60 count as large.
 */
typedef struct {
  float cap;           /* 0: none; else 2^-20 to 2^20 */
  int32_t reserved;    /* 0 */
  const float* slopes; /* device, [q_heads], finite (beyond 2^90 either way as 2^90), 4-byte aligned, or NULL */
} amx_scores_t;

/*
 * amxfp4_attention_merged (amxfp4.h) for rows that see a range of keys each, with the scores above. Row i of the queries stands
 * at position p = pos0 + i, key j at position j. The row sees the keys
 *     max(first[i], 0) <= j <= min(last[i], Sk - 1)     (NULL: from the first key on; up to the last one)
 *     and, with causal != 0, j <= p only,
 * the same for all heads. Over these the recurrence of amxfp4_attention: key tiles of 32 in ascending order, the probabilities of a
 * tile cast as one group of `fmt` against the running maximum. A row that sees no key gives zeros.
 * (Weights come out of FP32 scores, so one next to a boundary of the cast may be cast to either side; a tile whose largest score, in units of log2, is within
 * 2^-16 and 2^-22 of itself of the running maximum counts as holding it in a power-of-two scale.)
 *   documents   packed into one pass: first[i] = where row i's document begins, causal.
 *   prefixes    read in both directions: last[i] = the end of the prefix for its rows, p for those behind it; causal = 0.
 *   windows     first[i] = p - window + 1, causal.
 *   padding     rows: last[i] = -1. Keys behind the last that any row sees are not looked at (Sk is rounded up to 32 by what the
 *               caller likes).
 *   fmt, heads, Sq, Sk, head_dim, codes, scales, scale: as amxfp4_attention (groups of 32, heads of 128 or 64, Sk a multiple of 32, Sq
 *               and Sk at most 2^20). Sq may exceed Sk. Scales of V that are
 *               not finite make all rows of a workgroup (128 neighbouring ones) that walks over them undefined, also those that do not see
 *               them; scales of K only the rows that see them.
 *   scores      HOST, or NULL for neither.
 *   causal      0 or 1; 0 <= pos0 <= 2^30.
 *   first, last device int32 [Sq], any values, 4-byte aligned, or NULL.
 *   out_bf16    device out, [Sq][q_heads * head_dim] BF16 bit patterns, 16-byte aligned.
 *   workspace   at least amxfp4_attention_masked_workspace_bytes() bytes (which are more than amxfp4_attention's), 256-byte aligned
 *               (AMX_ERR_WORKSPACE otherwise).
 * The same call gives the same bits. (Few rows against many keys are split over the keys: each range's maxima first, so that every tile is
 * cast against the running maximum of all keys before it, as without the split. Keys that a slope puts 2^-60 and more below a row's sum,
 * by the norms of the queries and keys, may not be looked at: each leaves the result off by up to 2^-59 of its value.)
 */
size_t amxfp4_attention_masked_workspace_bytes(const amx_format_t* fmt, int64_t q_heads, int64_t kv_heads, int64_t Sq, int64_t Sk,
                                               int64_t head_dim);
int amxfp4_attention_masked(const amx_format_t* fmt, int64_t q_heads, int64_t kv_heads, int64_t Sq, int64_t Sk, int64_t head_dim,
                            const uint8_t* Q_codes, const uint8_t* Q_scales, const uint8_t* K_codes, const uint8_t* K_scales,
                            const uint8_t* V_codes, const uint8_t* V_scales, float scale, const amx_scores_t* scores, int32_t causal,
                            int64_t pos0, const int32_t* first, const int32_t* last, void* out_bf16, void* workspace,
                            size_t workspace_bytes, void* stream);

/*
 * amxfp4_paged_attention (amxfp4_paged.h) with the scores above, p = positions[row] (cut to the sequence's last token, which shifts
 * all scores of a row alike). Everything else, the workspace's size included, as there; scores as for amxfp4_attention_masked.
 */
int amxfp4_paged_attention_scored(const amx_format_t* fmt, const amx_paged_pool_t* pool, const void* q_bf16, int64_t rows,
                                  int64_t q_heads, const int32_t* table, int64_t seqs, int64_t max_pages, const int32_t* lens,
                                  const int32_t* starts, const int32_t* positions, float scale, const amx_scores_t* scores,
                                  int64_t max_keys, void* out_bf16, void* workspace, size_t workspace_bytes, void* stream);

/*
 * Log probabilities out of logits. For every row, with x_v = logits[row][v], or cap * tanh(logits[row][v] / cap) where cap > 0
 * (a logit of -inf stays -inf: a token that is ruled out), in FP32:
 *     lse = log sum_v exp(x_v);   p_v = exp(x_v - lse)
 *     logprob      = x_target - lse           0 where the target is outside the vocabulary (-1: padding)
 *     entropy      = -sum_v p_v (x_v - lse)   (of tokens with p_v > 0), in nats
 *     top_ids, top_logprobs   the `top` largest logits in descending order, of equal ones the lowest id first; x - lse of each
 * A row of which all logits are -inf: logprob (of a target inside) and top_logprobs -inf, entropy 0, ids 0, 1, ... A row with a logit of NaN or
 * +inf: logprob (of a target inside), entropy and top_logprobs may be NaN, ids any (within the vocabulary, or -1).
 * Finite logits may be of any size, the type's lowest value (as which a token may be ruled out: with a cap it is -cap, as any other) among them; a log
 * probability below FP32's range is -inf.
 *   logits     dtype 0 = float32, 1 = BF16; [rows][ld], ld >= vocab, aligned to its elements' size. Columns from vocab on are not looked at. A product's
 *              output (amxfp4_gemm: C, ldc) as it is.
 *   targets    int32 [rows], or NULL; logprob [rows], NULL exactly when targets is; entropy [rows], or NULL.
 *   top        0 to 64, at most vocab; top_logprobs FP32 [rows][top], top_ids int32 [rows][top]: NULL exactly when top is 0.
 *   cap        0 (none), or 2^-20 to 2^20.
 *   workspace  at least amxfp4_token_logprobs_workspace_bytes() bytes, 256-byte aligned (AMX_ERR_WORKSPACE otherwise); may be NULL when that is 0.
 *   limits     1 <= rows <= 2^23, 1 <= vocab <= 2^24, ld <= 2^31, rows * ld <= 2^40. All pointers aligned to their elements' size.
 * The same call gives the same bits.
 */
size_t amxfp4_token_logprobs_workspace_bytes(int32_t dtype, int64_t rows, int64_t vocab, int64_t top);
int amxfp4_token_logprobs(const void* logits, int32_t dtype, int64_t rows, int64_t vocab, int64_t ld, const int32_t* targets, float cap,
                          int64_t top, float* logprob, float* entropy, float* top_logprobs, int32_t* top_ids, void* workspace,
                          size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* AMXFP4_SCORING_H */
