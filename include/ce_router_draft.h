/*
 * Drafted decoding over the paged key/value cache, beside ce_router_paged.h.
 *
 * Decoding reads the compressed cache of the routed layers (section 3.4,
 * task-adaptive token compaction) once a step whatever the number of new tokens,
 * so a program drafts several, as a tree, and lets the model verify them together:
 *
 *   1. ce_kv_reserve            pages and slots for every row of the trees
 *   2. ce_draft_masks           who sees whom, and positions, from the parents
 *   3. ce_kv_append             keys and values of all rows (per layer)
 *   4. ce_paged_tree_attention  attention under the masks (per layer)
 *   5. ce_verify_drafts         which rows the target's probabilities accept, and the next token
 *   6. ce_kv_keep               the accepted rows move up in the pages (per layer)
 *   7. ce_kv_trim               lengths, and the other rows' pages, go back
 *
 * Row 0 of a sequence is its last accepted token, which is not in the cache
 * before the step; rows 1 .. are the drafted ones. The conventions of ce_router.h
 * and ce_router_paged.h hold.
 */
#ifndef CE_ROUTER_DRAFT_H
#define CE_ROUTER_DRAFT_H

#include "ce_router_paged.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Status bits of ce_draft_masks, beside CE_DEV_BAD_OFFSETS and CE_DEV_OVERFLOW. */
enum {
  CE_DEV_BAD_TREE = 32, /* a parent was not before its row; the row was taken for one without a parent */
  CE_DEV_TOO_WIDE = 64  /* a sequence has more rows than its masks have bits: the bits behind are left out */
};

/*
 * The trees of a step: sequence b has rows [offsets[b], offsets[b + 1]).
 *   offsets       device int32 [B+1], offsets[0] = 0, non-decreasing (clamped to [0, row_capacity])
 *   parents       device int32 [row_capacity]: the parent's row of the same sequence (0 its
 *                 row 0), always before the row itself; negative: none (row 0, and rows that
 *                 no walk from row 0 reaches). NULL: chains, the parent of row i is i - 1
 *   tokens        device int32 [row_capacity]: the token of each row; ce_verify_drafts only
 *   row_capacity  host upper bound on the rows: sizes the arrays
 * Limits: 1 <= B <= 65535, row_capacity < 2^24.
 */
typedef struct ce_drafts {
  int32_t B;
  int32_t row_capacity;
  const int32_t* offsets;
  const int32_t* parents;
  const int32_t* tokens;
} ce_drafts;

/*
 * The masks of the trees. Row i of a sequence gets bit j (of word j / 32, at j % 32) where
 * j is i itself or an ancestor of i.
 *   mask_words  32-bit words a row, 1 to 64
 *   base        device int32 [B] or NULL (0): position of row 0 of each sequence
 *   mask        device uint32 [row_capacity x mask_words] out, or NULL
 *   positions   device int32 [row_capacity] out, or NULL: base + the row's ancestors, as
 *               ce_rotary takes them
 *   status      device uint32 [1] out, or NULL: CE_DEV_* bits of this call
 * Rows behind the last sequence are left as they were. Deterministic, but where the offsets
 * are out of order (a row that lies in two sequences may have bits of both). A sequence of
 * more than 8192 rows is worked on 2048 at a time: positions of a chain of 65536 0.6 ms, with
 * masks of 64 words 4.2.
 * Errors: CE_ERR_INVALID_ARG for null pointers / sizes, CE_ERR_UNSUPPORTED outside the
 * limits, CE_ERR_HIP.
 */
int ce_draft_masks(const ce_drafts* drafts, int32_t mask_words, const int32_t* base, uint32_t* mask, int32_t* positions,
                   uint32_t* status, void* stream);

/*
 * Attention of new tokens over the paged cache as ce_paged_attention, whose arguments,
 * workspace and errors it has, with M given by bits: a sequence's tokens before its n_q
 * new ones (the last n_q of lens[b]) are seen by all its queries, new token j by
 * query i where bit j of row i of the mask is set, whatever the order of i and j. So the
 * masks of trees, and of prompts whose image tokens see each other.
 *   attn->causal  0
 *   mask          device uint32 [attn->q_capacity x mask_words]: the row of each row of q
 *   mask_words    1 to 64; new tokens behind the last bit, 32 mask_words of a sequence, are not seen
 * Bits from n_q on are not used. A query that sees no token outputs zeros.
 */
int ce_paged_tree_attention(const ce_kv_cache* cache, const ce_paged_attn* attn, const uint32_t* mask, int32_t mask_words,
                            const void* q, int64_t q_ld, void* o, void* ws, size_t ws_bytes, void* stream);

/*
 * Verification of drafted tokens against the target's probabilities, which keeps the
 * target's distribution. With p_r = softmax(logits[r] / T) of row r of a tree, the walk begins
 * at row 0 and moves from row r to an accepted child of r until there is none.
 *   - draft_probs NULL (drafts are chosen, not drawn): a token is sampled from p_r by
 *     u_sample[r]; the child with that token is accepted (of several the first). The
 *     sample of the row where the walk ends is the next token.
 *   - else draft_probs[r] = q_r is the distribution that the children of row r were drawn
 *     from, independently, in row order. With c = 0 and S = 1 at first, a child x
 *     with the number u = u_accept[child] is accepted if u q_r(x) S < max(p_r(x) - c q_r(x), 0);
 *     if it is not, c grows by S, S becomes sum_i max(p_r(i) - c q_r(i), 0), and the next child is
 *     asked. Where the walk ends the next token is sampled from max(p_r - c q_r, 0) / S
 *     (from p_r if S is 0).
 *   A sample of weights w by u is the first i with w_0 + .. + w_i > u (w_0 + .. + w_(vocab-1)),
 *   the last i of a positive weight where rounding leaves none. Weights below 2^-800 of a
 *   row's largest count as none (up to 2^-780 they may).
 *   T is not positive (or NaN): p_r is 1 at the lowest index of the largest logit, and the child with
 *   that token is accepted, with draft_probs as without.
 * Logits of NaN count as -infinity; where some are +infinity they share all probability. A row
 * without a logit above -infinity has no distribution: its walk ends there, without a next
 * token (-1). Drafted tokens outside [0, vocab) are not accepted, and not asked.
 *   logits       device dtype (CE_BF16 or CE_F32): row_capacity rows, row r at r * logits_ld elements,
 *                vocab of them; rows need no alignment beyond the element's
 *   temperature  device float32 [B] or NULL (1)
 *   draft_probs  device float32, row r at r * probs_ld, or NULL; negative and NaN count as 0
 *   u_accept     device float32 [row_capacity] in [0, 1); NULL without draft_probs
 *   u_sample     device float32 [row_capacity] in [0, 1)
 *   kept_rows    device int32 [row_capacity] out: for each sequence, from its offset on, the rows of
 *                the walk, ascending, row 0 first, then -1
 *   n_kept       device int32 [B] out: their number, 0 for a sequence without rows
 *   next_token   device int32 [B] out: the token after the walk's last row, -1 if there is none
 *   ws           device workspace of ce_verify_workspace_size(drafts, vocab, draft_probs != NULL) bytes,
 *                256-byte aligned, contents on entry do not matter; calls that may overlap,
 *                captured ones among them, need workspaces of their own
 * With draft_probs the first rejection of a sequence is worked on by the whole device, each further one, of
 * a sibling or farther down the walk, by one workgroup of the sequence's that reads the row again: 17 us each at
 * vocab 32000, 60 to 75 at 131072. Each row looks for its children among the rows behind it, which for a
 * sequence of very many rows takes a time that grows with their square: 65536 children of one row 1.4 ms.
 * Exponentials, sums and comparisons are of 64 bits. Entries of kept_rows behind the
 * last sequence are left as they were. Where the offsets are out of order a sequence that
 * shares rows with another may have no walk: n_kept 0, next_token -1, and its entries of
 * kept_rows left as they were. Deterministic.
 * Limits: 1 <= vocab < 2^24, row_capacity * vocab < 2^40, B * ceil(vocab / 4096) < 2^24. Errors: CE_ERR_INVALID_ARG for null
 * pointers, sizes, or a u_accept without draft_probs or the reverse; CE_ERR_UNSUPPORTED
 * outside the limits; CE_ERR_WORKSPACE; CE_ERR_HIP.
 */
size_t ce_verify_workspace_size(const ce_drafts* drafts, int32_t vocab, int with_probs);
int ce_verify_drafts(const ce_drafts* drafts, int32_t vocab, const void* logits, int64_t logits_ld, int dtype,
                     const float* temperature, const float* draft_probs, int64_t probs_ld, const float* u_accept,
                     const float* u_sample, int32_t* kept_rows, int32_t* n_kept, int32_t* next_token, void* ws,
                     size_t ws_bytes, void* stream);

/*
 * The accepted rows of a step move up in the pages: token start[b] + j becomes what token
 * start[b] + kept_rows[offsets[b] + j] was, for j < n_kept[b].
 *   offsets, row_capacity  as in ce_drafts
 *   start      device int32 [B]: ce_kv_reserve's; a sequence that it refused (-1) is left as it is
 *   kept_rows, n_kept  ce_verify_drafts'. From the first entry on that is not above the one
 *              before it, or is no row of the sequence, the rows stay where they are
 * Keys and values are copied as they are; tokens past the table's row or on a page number out of
 * range are skipped. Deterministic. Errors as ce_kv_append.
 */
int ce_kv_keep(const ce_kv_cache* cache, const int32_t* offsets, int32_t row_capacity, const int32_t* start,
               const int32_t* kept_rows, const int32_t* n_kept, void* stream);

/*
 * And the lengths follow: lens_out[b] = min(lens[b], start[b] + n_kept[b]), or lens[b] where start[b]
 * is negative. Pages that hold no token any more are pushed on the free stack, sequences in
 * order, each sequence's pages in table order; the table keeps their numbers, which no
 * call reads behind the new length.
 *   cache       as in ce_kv_reserve (k and v are not touched)
 *   lens        device int32 [B]: ce_kv_reserve's lens_out
 *   start, n_kept  as in ce_kv_keep
 *   free_pages, free_count, lens_out, free_count_out  as in ce_kv_reserve
 *   status      device uint32 [1] out or NULL: CE_DEV_BAD_CACHE where a length, count or page
 *               number was out of its range, or more pages came back than the stack has room for
 * Calls on one pool must not overlap. Deterministic. Errors as ce_kv_reserve.
 */
int ce_kv_trim(const ce_kv_cache* cache, const int32_t* lens, const int32_t* start, const int32_t* n_kept,
               int32_t* free_pages, const int32_t* free_count, int32_t* lens_out, int32_t* free_count_out,
               uint32_t* status, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* CE_ROUTER_DRAFT_H */
