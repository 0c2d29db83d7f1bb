/*
 * The paged key/value cache of routed layers, beside ce_router.h (which holds
 * the routed block, the types and the status codes).
 *
 * The retained tokens of a routed layer are packed into a shorter sequence and
 * their keys and values are the compressed cache that decoding reuses (section
 * 3.4, task-adaptive token compaction). How many rows a layer adds to a
 * sequence is known only on the device (ce_topk_compact's kept_offsets), so
 * the memory of the cache is handed out there too, in pages:
 *
 *   1. ce_kv_reserve       pages and slots for the new rows of every sequence
 *   2. ce_kv_append        the new keys and values into their slots
 *   3. ce_paged_attention  attention of the new tokens over the cache
 *
 * The conventions of ce_router.h hold: caller-owned device buffers, 16-byte
 * aligned; validation on the host before anything is enqueued; no allocation,
 * no synchronisation, no copies to the host; no read or write out of bounds
 * whatever the device data say.
 */
#ifndef CE_ROUTER_PAGED_H
#define CE_ROUTER_PAGED_H

#include "ce_router.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element type of 8-bit pages: OCP e4m3 (largest value 448, NaN, no infinity). */
enum { CE_E4M3 = 2 };

/* Status bits of ce_kv_reserve, beside CE_DEV_BAD_OFFSETS and CE_DEV_OVERFLOW. */
enum {
  CE_DEV_NO_PAGES = 4,  /* the free pages did not suffice for every sequence           */
  CE_DEV_TOO_LONG = 8,  /* a sequence would outgrow its row of the page table          */
  CE_DEV_BAD_CACHE = 16 /* a length or count out of its range was clamped, or a page number out of
                         * its range was given back or handed out (as it is: its rows get no slot) */
};

/*
 * A cache of B sequences. Token j of sequence b sits in row j % page_size of
 * page page_table[b * max_pages + j / page_size].
 *   k, v         device dtype, page p at p * page_stride elements, each
 *                [n_kv_heads x page_size x head_dim]: the rows of one head are
 *                contiguous, as attention reads them
 *   page_stride  elements between pages, >= n_kv_heads * page_size * head_dim, a
 *                multiple of 16, below 2^31 (several layers may interleave in one
 *                allocation)
 *   k_scale, v_scale  CE_E4M3: device float32 [n_kv_heads], positive and finite, or
 *                both NULL (1): a stored value x stands for x * scale. CE_BF16: NULL
 *   page_table   device int32 [B x max_pages]; entries behind a sequence's last
 *                page are not read
 * Limits: head_dim 128; page_size a power of two from 16 to 256; n_pages *
 * page_size below 2^31, max_pages * page_size at most 2^30; 1 <= B <= 65535.
 */
typedef struct ce_kv_cache {
  int32_t B;
  int32_t n_kv_heads;
  int32_t head_dim;
  int32_t page_size;
  int32_t n_pages;
  int32_t max_pages;
  int32_t dtype; /* CE_BF16 or CE_E4M3 */
  int64_t page_stride;
  void* k;
  void* v;
  const float* k_scale;
  const float* v_scale;
  int32_t* page_table;
} ce_kv_cache;

/*
 * Pages and slots for the new rows of a step (section 3.4: the packed rows
 * that the compressed cache grows by). Sequence b has lens[b] tokens in the
 * cache (none, and its pages go back, where reset[b] != 0) and gets n_b =
 * new_offsets[b + 1] - new_offsets[b] more (ce_topk_compact's kept_offsets).
 *   - pages given back are pushed on the free stack, sequences in order, each
 *     sequence's pages in table order (users of a page are not counted: one that
 *     stands in two rows of the table, which ce_paged_attention may read, would be
 *     pushed by each of them, so only one of the two may be handed on);
 *   - then every sequence in order pops the pages it still needs from the top
 *     into its row of the table. A sequence is refused, and stays as it is
 *     (after its reset), if its row of the table is too short, or if it needs
 *     pages and these and those that the sequences before it needed (refused
 *     for want of pages or not) are more than the stack holds;
 *   - row r of sequence b becomes token start[b] + r - new_offsets[b], in slot
 *     page * page_size + row of the page. Rows of a refused sequence (start -1) are not
 *     in the cache: ce_kv_append skips them, and what ce_paged_attention gives for
 *     them is attention over the end of what the cache holds, not their answer.
 *   cache       k and v are not touched (and may be NULL); n_kv_heads, head_dim,
 *               dtype, page_stride are not read
 *   lens        device int32 [B]
 *   new_offsets device int32 [B+1], or NULL: no new rows (row_capacity is then 0)
 *   row_capacity  host upper bound on the new rows: entries of slots
 *   reset       device uint8 [B] or NULL
 *   free_pages  device int32 [n_pages]: the free stack, its lowest *free_count entries in use
 *   free_count  device int32 [1]
 *   lens_out    device int32 [B] out, may be lens: lengths with the new rows
 *   free_count_out  device int32 [1] out, may be free_count
 *   start       device int32 [B] out: position of the first new row, -1 where refused
 *   slots       device int32 [row_capacity] out: slot of each row; -1 for rows of
 *               refused sequences and rows behind the last
 *   status      device uint32 [1] out or NULL: CE_DEV_* bits of this call
 * Calls on one pool change it and must not overlap. Deterministic, but where the
 * offsets are out of order (CE_DEV_BAD_OFFSETS): a row that lies in the ranges of
 * several sequences then has the slot of one of them. Errors:
 * CE_ERR_INVALID_ARG for null pointers / sizes, CE_ERR_UNSUPPORTED outside the
 * limits, CE_ERR_HIP.
 */
int ce_kv_reserve(const ce_kv_cache* cache, const int32_t* lens, const int32_t* new_offsets, int32_t row_capacity,
                  const uint8_t* reset, int32_t* free_pages, const int32_t* free_count, int32_t* lens_out,
                  int32_t* free_count_out, int32_t* start, int32_t* slots, uint32_t* status, void* stream);

/*
 * New keys and values into the pages (section 3.4, compressed cache).
 *   k_new, v_new  device bf16: row r at r * k_ld (v_ld) elements, its n_kv_heads x
 *                 head_dim values contiguous (a part of a fused projection's rows);
 *                 k_ld, v_ld multiples of 8
 *   slots         device int32 [rows]: ce_kv_reserve's; rows whose slot is outside
 *                 [0, n_pages * page_size) are skipped. Rows with the same slot race:
 *                 each 16 bytes of the page are one row's
 * CE_BF16 pages take the values as they are, CE_E4M3 pages x / scale (one float32
 * division) limited to +-448 and rounded to nearest even; NaN stays NaN.
 * The page table is not read. Errors as ce_kv_reserve.
 */
int ce_kv_append(const ce_kv_cache* cache, const void* k_new, int64_t k_ld, const void* v_new, int64_t v_ld,
                 const int32_t* slots, int32_t rows, void* stream);

/*
 * Attention of new tokens over the paged cache, which holds theirs as well
 * (section 3.4): a chunk of a prompt, single tokens, and batches of both. With
 * kv(h) = h / (n_heads / n_kv_heads) and n_k = lens[b], for each sequence b and head h
 *   O_b[:, h] = softmax(scale * Q_b[:, h] K_b[:, kv(h)]^T + M) V_b[:, kv(h)]
 * M = 0, or with causal != 0, -inf for token j > i + (n_k - n_q) (end-aligned). A
 * query that sees no token outputs zeros; what it does not see has no influence,
 * NaN and infinities included.
 */
typedef struct ce_paged_attn {
  int32_t n_heads;          /* query heads; a multiple of the cache's n_kv_heads */
  int32_t q_capacity;       /* rows of q and o (grid bound; offsets are clamped to it) */
  const int32_t* q_offsets; /* device int32 [B+1]: new rows of each sequence */
  const int32_t* lens;      /* device int32 [B]: tokens of each in the cache, the new ones included */
  int32_t causal;           /* 0 or 1 */
  float scale;              /* softmax scale > 0 */
} ce_paged_attn;

/*
 *   q   device bf16: row r at r * q_ld elements, its n_heads x head_dim values
 *       contiguous; q_ld a multiple of 8, below 2^22
 *   o   device bf16 [q_capacity x n_heads x head_dim] out (rows of real queries only)
 *   ws  device workspace of ce_paged_workspace_size(cache, attn) bytes, 256-byte
 *       aligned, contents on entry do not matter. Calls that may overlap, captured
 *       ones among them, need workspaces of their own
 * Lengths are clamped to [0, max_pages * page_size]; a page number outside
 * [0, n_pages) reads as zeros. fp32 scores, statistics and accumulation (scale * k_scale
 * and scale * Q K^T may be past float32 or round to zero, the products of Q with stored
 * keys may not be past it); the probabilities are rounded to bf16 for the product with V.
 * Deterministic.
 * Errors: CE_ERR_INVALID_ARG for null pointers, sizes, a scale that is not
 * positive with scale * log2 e finite or causal outside {0, 1}; CE_ERR_UNSUPPORTED outside
 * the limits, for more than 4096 query heads a key/value head, q_capacity * n_heads
 * >= 2^28 or B * n_kv_heads >= 2^22;
 * CE_ERR_WORKSPACE; CE_ERR_HIP.
 * ce_paged_workspace_size depends on the sizes in cache and attn only (no device
 * pointer is read), is at most 35135744 bytes, and 0 where none is used or the call
 * would refuse the sizes.
 */
size_t ce_paged_workspace_size(const ce_kv_cache* cache, const ce_paged_attn* attn);
int ce_paged_attention(const ce_kv_cache* cache, const ce_paged_attn* attn, const void* q, int64_t q_ld, void* o,
                       void* ws, size_t ws_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* CE_ROUTER_PAGED_H */
