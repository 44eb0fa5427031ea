/*
 * bana_tokens.h -- C ABI of libbana.so for new tokens and for the blocks of the paged K/V cache.
 *
 * What a serving program does with the cache of bana.h besides attending to it from one token per
 * sequence: it writes the keys and values of new tokens (bana_append_kv), attends from several new
 * tokens of a sequence at once -- the drafts of a speculative step (bana_tree_attn), a prompt, a piece
 * of one or a single token under a sliding window (bana_window_attn) -- and hands blocks out, shares
 * them, moves tokens together and takes blocks back without asking the host (bana_reserve_kv_blocks,
 * bana_fork_kv_seqs, bana_compact_kv_tokens, bana_release_kv_blocks).
 *
 * The conventions of bana.h hold: caller-owned device memory, 16-byte aligned and densely packed;
 * nothing is allocated, nothing synchronises, no state is kept between calls; host-checkable errors
 * return before any HIP call.  Pools, block tables and bana_dims are those of bana.h.  Of bana_dims
 * these calls read the shapes and, as hints for the attention, max_range_tokens (the most cached
 * tokens of a sequence, new ones included) and total_range_tokens (their sum over sequences); the other
 * hints must be valid and are ignored.  Without max_range_tokens the attention is split over workgroups
 * for sequences as long as the table: much shorter ones are split less, or not at all.  Values that live on
 * the device are not checked on the host, but no value makes a call read or write outside the buffers it
 * was given: offsets outside the rows, the table or the pool are clamped or skipped.  A wrong value gives
 * wrong results, not a fault.
 *
 * Packed rows.  The new tokens of a batch are rows of dense arrays: sequence b has the rows
 * [row_begin[b], row_begin[b + 1]), n_b of them (possibly none); row_begin is int32 [batch + 1] and
 * does not decrease.  The arrays hold `rows` rows; rows outside [row_begin[0], row_begin[batch]) belong
 * to no sequence: they are not read, and nothing is written there.  rows = 0 does nothing.
 */
#ifndef BANA_TOKENS_H
#define BANA_TOKENS_H

#include "bana.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Type of an attention result. */
#define BANA_OUT_F32 0
#define BANA_OUT_BF16 1

/*
 * Attention of drafted tokens.  Row r = row_begin[b] + i is node i of the tree drafted for sequence b;
 * the keys and values of the nodes are in the cache, node j at token tree_begin[b] + j.  A node sees the
 * tokens of the ranges [kv_range_begin[p][b], kv_range_end[p][b]), p < n_parts (a token covered twice
 * counts twice), and node j < min(n_b, 64) where bit j of tree_mask[r] is set:
 *   out[r][h] = sum_t exp(scale q[r][h].k_t - lse) v_t,   lse[r][h] = ln sum_t exp(scale q[r][h].k_t)
 * A row that sees nothing gives out = 0, lse = -inf.  tree_begin[b] < 0: the nodes are not in
 * this call's cache (another partition has them), rows see the ranges only.  Scores and sums are fp32; with
 * an fp32 result the weights enter the product with the values to 24 bits, with a bf16 result rounded to
 * bf16.  The fp32 result and lse of several calls over disjoint tokens merge exactly with
 * bana_merge_partials (batch = rows).  A NaN or +inf among a row's scores makes the row NaN; a row whose
 * scores are all -inf gives 0 and -inf as one that sees nothing does.  A value that is not finite gives the rows
 * that see it, in its dim, what the formula gives: +-inf, or NaN for a NaN, both signs or a weight that is 0 in
 * fp32.  (The sums are of weights up to 2^8: finite values below 2^90 never overflow them.)  What a row does not
 * see never reaches it, whatever its keys and values hold.
 *   q           bf16 [rows][num_q_heads][128]
 *   kv_range_*  int32 [n_parts][batch], 1 <= n_parts <= 63
 *   tree_begin  int32 [batch]
 *   tree_mask   uint64 [rows]; bits from n_b on are ignored
 *   out         fp32 or bf16 (out_type) [rows][num_q_heads][128]
 *   lse         fp32 [rows][num_q_heads], or NULL
 *   scale       > 0, finite
 * workspace: optional, bana_tree_attn_workspace_bytes bytes let the library split long ranges over
 * workgroups (with less the call runs unsplit, the same result up to rounding).  Calls that may overlap must
 * not share one; its contents need no initialisation.  Results are bit-identical run to run for the same
 * inputs and dims.  BANA_ERR_UNSUPPORTED: rows of 2^24 or rows * num_q_heads of 2^26 or more,
 * batch * num_kv_heads above 2^23, n_parts above 63, n_parts * max_blocks_per_seq above 2^30.
 */
bana_status bana_tree_attn(const bana_dims* d, int64_t rows, const int32_t* row_begin, const void* q,
                           const void* k_cache, const void* v_cache, const int32_t* block_table,
                           const int32_t* kv_range_begin, const int32_t* kv_range_end, int32_t n_parts,
                           const int32_t* tree_begin, const uint64_t* tree_mask, float scale, void* out,
                           int32_t out_type, float* lse, void* workspace, size_t workspace_bytes, void* stream);
size_t bana_tree_attn_workspace_bytes(const bana_dims* d, int64_t rows, int32_t n_parts);

/*
 * Attention of new tokens under a sliding window whose first tokens stay visible ("sinks").  The keys
 * and values of the new tokens are in the cache; seq_lens[b] counts them.  Row r = row_begin[b] + i is
 * the token at position pos = seq_lens[b] - n_b + i and sees the tokens t <= pos with pos - t < window or
 * t < sinks, of these the ones in [kv_range_begin[b], kv_range_end[b]) where those are given
 * (both or neither NULL; int32 [batch]: the tokens of one partition, merged as above).  A row at a negative
 * position sees nothing.
 * window >= 1 (INT32_MAX: no window, plain causal attention), sinks >= 0.  n_b may be 1 (a decode step),
 * seq_lens[b] (a whole prompt) or anything between.  Everything else as for bana_tree_attn.
 */
bana_status bana_window_attn(const bana_dims* d, int64_t rows, const int32_t* row_begin, const void* q,
                             const void* k_cache, const void* v_cache, const int32_t* block_table,
                             const int32_t* seq_lens, const int32_t* kv_range_begin, const int32_t* kv_range_end,
                             int32_t window, int32_t sinks, float scale, void* out, int32_t out_type, float* lse,
                             void* workspace, size_t workspace_bytes, void* stream);
size_t bana_window_attn_workspace_bytes(const bana_dims* d, int64_t rows, int32_t window, int32_t sinks);

/*
 * Keys and values of new tokens into the cache: row row_begin[b] + i becomes token first_token[b] + i of
 * sequence b, bit for bit.  Rows whose token lies outside the table, or whose table entry names no block of the pool,
 * are skipped.  Two rows of one call must not name the same slot, and the blocks written must belong to one sequence
 * only: a whole block that a fork shares stays shared when a release cuts into it.  Of d, num_q_heads is not used.
 * BANA_ERR_UNSUPPORTED: rows as above, batch * num_kv_heads above 2^18.
 *   k_rows, v_rows  bf16 [rows][num_kv_heads][128]
 */
bana_status bana_append_kv(const bana_dims* d, int64_t rows, const int32_t* row_begin, const int32_t* first_token,
                           const void* k_rows, const void* v_rows, const int32_t* block_table, void* k_cache,
                           void* v_cache, void* stream);

/*
 * The kept tokens of each sequence moved together, in place: token first_token[b] + i becomes what token
 * first_token[b] + kept[b][i] was, i < n_kept[b], bit for bit.  kept[b] increases strictly from
 * kept[b][0] >= 0 on (an accepted path among drafted tokens, or what an eviction leaves of a sequence).
 * The tokens behind the last one moved keep what they held.  The blocks written must belong to one
 * sequence only.  Tokens outside the table or in no block of the pool are skipped.  BANA_ERR_UNSUPPORTED:
 * batch * num_kv_heads above 2^18, max_kept of 2^30 or more.
 *   kept    int32 [batch][max_kept]
 *   n_kept  int32 [batch], clamped to [0, max_kept]
 */
bana_status bana_compact_kv_tokens(const bana_dims* d, void* k_cache, void* v_cache, const int32_t* block_table,
                                   const int32_t* first_token, const int32_t* kept, int32_t max_kept,
                                   const int32_t* n_kept, void* stream);

/*
 * Blocks handed out, shared and taken back.  block_refs, int32 [num_blocks], counts for each block of
 * the pool the table entries that name it; a block with the count 0 is free.  Table entries are -1 where
 * a sequence has no block.  *status, int32 in device memory, is raised to the highest code that applies
 * and never lowered: the caller sets it to 0 once and looks at it when it next waits for the device.
 *   1  too few free blocks                              (reserve, fork: the call changed nothing else)
 *   2  a sequence index outside [0, batch), a destination named twice or that is a source as well, or one
 *      whose first table entry is not -1                (fork: the call changed nothing else)
 *   3  a table too short for the tokens asked for       (reserve: the call changed nothing else)
 *   4  a table entry that names no block of the pool, or whose block has no reference left
 *      (release: the entry is cleared; fork: see there)
 * All results are the same from run to run.  These calls change one table: they must not overlap.
 * workspace (bana_kv_blocks_workspace_bytes bytes, needed): not shared by calls that may overlap.
 *
 * bana_reserve_kv_blocks: for every sequence b the entries j in [ceil(seq_lens[b] / 16),
 * ceil(need_lens[b] / 16)) that are -1 receive the free blocks of the lowest numbers, in the order of
 * (b, j); their counts become 1.
 * bana_fork_kv_seqs: for i < n, sequence dst_seq[i], which has no block, becomes a copy of sequence
 * src_seq[i]: its whole blocks are shared (counts + 1), a last block that is only partly filled is copied
 * into the free block of the lowest number left, in the order of i (count 1),
 * seq_lens[dst_seq[i]] = seq_lens[src_seq[i]] (clamped to the table's span).  One source may have several
 * destinations.  An entry of a source that names no block of the pool, or one without references: a whole block's is
 * copied and its count left alone; a partly filled one's tokens are copied if there are any (the destination has its
 * free block in any case); a block without references that a source names is no free block of this call.  Status 4.
 * bana_release_kv_blocks: for every sequence the entries from ceil(keep_lens[b] / 16) on are given back:
 * count - 1, entry -1 (keep_lens[b] <= 0: all of them; beyond the table: none).
 * Of d, num_q_heads is not used; nor are the heads in reserve and release.  BANA_ERR_UNSUPPORTED:
 * num_blocks above 2^31 - 1, n of 2^20 or more, in reserve a table of 2^31 entries or more.
 */
bana_status bana_reserve_kv_blocks(const bana_dims* d, int32_t* block_table, const int32_t* seq_lens,
                                   const int32_t* need_lens, int32_t* block_refs, int32_t* status, void* workspace,
                                   size_t workspace_bytes, void* stream);
bana_status bana_fork_kv_seqs(const bana_dims* d, const int32_t* src_seq, const int32_t* dst_seq, int32_t n,
                              void* k_cache, void* v_cache, int32_t* block_table, int32_t* seq_lens,
                              int32_t* block_refs, int32_t* status, void* workspace, size_t workspace_bytes,
                              void* stream);
bana_status bana_release_kv_blocks(const bana_dims* d, int32_t* block_table, const int32_t* keep_lens,
                                   int32_t* block_refs, int32_t* status, void* stream);
size_t bana_kv_blocks_workspace_bytes(const bana_dims* d);

#ifdef __cplusplus
}
#endif

#endif /* BANA_TOKENS_H */
