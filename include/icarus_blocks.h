/*
 * icarus_blocks.h -- decode over selected blocks of the paged cache, with lengths that stay on the GPU.
 *
 * The calls of icarus.h take lengths and row lists from the host.  The calls here read theirs from device memory, check
 * nothing on the host that only the device knows, and make the same launches whatever the lengths are: a step
 * made of them can be captured into a HIP graph once and replayed while the sequences grow.  They are the attention half
 * of a step for a program that runs its own projections, beside icarus_attn_shared_kv:
 *
 *   icarus_extend_sequences   lengths of the sequences -> block tables, and sequence, position and slot of every row
 *   icarus_rope_append        QK-RMSNorm (qk_norm), rotation, append of K and V to the pool
 *   icarus_key_bounds         largest and smallest key of each block, per channel, in 8 bits
 *   icarus_select_blocks      for each sequence and kv-head the blocks whose bounds promise the largest scores
 *   icarus_attn_blocks        attention over the selected blocks, one token per row
 *
 * As in icarus.h: an icarus_status is returned and icarus_last_error() explains it, the caller owns all device memory, all
 * work goes to the caller's stream (of the current device), the pool has the layout of that header, and the cache is
 * shared by all streams of a sequence.  Nothing is kept from one call for the next, so calls that do not touch the same
 * memory may overlap; a workspace belongs to one call at a time.
 * Pointers: float and code arrays, pool and workspace 16-byte aligned; integer arrays and scales aligned to their element.
 *
 * A call takes up to 65535 sequences (icarus_extend_sequences: 2^29, as many free ids), 2^29 rows and 2^30 queries of a kv-head; a table that
 * icarus_select_blocks chooses from up to 2^22 blocks of a sequence, and it makes up to 2^22 - 1 lists (sequences x kv-heads) of 2^22 entries; icarus_attn_blocks takes
 * lists of 2^22 entries, and 2^20 parts of 256 entries (an empty list: one) over all of them.  More is ICARUS_ERR_UNSUPPORTED, and a workspace for more has size 0.
 *
 * What the device finds out of range is not followed: a block id outside the pool, a position beyond the table, a slot outside
 * the pool or a negative length are skipped as each call says.  Results never depend on max_new and seq_rows, which
 * at most size a launch.
 */
#ifndef ICARUS_BLOCKS_H
#define ICARUS_BLOCKS_H

#include "icarus.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Sequence s holds ctx_lens[s] tokens and receives new_lens[s] more; streams[s] decoder rows (null: none) attend with the
 * last of them.  Its rows -- none without a new token -- are the new tokens in order, then one row per stream at the last new token's
 * position: with one new token the encoder row and the decoder rows of icarus_decode_step.  Rows of all sequences stand
 * one after the other, in the order of the sequences.
 * The new tokens go to the free places of the sequence's last block and then to blocks from free_ids, taken in the order of
 * the sequences from entry *free_used on; the ids are entered in the block table (no other entry is written).
 * A sequence is REFUSED whole -- its length stays, it takes no block, and its rows are entered as -1 -- where a length or
 * streams[s] is negative, the tokens pass max_position or the row of the table, its rows pass max_rows, or its blocks would pass
 * the end of the list (then every later sequence that needs a block is refused too, so that the blocks are handed out in order).
 * An id outside the pool is entered as -1, and tokens of such a block have slot -1.
 *   ctx_lens, new_lens, streams  device int32 [S]
 *   block_tables                 device int32 [S, max_blocks], in and out
 *   free_ids, free_used          device int32 [n_free] and [1] (taken as 0 or n_free where it is below or above)
 *   kv_lens                      device int32 [S]: ctx_lens + new_lens, or ctx_lens of a refused sequence; not ctx_lens itself
 *   row_start                    device int32 [S + 1]: first row of each sequence, at most max_rows; [S]: number of rows
 *   row_seq, row_pos, row_slot   device int32, int32, int64 [max_rows]: sequence, position, slot of the row's token in the pool; slot -1: the row
 *                                writes nothing (a stream); all -1: no row (of a refused sequence, or behind the last one)
 *   counts                       device int32 [2]: entries of free_ids that are taken now; sequences refused.  Not free_used itself */
icarus_status icarus_extend_sequences(icarus_ctx *ctx, int32_t S, const int32_t *ctx_lens, const int32_t *new_lens, const int32_t *streams,
                                      int32_t *block_tables, int32_t max_blocks, const int32_t *free_ids, int32_t n_free,
                                      const int32_t *free_used, int32_t max_rows, int32_t *kv_lens, int32_t *row_start,
                                      int32_t *row_seq, int32_t *row_pos, int64_t *row_slot, int32_t *counts, void *stream);

/* Row r of qkv holds the projections of one token: Hq query, Hkv key, Hkv value heads.  Query and key heads go through
 * RMSNorm (qk_norm) and are rotated to position row_pos[r]; q_out [R, Hq, D] receives the queries, the pool K and V at slot
 * row_slot[r].  Rows with a negative position are left out, q_out with them; with a slot outside the pool only the append
 * is left out and the row's K and V are not read.  The entries are those that icarus_prefill_kv and icarus_decode_step write, bit for bit, where their
 * projections (float32) are the same numbers.  Slots that are not named keep every byte.  Of a slot that is named twice each element is one of its rows'.
 *   qkv                 device, dtype elements, rows ld elements apart (ld >= (Hq + 2 Hkv) * D)
 *   row_pos, row_slot   device int32, int64 [R] */
icarus_status icarus_rope_append(icarus_ctx *ctx, const void *qkv, int64_t ld, int32_t R, const int32_t *row_pos,
                                 const int64_t *row_slot, void *q_out, void *kv_pool, void *stream);

/* Bounds of the keys of every block of sequence s that holds a position in [from_lens[s], to_lens[s]), over all of the block's positions
 * below to_lens[s].  hi[d], lo[d]: largest and smallest k[d] (a NaN counts as 0, an infinity as the largest finite value; FP8 cache:
 * of the codes' values, without k_scale).  With 2^e the smallest power of two, -40 <= e <= 40, with 127 * 2^e >= every |hi[d]| and |lo[d]|:
 *   codes[block][kv-head][0][d] = ceil(hi[d] / 2^e), codes[..][1][d] = floor(lo[d] / 2^e), at most 127 in size; scales[block][kv-head] = 2^e
 * so that code * scale bounds the keys (wherever e = 40 suffices).  Blocks outside the pool are left out.  A block of two sequences (a common
 * cached prefix) has to hold as many tokens for one as for the other.  After icarus_prefill_kv or icarus_decode_step: from_lens = the
 * lengths before, to_lens = after.
 *   block_tables          device int32 [S, max_blocks]
 *   from_lens, to_lens    device int32 [S]
 *   max_new               about the largest to_lens - from_lens, 0 if unknown: sizes the launch
 *   codes, scales         device int8 [num_blocks, Hkv, 2, D], float [num_blocks, Hkv] */
icarus_status icarus_key_bounds(icarus_ctx *ctx, const void *kv_pool, const int32_t *block_tables, int32_t max_blocks, int32_t S,
                                const int32_t *from_lens, const int32_t *to_lens, int32_t max_new, int8_t *codes, float *scales,
                                void *stream);

/* For every sequence and kv-head: which blocks to attend to, shared by the sequence's rows as the cache is.  Rows row_start[s] .. row_start[s + 1] - 1
 * of q belong to sequence s; their heads that use the kv-head are its queries.  Each query is brought to 8 bits as the keys are (its own 2^e, round
 * to nearest even; NaN counts as 0), and the score of a block is
 *     max over the queries of   2^e(query) * scale * sum over d of (q[d] > 0 ? q[d] * code_hi[d] : q[d] * code_lo[d])
 * -- whole numbers below 2^23 and powers of two, so it has one value whatever the order of the sum.  Of the ceil(kv_lens[s] / block_size) blocks
 * the first `first` and the last `last` are taken, then the ones with the largest scores until there are top_k; equal scores: the lowest index.  A block
 * whose id is outside the pool scores below all others; with no query all blocks score alike.
 *   q          device [R, Hq, D] as icarus_attn_blocks takes it
 *   kv_lens    device int32 [S]: tokens in the cache (negative: 0)
 *   row_start  device int32 [S + 1], not decreasing, within 0 .. R
 *   blocks     device int32 [S, Hkv, top_k]: indexes into the sequence's row of the table, ascending, -1 behind the last
 *   counts     device int32 [S]: how many, min(top_k, number of blocks)
 *   seq_rows   as icarus_attn_blocks takes it, not negative; the launches here go by S and max_blocks alone
 *   workspace  at least icarus_select_workspace_bytes(ctx, S, max_blocks) */
size_t icarus_select_workspace_bytes(const icarus_ctx *ctx, int32_t S, int32_t max_blocks);
icarus_status icarus_select_blocks(icarus_ctx *ctx, const void *q, const int8_t *codes, const float *scales, const int32_t *block_tables,
                                   int32_t max_blocks, int32_t S, const int32_t *kv_lens, int32_t R, const int32_t *row_start,
                                   int32_t seq_rows, int32_t top_k, int32_t first, int32_t last, int32_t *blocks, int32_t *counts,
                                   void *workspace, size_t workspace_bytes, void *stream);

/* out[r, h] = softmax(q[r, h] K^T / sqrt(D)) V over the positions below kv_lens[s] of the blocks that blocks[s][kv-head of h][0 .. counts[s]) names, for
 * the rows r of each sequence s.  S, R, the kv-heads and max_selected say how the sums of a list are split: calls that differ in one of them agree up to rounding.  Entries outside the table, blocks outside the pool and positions from kv_lens[s] on are
 * left out; a block named twice counts twice.  A row that has nothing to attend to, or
 * only scores of minus infinity, becomes zeros; a NaN or a score of plus infinity makes NaN, as in the formula; rows of no sequence keep what out holds.
 *   blocks, counts   device int32 [S, Hkv, max_selected] and [S], as icarus_select_blocks gives them (in any order)
 *   seq_rows         about the most rows of a sequence, 0 if unknown: sizes the launch
 *   out              device [R, Hq, D], no memory of q
 *   workspace        at least icarus_attn_blocks_workspace_bytes(ctx, S, R, max_selected) */
size_t icarus_attn_blocks_workspace_bytes(const icarus_ctx *ctx, int32_t S, int32_t R, int32_t max_selected);
icarus_status icarus_attn_blocks(icarus_ctx *ctx, const void *q, const void *kv_pool, const int32_t *block_tables, int32_t max_blocks,
                                 int32_t S, const int32_t *kv_lens, int32_t R, const int32_t *row_start, int32_t seq_rows,
                                 const int32_t *blocks, const int32_t *counts, int32_t max_selected, void *out, void *workspace,
                                 size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* ICARUS_BLOCKS_H */
