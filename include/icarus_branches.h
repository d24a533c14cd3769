/*
 * icarus_branches.h -- sequences that branch over a shared prefix: beams and samples that fork, end and read a common prefix once.
 *
 * The calls belong beside those of icarus_blocks.h and follow its rules: lengths, tables and choices stay on the device, nothing that
 * only the device knows is checked on the host, and the launches go by the arrays' sizes alone, so that a step made of them can be captured
 * into a HIP graph.  A group is a run of consecutive sequences.  A step of a beam search:
 *
 *   icarus_beam_select        logits and scores of a group's beams -> its best continuations: parent, token, score
 *   icarus_fork_sequences     parents -> tables and lengths of the children, blocks that nobody holds any more back to the free list
 *   icarus_copy_blocks        the blocks that two children may not share, in the pools of all layers
 *   icarus_extend_sequences, the layers' projections, icarus_rope_append   (icarus_blocks.h); new_lens is 0 for children that are empty: they would begin a sequence of their own, with
 *                             blocks in shared columns, which no fork frees; and it may be 0 for beams that are done
 *   icarus_attn_prefix        attention of single-token rows; the blocks that a group shares are read once for all of its rows
 *
 * As in those headers an icarus_status is returned and icarus_last_error() explains it, the caller owns all device memory and all work goes to the
 * caller's stream (of the current device).  Nothing is kept from one call for the next, so calls that do not touch the same memory may overlap; a
 * workspace belongs to one call at a time.  What the device finds out of range is not followed, as each call says.
 * Pointers: logits, pools, q, out and workspaces 16-byte aligned; integer and float arrays aligned to their element.
 *
 * A call takes up to 65535 sequences and groups, 64 sequences in a group that is chosen from or forked, 2^29 rows, 2^30 queries of a kv-head, tables of
 * 2^22 blocks (to fork: 2^17 parts of 128 columns over all groups), vocabularies of 2^24 tokens, 2^29 free ids and 2^20 copies; icarus_attn_prefix about
 * (rows * query heads / 8 + sequences and groups times kv-heads) * (max_blocks / 1024 + 3) < 2^24, and fewer than 2^30 parts of rows in its workspace (500 GB).  More is
 * ICARUS_ERR_UNSUPPORTED, and a workspace for more has size 0.
 */
#ifndef ICARUS_BRANCHES_H
#define ICARUS_BRANCHES_H

#include "icarus_blocks.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Beams g * width .. g * width + width - 1 form group g.  A beam continues with token t at the score
 *     scores[beam] + x[t] - log(sum over u of exp(x[u])),   x its row of logits,
 * and the group's best `width` continuations, best first, are its next beams: equal scores go to the lowest beam, then the larger logit, then the lowest token.  A beam that is done has one
 * continuation: itself, with token eos and its score as it is.  The sums are formed in float64, and the scores compared in it.
 * A beam takes the logits of its last row, row_start[beam + 1] - 1, as icarus_stack_decode's seq_next does; one that is done takes none and needs no row.  No continuations: a beam with a score
 * that is not finite, one that is not done and has no rows or a row outside 0 .. R - 1; tokens with logits of minus infinity, which NaN counts as.  Plus infinity counts as the largest finite float.
 *   logits        device [R, ld], elements of logits_dtype (ICARUS_F32 as icarus_stack_decode gives them, or ICARUS_BF16); ld >= vocab elements between rows
 *   row_start     device int32 [groups * width + 1], or null: beam i has row i
 *   scores        device float [groups * width]
 *   done          device int32 [groups * width], not 0: the beam is done; or null
 *   eos           the end token, 0 .. vocab - 1; -1: none (then done must be null)
 *   parents       device int32 [groups * width]: number of the parent within the group; -1: there are fewer continuations
 *   tokens, scores_out, done_out  device int32, float, int32 [groups * width]: token (-1), score (minus infinity), 1 where the beam is done now (0); in the place of no continuation
 *                 what is in brackets.  done_out may be null; none of the outputs shares memory with an input
 *   workspace     at least icarus_beam_workspace_bytes(ctx, groups, width, vocab) */
size_t icarus_beam_workspace_bytes(const icarus_ctx *ctx, int32_t groups, int32_t width, int32_t vocab);
icarus_status icarus_beam_select(icarus_ctx *ctx, const void *logits, int32_t logits_dtype, int32_t vocab, int64_t ld, int32_t R, int32_t groups, int32_t width,
                                 const int32_t *row_start, const float *scores, const int32_t *done, int32_t eos, int32_t *parents, int32_t *tokens,
                                 float *scores_out, int32_t *done_out, void *workspace, size_t workspace_bytes, void *stream);

/* Sequence i of a group becomes a child of the group's sequence parents[i]: it takes that one's length and table.  A parent outside 0 .. width - 1 leaves it empty (length 0).
 * Whole blocks are shared.  A block that is partly filled goes to its parent's first child; every further child gets a block from the free list and an entry in the list of
 * copies.  (Among the group's shared columns every child gets its own.)  So outside the shared columns two sequences that have children may not name the same partly filled block: each would hand
 * it to its first child, and both children would write to it.  Beams that begin from one context in one live sequence do not, nor do children of earlier forks.  Samples of a prompt that
 * ends inside a block, tables alike and each its own parent, do: for their first fork shared counts that block's column too, so that every child gets a copy and the block stays the prompt's; from the
 * second one on it counts the prompt's whole blocks alone, since in a shared column every fork copies again and frees nothing.
 * A block that the old tables name in a column from shared[g] on and below the old length, and that no child's table names in that column, goes back to the free list.
 * Blocks of the columns before shared[g], the common prefix, belong to others and stay theirs.  Sequences may share blocks only within their group and in the same column.
 * The free list is that of icarus_extend_sequences: entries free_ids[*free_used ..] are free.  Freed ids are entered before them, in the order of group, column, sequence (those for which the list has
 * no room in front are left out), and then fresh ones are taken from the first free entry on, in the order of the sequences.  A child for which none is left is refused: it is empty, its length 0.
 * Ids outside the pool are not freed; a fresh one is entered as -1, and copies are listed only between blocks of the pool.
 *   parents, kv_lens      device int32 [groups * width] (a length below 0 counts as 0, beyond the table as the table's)
 *   block_tables          device int32 [groups * width, max_blocks]
 *   shared                device int32 [groups] or null (0)
 *   free_ids, free_used   device int32 [n_free], in and out, and [1] (taken as 0 or n_free where it is below or above)
 *   new_lens, new_tables  device int32 [groups * width], [groups * width, max_blocks]: entries behind a child's length are not written; no memory of the inputs
 *   copy_src, copy_dst    device int32 [groups * width]: blocks for icarus_copy_blocks, -1 where the child needs no copy
 *   counts                device int32 [3]: entries of free_ids that are taken now (the next free_used); children refused; blocks freed.  Not free_used itself
 *   workspace             at least icarus_fork_workspace_bytes(ctx, groups, width, max_blocks) */
size_t icarus_fork_workspace_bytes(const icarus_ctx *ctx, int32_t groups, int32_t width, int32_t max_blocks);
icarus_status icarus_fork_sequences(icarus_ctx *ctx, int32_t groups, int32_t width, const int32_t *parents, const int32_t *kv_lens, const int32_t *block_tables,
                                    int32_t max_blocks, const int32_t *shared, int32_t *free_ids, int32_t n_free, const int32_t *free_used,
                                    int32_t *new_lens, int32_t *new_tables, int32_t *copy_src, int32_t *copy_dst, int32_t *counts, void *workspace,
                                    size_t workspace_bytes, void *stream);

/* Block src[i] is copied to block dst[i], in each of the arrays, for every i where both are in 0 .. num_blocks - 1 and differ.  A block that is copied to may be named once in dst and not in
 * src; otherwise its bytes are any of those that would be written or read.
 *   arrays        host [n_arrays]: device arrays of num_blocks blocks each -- pools of the layers, codes and scales of icarus_key_bounds --, 4-byte aligned
 *   block_bytes   host [n_arrays]: bytes of a block, a multiple of 4, at most 2^30
 *   src, dst      device int32 [n] */
icarus_status icarus_copy_blocks(icarus_ctx *ctx, void *const *arrays /*host*/, const int64_t *block_bytes /*host*/, int32_t n_arrays, const int32_t *src,
                                 const int32_t *dst, int32_t n, void *stream);

/* out[r, h] = softmax(q[r, h] K^T / sqrt(D)) V over positions 0 .. kv_lens[s] - 1 of sequence s, for the rows row_start[s] .. row_start[s + 1] - 1 of each sequence, one token per row, as
 * icarus_attn_shared_kv.  Sequences group_start[g] .. group_start[g + 1] - 1 form group g; the first prefix_lens[g] / block_size columns (rounded down) of
 * their tables name the same blocks, which are read once for all rows of the group (short tables may be read by every sequence).  Results go by the tables alone where that holds; what is shared, the lengths and the sizes of the arrays say
 * how sums are split, so calls that differ in them agree up to rounding.
 * Positions whose block lies outside the pool and positions beyond the table are left out.  A row with nothing to attend to, or only scores of minus infinity, becomes zeros; a NaN or a score of
 * plus infinity makes NaN.  Rows of no sequence, and of sequences in no group, keep what out holds.  Shared columns count up to the shortest sequence of the group that is not empty.
 *   q             device [R, Hq, D], normed and rotated
 *   kv_lens       device int32 [S], the current token included (negative: 0)
 *   row_start     device int32 [S + 1], not decreasing, within 0 .. R (rows that lie outside their group's have no part in what it shares)
 *   group_start   device int32 [G + 1], not decreasing, within 0 .. S
 *   prefix_lens   device int32 [G] (negative: 0)
 *   out           device [R, Hq, D], no memory of q
 *   workspace     at least icarus_attn_prefix_workspace_bytes(ctx, S, G, R, max_blocks) */
size_t icarus_attn_prefix_workspace_bytes(const icarus_ctx *ctx, int32_t S, int32_t G, int32_t R, int32_t max_blocks);
icarus_status icarus_attn_prefix(icarus_ctx *ctx, const void *q, const void *kv_pool, const int32_t *block_tables, int32_t max_blocks, int32_t S,
                                 const int32_t *kv_lens, int32_t R, const int32_t *row_start, int32_t G, const int32_t *group_start,
                                 const int32_t *prefix_lens, void *out, void *workspace, size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* ICARUS_BRANCHES_H */
