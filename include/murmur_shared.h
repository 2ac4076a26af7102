/*
 * libmurmur -- decoding several hypotheses of one chunk (beams, samples, drafted
 * tokens): block tables whose rows share blocks, and decode-step attention that
 * reads what a group of sequences shares once.  The conventions are murmur.h's.
 *
 * One token of a beam decode:
 *   murmur_paged_fork          -- every sequence continues its parent;
 *   murmur_paged_step_shared   -- free, take or copy a block, append K and V;
 *   murmur_evict_compact_paged -- the retained lists, as pool rows;
 *   murmur_shared_plan         -- what the groups share, and the work it makes;
 *   murmur_decode_attn_shared  -- per layer (or for all of them);
 * and now and then murmur_paged_compact.
 *
 * A sequence that is not there (a hypothesis that ended, a row of a padded batch) has
 * a murmur_seg of zeros.  murmur_paged_step_shared leaves its row as it is, gives it
 * no block and writes nothing for it; murmur_evict_compact_paged gives it the count
 * -1; murmur_shared_plan takes a list of the count -1 (or a range table whose lengths
 * add up to -1) for one that is not there, wherever it stands in its group: the others
 * share as if it were not in it, and its outputs stay as they were.  None of this sets
 * a bit of the device error word.
 */
#ifndef MURMUR_SHARED_H
#define MURMUR_SHARED_H

#include "murmur.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Shared pages.  The hypotheses of a decode (beams, samples) that go back to one
 * prompt have block tables that name the same blocks up to where they parted.
 * ref_dev holds, per physical block, how many table entries name it (and any
 * reference that the caller adds for itself); a block is free when that is 0, and
 * its number is then on the free stack.  The calls below keep tables, counts and
 * stack together; a pool is theirs alone (murmur_paged_step knows no counts).
 * Shared arguments:
 *   B:               rows of the table (sequences), at most 65535;
 *   block_table_dev: device int32 [B][max_blocks], physical block numbers below
 *                    n_blocks, -1 where there is none; B * max_blocks <= 2^30;
 *   ref_dev:         device int32 [n_blocks];
 *   free_stack_dev:  device int32 [capacity], free blocks in [0, *free_top_dev),
 *                    capacity >= n_blocks;
 *   free_top_dev:    device int32.
 * Rows that name one block name it in the same column, as the forks leave them.
 * Every result is the same on every run: counts are integers, and what one call
 * pushes and pops has a stated order.  A table entry of n_blocks or more gives
 * MURMUR_DEVERR_BLOCK and is otherwise passed over; pushes beyond n_blocks (a stack
 * that does not agree with the counts) give MURMUR_DEVERR_POOL and are dropped. */

/* Workspace bytes of murmur_paged_fork and murmur_paged_compact (one workspace
 * serves both, for one B, max_blocks and n_blocks): 256-byte aligned, zero-filled
 * once before its first use, and not used by two calls at the same time. */
int murmur_paged_workspace(int32_t B, int32_t max_blocks, int32_t n_blocks, size_t *bytes);

/* Forks, reorders and ends sequences: row b of the table becomes a copy of what
 * row parent_dev[b] was before the call (itself: unchanged; -1: empty, every entry
 * -1).  Rows copy names, not blocks; the first write into a block that several
 * rows name copies it (murmur_paged_step_shared).  Blocks that no row names any
 * more go onto the free stack, in the order of the first entry (by row, then
 * column) that named them.  What the new row's sequence is (its murmur_seg, zeros if
 * it has ended; its tokens) is the caller's.
 *   parent_dev: device int32 [B];
 *   ws_dev, ws_bytes: see murmur_paged_workspace.
 * Errors: MURMUR_EINVAL, MURMUR_ENOSPACE (workspace), MURMUR_EHIP; device error
 * MURMUR_DEVERR_PARENT for a parent outside [-1, B) (the row stays as it is). */
int murmur_paged_fork(const int32_t *parent_dev, int32_t B, int32_t *block_table_dev, int32_t max_blocks,
                      int32_t *ref_dev, int32_t n_blocks, int32_t *free_stack_dev, int32_t *free_top_dev,
                      int32_t capacity, void *ws_dev, size_t ws_bytes, murmur_stream_t stream);

/* murmur_paged_step on shared pages: one decode step of the block manager, in
 * three parts and two launches (one without a pool):
 *   1. every entry that lies wholly in positions that no step from out_len on
 *      retains gives its block up (entry -1, count - 1); blocks that nobody names
 *      then are pushed, in the order of the first sequence that gave them up, its
 *      columns ascending;
 *   2. a sequence whose current token's logical block has no block takes one, and
 *      one whose block others name too takes a copy: the rows before the current
 *      token are copied from the old block, whose count drops by one.  Of several
 *      such sequences the one furthest ahead (the last one of equals) keeps the
 *      block, if nobody else names it.  Blocks are popped in sequence order;
 *   3. the current token's K and V are written into its row.
 *   copied_dev: device int32 [B], output: the block that a sequence's current block
 *               was copied from, -1 if it was not copied (nor is a token past the
 *               table, which has no row to be written to), -2 if nothing is written
 *               for the sequence (not there, an invalid layout or policy, a current
 *               block of n_blocks or more, or no free block);
 *   every other argument as murmur_paged_step; with a pool, pool->max_len >=
 *   n_blocks * block_size.  Without one the copies that copied_dev names are the
 *   caller's to make.
 * Errors and device errors as murmur_paged_step; a sequence that finds the stack
 * empty loses the entry of its current block (-1), so the attention reports it.
 * One workgroup does parts 1 and 2, and the sequences that share their current block
 * cost it a comparison with every other one: 13 us for 96 sequences of which 84 copy,
 * 88 for 1024 (896), 1.2 ms for 4096 (3584). */
int murmur_paged_step_shared(const murmur_seg *seg_dev, const murmur_policy *pol_dev, int32_t pol_per_seq, int32_t B,
                             int32_t *block_table_dev, int32_t max_blocks, int32_t block_size, int32_t *ref_dev,
                             int32_t n_blocks, int32_t *free_stack_dev, int32_t *free_top_dev, int32_t capacity,
                             int32_t full_scan, int32_t *copied_dev, const murmur_kv *pool, int32_t Hkv,
                             const void *k_new_dev, const void *v_new_dev, murmur_stream_t stream);

/* Compacts the pool: the n blocks in use (count > 0) end up as blocks 0 .. n-1.
 * Those below n stay; the others move, in ascending order, into the free ones
 * below n, in ascending order.  Their K and V are copied in every layer, table
 * entries and counts renamed, and the free stack becomes n_blocks-1 .. n (n on
 * top).
 *   map_dev: device int32 [n_blocks], output: every block's new number, -1 for one
 *            that was free (for block numbers that the caller keeps elsewhere);
 *   pool:    nullable, as murmur_paged_step_shared (without it the caller copies
 *            blocks by map_dev); Hkv: KV heads (with a pool);
 *   ws_dev, ws_bytes: see murmur_paged_workspace.
 * Errors: MURMUR_EINVAL, MURMUR_ENOSPACE (workspace), MURMUR_EHIP; device error
 * MURMUR_DEVERR_BLOCK for an entry that names a free block (it becomes -1). */
int murmur_paged_compact(int32_t B, int32_t *block_table_dev, int32_t max_blocks, int32_t block_size,
                         int32_t *ref_dev, int32_t n_blocks, int32_t *free_stack_dev, int32_t *free_top_dev,
                         int32_t capacity, int32_t *map_dev, const murmur_kv *pool, int32_t Hkv, void *ws_dev,
                         size_t ws_bytes, murmur_stream_t stream);

/* Attention over shared prefixes.  Sequences come in groups of neighbours whose
 * retained lists begin alike (hypotheses of one chunk, drafted tokens of one
 * sequence, chunks behind one long prompt).  What a group shares is read once for
 * the query rows of all its sequences, the rest of each list for its own, and the
 * parts are joined by log-sum-exp: the result is murmur_decode_attn's.
 *
 * murmur_decode_attn_shared_workspace gives the bytes of the two buffers that a
 * call of these sizes needs: a plan (16-byte aligned), which murmur_shared_plan
 * writes and murmur_decode_attn_shared reads, and a workspace (256-byte aligned)
 * for the partial sums.  Neither needs to be initialised; a larger buffer is fine.
 * The sizes grow with B, max_keep and n_groups, so the buffers of the largest batch
 * serve every smaller one.  A call leaves its lists whole or cuts them, by these sizes
 * alone (max_keep stands for the lists' lengths, so one close to them is best), and the
 * workspace holds either: for lists of 850, 28/4 heads, 96 sequences in 12 groups 8.3
 * MiB a layer in a call of its own and 95 for 28 layers in one call; for lists of 3657,
 * 1024 sequences in 64 groups and 28 layers in one call 1.1 GiB.
 * At most 4096 sequences (MURMUR_EUNSUPPORTED beyond) and as many groups.
 * Calls that run at the same time need workspaces of their own, and may share a
 * plan. */
int murmur_decode_attn_shared_workspace(int32_t n_layers, int32_t B, int32_t Hq, int32_t Hkv, int32_t max_keep,
                                        int32_t n_groups, size_t *ws_bytes, size_t *plan_bytes);

/* Cuts the work of murmur_decode_attn_shared; once per token, for all its layers.
 *   idx_dev, ranges_dev, count_dev, max_keep: the lists, as murmur_decode_attn
 *               takes them (ranges_dev with precedence, then count_dev is not
 *               read); lists of pool rows have one meaning for all sequences, and
 *               positions of sequence-ordered caches the same content in each;
 *   group_dev:  device int32 [n_groups + 1], ascending from 0 to at most B: group p
 *               holds sequences group[p] .. group[p+1]-1 (it may be empty).
 *               Sequences from group[n_groups] on are left out: their outputs stay
 *               as they were;
 *   shared_dev: device int32 [n_groups]: how many leading list entries the group's
 *               sequences share.  find_shared 1: output, the most that the index
 *               lists allow (ranges_dev NULL; for a group of one its whole list; 0
 *               if none of the group has a valid count, or its first sequence that
 *               is there one below 1; other invalid lists are passed over);
 *               0: input, a promise of the caller, who may share less than that
 *               (the way for sequence-ordered caches, whose lists do not tell);
 *   n_layers, Hq, Hkv: of each murmur_decode_attn_shared call that uses the plan;
 *   plan_dev, plan_bytes: see murmur_decode_attn_shared_workspace.
 * Errors: MURMUR_EINVAL, MURMUR_EUNSUPPORTED, MURMUR_ENOSPACE, MURMUR_EHIP.  Device
 * errors: MURMUR_DEVERR_COUNT for a sequence whose count is neither -1 nor in
 * [1, max_keep], or is below what its group shares, and for all of a group that shares
 * more than the count of its first sequence that is there (NaN outputs);
 * MURMUR_DEVERR_GROUP for groups out of order (every output is NaN). */
int murmur_shared_plan(const int32_t *idx_dev, const int32_t *ranges_dev, const int32_t *count_dev, int32_t max_keep,
                       int32_t B, const int32_t *group_dev, int32_t n_groups, int32_t *shared_dev,
                       int32_t find_shared, int32_t n_layers, int32_t Hq, int32_t Hkv, void *plan_dev,
                       size_t plan_bytes, murmur_stream_t stream);

/* Decode-step attention (Equation 1) of every sequence over its list, as
 * murmur_decode_attn, reading what a group shares once: from the list, and in
 * sequence-ordered caches from the cache, of the group's first sequence that is there.
 *   idx_dev, ranges_dev: the lists the plan was made from, unchanged since;
 *   n_groups:   of the plan;
 *   plan_dev, plan_bytes, ws_dev, ws_bytes: see
 *               murmur_decode_attn_shared_workspace;
 *   every other argument and the outputs as murmur_decode_attn.
 * Accumulation is fp32 throughout.  Errors as murmur_decode_attn; device errors
 * MURMUR_DEVERR_POSITION (NaN for the sequences whose lists hold the position) and
 * MURMUR_DEVERR_GROUP for a plan that was not made for these sizes, or with
 * find_shared 1 where kv->stride_b is not 0 and lists of several sequences begin alike:
 * equal positions of two caches are different rows (every output is NaN). */
int murmur_decode_attn_shared(const void *q_dev, const murmur_kv *kv, const int32_t *idx_dev,
                              const int32_t *ranges_dev, int32_t max_keep, int32_t B, int32_t n_groups, int32_t Hq,
                              int32_t Hkv, int32_t D, float scale, void *out_dev, int32_t out_dtype, float *lse_dev,
                              const void *plan_dev, size_t plan_bytes, void *ws_dev, size_t ws_bytes,
                              murmur_stream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* MURMUR_SHARED_H */
