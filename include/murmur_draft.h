/*
 * libmurmur -- requests into a paged pool, rotary positions, and trees of drafted
 * tokens.  The conventions are murmur.h's.
 *
 * Prompts of new requests:
 *   murmur_paged_reserve   -- blocks and a slot map for every new token;
 *   murmur_rope_append     -- per layer: q and k rotated, K and V into their slots.
 * One round of speculative decoding (a draft proposes a tree of tokens for every
 * sequence, whose root is the current token; the decoder looks at all of them in one
 * pass and keeps the longest path that it agrees with):
 *   murmur_paged_reserve   -- room for the longest path;
 *   murmur_rope_append     -- per layer: the nodes' q and k, rotated by the depth of
 *                             each, K and V into the tree's own buffers;
 *   murmur_decode_attn_tree -- per layer: every node over the retained cache, its
 *                             ancestors and itself;
 *   murmur_tree_accept     -- the accepted path, its K and V into the cache.
 * Rejected nodes leave no trace in the cache, and the windows of the policy are those
 * that single steps would have had.
 */
#ifndef MURMUR_DRAFT_H
#define MURMUR_DRAFT_H

#include "murmur.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Blocks and slot maps for new tokens, from the requests' lengths, on the device.
 * Sequence b has positions 0 .. len[b]-1 and gets new[b] more.  Every block of its row
 * of the table that these lie in and that has none (entry < 0) is popped from the free
 * stack: sequences in order, the columns of each ascending.  A sequence is served
 * whole or not at all, and one that the pool is too small for is refused together with
 * every later one that needs a block; those that need none are served.
 *   len_dev, new_dev: device int32 [B], >= 0;
 *   block_table_dev:  device int32 [B][max_blocks], updated (see murmur_paged_step);
 *   ref_dev:          device int32 [n_blocks], nullable: the counts of a pool with
 *                     shared blocks (murmur_shared.h); a block that is taken gets 1, and
 *                     a sequence whose new tokens lie in a block that others name too is
 *                     refused (MURMUR_DEVERR_BLOCK; murmur_paged_step_shared copies it);
 *   free_stack_dev, free_top_dev, capacity: as murmur_paged_step, capacity >= n_blocks;
 *   per_seq:          where sequence b's tokens stand in the maps: 0: packed, behind
 *                     those of the sequences before it (refused ones too); else from
 *                     b * per_seq on, and new[b] <= per_seq;
 *   n_tokens:         entries of each map, >= B * per_seq; entries that no token has
 *                     are -1;
 *   start_dev:        device int32 [B + 1], output: the first token of each sequence
 *                     and the end of the last (at most 2^31 - 1);
 *   got_dev:          device int32 [B], output: new[b], or -1 for a refused sequence;
 *   slot_dev:         device int32 [n_tokens], output: the token's pool row, -1 for
 *                     those of a refused sequence;
 *   pos_dev, seq_dev: device int32 [n_tokens], nullable outputs: the token's position
 *                     in its sequence, and its sequence;
 *   ws_dev, ws_bytes: see murmur_paged_reserve_workspace; 256-byte aligned, not
 *                     initialised, not used by two calls at the same time.
 * Errors: MURMUR_EINVAL, MURMUR_ENOSPACE (workspace), MURMUR_EHIP.  Device errors, all
 * of which refuse the sequence: MURMUR_DEVERR_POOL (too few free blocks, or one on the
 * stack that is not the pool's: then the entry stays -1), MURMUR_DEVERR_BLOCK (past
 * max_blocks, an entry of n_blocks or more, a pool row beyond 2^31 - 1, a shared block),
 * MURMUR_DEVERR_COUNT (a negative length or number), MURMUR_DEVERR_OVERFLOW (its tokens
 * end behind per_seq or n_tokens). */
int murmur_paged_reserve_workspace(int32_t B, size_t *bytes);
int murmur_paged_reserve(const int32_t *len_dev, const int32_t *new_dev, int32_t B, int32_t *block_table_dev,
                         int32_t max_blocks, int32_t block_size, int32_t *ref_dev, int32_t n_blocks,
                         int32_t *free_stack_dev, int32_t *free_top_dev, int32_t capacity, int32_t per_seq,
                         int32_t n_tokens, int32_t *start_dev, int32_t *got_dev, int32_t *slot_dev, int32_t *pos_dev,
                         int32_t *seq_dev, void *ws_dev, size_t ws_bytes, murmur_stream_t stream);

/* Rotary positions.  Pair i of a head (i < rot_dim / 2) turns by f_i whole turns per
 * position; f_i = base^(-2 i / rot_dim) / (2 pi), scaled for contexts longer than the
 * trained one by `factor`: */
enum {
    MURMUR_ROPE_PLAIN = 0,  /* f_i */
    MURMUR_ROPE_LINEAR = 1, /* f_i / factor (positions interpolated) */
    MURMUR_ROPE_BASE = 2,   /* base * factor^(rot_dim / (rot_dim - 2)) for base: the slowest pair takes the factor */
    MURMUR_ROPE_BANDS = 3,  /* by the turns n_i = original_len * f_i within the trained context: f_i / factor up to
                             * slow_turns, f_i from fast_turns on, linear in n_i between */
    MURMUR_ROPE_YARN = 4,   /* the same, and a gain of 1 + 0.1 ln(factor) on the rotated part of q and of k */
};

/* Host only: the table of a rotation.  freq[i] is f_i as a fraction of 2^64, within two
 * steps of it, and position p's turn is the fraction p * freq[i] mod 2^64, an exact
 * integer product: at position 2^31 it is within 2^-32 of a turn.  (The bands are linear
 * in the turns n_i, as Peng et al. give them; a ramp over the pair's index is a table of
 * the caller's own.)
 *   rot_dim: even, in [2, 128]; base > 1; factor >= 1 (ignored by MURMUR_ROPE_PLAIN);
 *   original_len, slow_turns, fast_turns: of MURMUR_ROPE_BANDS and MURMUR_ROPE_YARN,
 *            0 < original_len, 0 <= slow_turns < fast_turns (ignored by the others);
 *   freq:    host [rot_dim / 2]; gain: host, 1 but for MURMUR_ROPE_YARN.
 * Errors: MURMUR_EINVAL. */
int murmur_rope_freqs_host(int32_t rot_dim, double base, int32_t kind, double factor, double original_len,
                           double slow_turns, double fast_turns, uint64_t *freq, float *gain);

/* How heads are rotated.
 *   rot_dim:     the leading elements of a head that are (even, in [0, 128]); the rest
 *                is passed on;
 *   interleaved: 0: element i pairs with i + rot_dim / 2; 1: 2 i with 2 i + 1;
 *   gain:        finite; the rotated elements are multiplied by it;
 *   freq:        device uint64 [rot_dim / 2], 8-byte aligned (murmur_rope_freqs_host). */
typedef struct murmur_rope {
    int32_t rot_dim;
    int32_t interleaved;
    float gain;
    const uint64_t *freq;
} murmur_rope;

/* A layer's (or several layers') projections: head h, element e of token t of layer l
 * at q + l*q_layer + t*q_token + h*128 + e, and k and v likewise with kv_layer and
 * kv_token (elements; q, k and v may be parts of one row).  dtype: MURMUR_DTYPE_BF16 or
 * MURMUR_DTYPE_F32.  Pointers are aligned to an element; with 16-byte aligned ones and
 * strides of multiples of 16 bytes loads are wide. */
typedef struct murmur_qkv {
    const void *q;
    const void *k;
    const void *v;
    int32_t dtype;
    int64_t q_layer;
    int64_t q_token;
    int64_t kv_layer;
    int64_t kv_token;
} murmur_qkv;

/* Rotates q and k of every token to its position, in every layer, and writes K and V
 * into the cache rows of a slot map, all in one launch.  The turns are the table's, cut to
 * 2^-32 of one (see murmur_rope_freqs_host), sines and products fp32; bf16 results are
 * rounded once.
 *   pos_dev:   device int32 [n_tokens]: rotary positions; a token of a negative one is
 *              not there: nothing is written for it;
 *   slot_dev:  device int32 [n_tokens]: the row of K and V, as a position of sequence
 *              seq[t] of the cache; -1: K and V are not kept.  No two tokens have the
 *              same row;
 *   seq_dev:   device int32 [n_tokens], nullable (0 for all of them): only for caches
 *              with kv->stride_b; in [0, n_seqs);
 *   n_seqs:    sequences of the cache;
 *   q_out_dev: bf16 [n_layers][n_tokens][Hq][D], contiguous, 16-byte aligned (with a
 *              contiguous bf16 q it may be q itself);
 *   kv:        the cache (see murmur_kv), written: n_layers layers and max_len rows a
 *              sequence;
 *   D:         head_dim, must be 128.
 * Errors: MURMUR_EINVAL, MURMUR_EUNSUPPORTED (head_dim), MURMUR_EHIP.  Device error
 * MURMUR_DEVERR_POSITION for a slot of max_len or more, or a sequence out of range (K
 * and V are not kept; q is rotated). */
int murmur_rope_append(const murmur_rope *rope, const murmur_qkv *in, const int32_t *pos_dev, const int32_t *slot_dev,
                       const int32_t *seq_dev, int32_t n_seqs, int32_t n_tokens, int32_t Hq, int32_t Hkv, int32_t D,
                       void *q_out_dev, const murmur_kv *kv, murmur_stream_t stream);

/* Trees of drafted tokens.  A tree of up to 64 nodes a sequence is an array of parents:
 * parent[0] = -1 (the root, the current token), parent[i] in [0, i) for a node that
 * follows node parent[i], -2 for a node that is not there.  Node i of depth d (the root
 * 0) is output token out_len + d of its sequence, where out_len counts the root
 * (murmur_seg).  K and V of the nodes are not in the cache: they have buffers of their
 * own, bf16 [n_layers][B][n_nodes][Hkv][128], contiguous, 16-byte aligned.
 *   parent_dev: device int32 [parent_per_seq ? B : 1][n_nodes].
 * Another tree is invalid (MURMUR_DEVERR_TREE for its sequence). */

/* Workspace bytes of murmur_decode_attn_tree (may be 0): 256-byte aligned, not
 * initialised; a larger one is fine.  The sizes grow with n_layers, B, n_nodes and
 * max_keep, up to 98 MiB, so the workspace of the largest call serves every smaller one
 * of the same heads.  Calls that run at the same time need workspaces of their own. */
int murmur_decode_attn_tree_workspace(int32_t n_layers, int32_t B, int32_t Hq, int32_t Hkv, int32_t n_nodes,
                                      int32_t max_keep, size_t *bytes);

/* Attention (Equation 1) of every node of every sequence's tree, in every layer, as if
 * its path had been decoded token by token: over what the policy retains at step
 * out_len + depth (Section 3.2: Algorithms 1-2 and Equation 2) of the prompts, the
 * speech and the outputs, where the outputs are the 0 .. out_len-2 of the cache and then
 * the node's ancestors and itself.
 *   seg_dev, pol_dev, pol_per_seq: as murmur_decode_step; out_len counts the root.  A
 *               sequence with a murmur_seg of zeros is not there: its outputs stay as
 *               they were, and so do those of nodes that are not there;
 *   n_nodes:    T, in [1, 64];
 *   q_dev:      bf16 [n_layers][B][T][Hq][D], contiguous, 16-byte aligned;
 *   kv:         the cache; every position before the root's that a node retains must be
 *               there;
 *   k_tree_dev, v_tree_dev: see above;
 *   block_table_dev, max_blocks, block_size: of a paged cache (as
 *               murmur_evict_compact_paged; kv->stride_b is 0 then); NULL, 0, 0 for
 *               sequence-ordered ones;
 *   max_keep:   the most that a tree's nodes retain together, nodes counted (the
 *               schedule is made for it; longer lists are computed too);
 *   out_dev:    [n_layers][B][T][Hq][D] of out_dtype, 16-byte aligned;
 *   lse_dev:    nullable fp32 [n_layers][B][T][Hq], natural log;
 *   ws_dev, ws_bytes: see murmur_decode_attn_tree_workspace;
 *   every other argument as murmur_decode_step.
 * Accumulation is fp32 throughout.  Errors as murmur_decode_attn.  Device errors, each
 * with NaN outputs for the sequence's nodes: MURMUR_DEVERR_POLICY (also for a layout
 * that ends within 64 positions of 2^31, or a list within 96), MURMUR_DEVERR_TREE,
 * MURMUR_DEVERR_POSITION (a retained position outside [0, max_len)),
 * MURMUR_DEVERR_BLOCK (one without a block, or past max_blocks). */
int murmur_decode_attn_tree(const murmur_seg *seg_dev, const murmur_policy *pol_dev, int32_t pol_per_seq,
                            const int32_t *parent_dev, int32_t parent_per_seq, int32_t n_nodes, const void *q_dev,
                            const murmur_kv *kv, const void *k_tree_dev, const void *v_tree_dev,
                            const int32_t *block_table_dev, int32_t max_blocks, int32_t block_size, int32_t max_keep,
                            int32_t B, int32_t Hq, int32_t Hkv, int32_t D, float scale, void *out_dev,
                            int32_t out_dtype, float *lse_dev, void *ws_dev, size_t ws_bytes, murmur_stream_t stream);

/* The path that the decoder agrees with: the root, and from an accepted node on the
 * child whose token is the one that the decoder gives there (of several, the one of the
 * lowest index).  Its K and V go into the cache, in every layer; the sequence is then
 * count tokens longer, and last its next root.
 *   token_dev: device int32 [B][n_nodes]: the nodes' tokens; a sequence whose root's is
 *              negative is not there (count 0, path and last -1), and other nodes with
 *              negative ones are never accepted;
 *   next_dev:  device int32 [B][n_nodes]: the token that the decoder gives after each;
 *   slot_dev:  device int32 [B][n_nodes]: the cache rows of the path's first, second,
 *              ... node, as positions of sequence b of the cache, all different; -1: not
 *              kept, but counted (the root of a sequence that murmur_paged_reserve has
 *              refused is therefore given a negative token: it sits the round out);
 *   kv:        the cache, written (n_layers of it), as murmur_rope_append;
 *   path_dev:  device int32 [B][n_nodes], output: the path's nodes, then -1;
 *   count_dev, last_dev: device int32 [B], outputs: nodes of the path, and the token
 *              that the decoder gives after the last of them.
 * Errors: MURMUR_EINVAL, MURMUR_EHIP.  Device errors: MURMUR_DEVERR_TREE (the sequence
 * is treated as not there), MURMUR_DEVERR_POSITION (a slot of max_len or more is not
 * written). */
int murmur_tree_accept(const int32_t *parent_dev, int32_t parent_per_seq, int32_t n_nodes, const int32_t *token_dev,
                       const int32_t *next_dev, const int32_t *slot_dev, int32_t B, const void *k_tree_dev,
                       const void *v_tree_dev, const murmur_kv *kv, int32_t Hkv, int32_t *path_dev,
                       int32_t *count_dev, int32_t *last_dev, murmur_stream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* MURMUR_DRAFT_H */
