/*
 * alora_tree.h -- drafted tokens that form a tree: what each of them sees, and attention over the paged cache (C ABI of
 * libalora_qkv.so, gfx950).  A sequence's drafts are rows that follow each other in the batch, a parent in front of its
 * children; draft i of a sequence with `context` tokens in the cache is stored at the context + i-th place of its block table
 * (the slots alora_step_rows gives), and stands for position context + depth.  One step then verifies several continuations at once; the
 * rows of the accepted path are moved together with alora_cache_move_rows, the others given back with alora_step_rows.
 *
 * Conventions are those of alora_qkv.h and alora_attention.h.  All pointers are DEVICE pointers.
 */
#ifndef ALORA_TREE_H
#define ALORA_TREE_H

#include <stddef.h>
#include <stdint.h>
#include "alora_qkv.h"
#include "alora_attention.h"

#ifdef __cplusplus
extern "C" {
#endif

#define ALORA_MAX_TREE_WORDS 4

/*
 * Masks and positions from parents.  Rows row_offsets[s] .. row_offsets[s + 1] - 1 are sequence s's.
 *   tree_parents     [n_tokens] the parent's place in its sequence's tree, in front of the row's own; -1: the context's last token
 *   context_lens     [n_seqs]
 *   tree_mask        uint64 [n_tokens, mask_words]: bit j is set if the sequence's draft j is the row's ancestor or the row itself
 *   token_positions  [n_tokens] context_lens + number of ancestors
 * A row whose parent, or an ancestor's, is not in front of it, and one behind the first 64 * mask_words of its sequence, gets an empty mask and
 * position context_lens; a row of no sequence an empty mask and position 0.
 * mask_words in 1 .. ALORA_MAX_TREE_WORDS; n_seqs <= 2^20 (ALORA_ESHAPE).
 */
int alora_tree_rows(const int32_t *tree_parents, const int32_t *row_offsets, const int32_t *context_lens, uint64_t *tree_mask,
                    int32_t *token_positions, int32_t n_tokens, int32_t n_seqs, int32_t mask_words, void *hip_stream);

/*
 * Attention of the drafts: row t, draft i of sequence s, with context c = context_lens[s] and n = row_offsets[s + 1] - row_offsets[s] drafts,
 *
 *     o[t, h, :] = sum_j softmax_j( scale * <q[t, h, :], K_j[g(h), :]> ) * V_j[g(h), :]      over j < c, and j = c + i' with bit i' of the
 *                                                                                          row's mask set, i' < n
 *
 * K_j, V_j, g(h) and scale as in alora_attention.h; any mask may be given, not only that of a tree.  A row that sees nothing, and a row of no sequence, gets zeros; a place whose
 * table entry is outside the cache is left out of the softmax.
 *   block_tables, context_lens may be NULL where n_seqs is 0, and block_tables where max_blocks is
 *   row_offsets [n_seqs + 1] ascending, tree_mask uint64 [n_tokens, mask_words], 8-byte aligned
 *   workspace   device, 16-byte aligned, >= alora_tree_attention_workspace_bytes() bytes, contents on entry irrelevant; calls that share it must be
 *               stream-ordered.  ALORA_EWORKSPACE otherwise.
 * The contexts are cut into parts of equal length, which a second kernel combines in a fixed order: results do not depend on timing, but a
 * row's low bits depend on the lengths of all sequences of the call.
 * Limits as in alora_attention.h; mask_words in 1 .. ALORA_MAX_TREE_WORDS, n_seqs <= 2^20, max_blocks * block_size <= 2^30, and fewer than 2^24 workgroups: each
 * K/V head takes one for every tile of rows (128 columns in bf16, 8 in fp32 at most, n_q_heads / n_kv_heads to a row) and a few hundred (ALORA_ESHAPE).  bf16 runs on matrix instructions (a
 * weight of the softmax is two bf16 numbers in the weighted sum of V, off by 2^-14 of itself at most; scores, maxima and sums stay fp32).
 */
int alora_tree_attention_workspace_bytes(const alora_attn_dims *dims, int32_t mask_words, size_t *out_bytes);
int alora_tree_attention(const void *q, const void *k_cache, const void *v_cache, const int32_t *block_tables, const int32_t *row_offsets,
                         const int32_t *context_lens, const uint64_t *tree_mask, int32_t mask_words, void *out, const alora_attn_dims *dims,
                         void *workspace, size_t workspace_bytes, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* ALORA_TREE_H */
