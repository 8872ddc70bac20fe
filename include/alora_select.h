/*
 * alora_select.h -- long contexts read in part: bounds of every cache block's keys in 8 bits, the blocks whose bounds promise a query
 * the largest scores, and attention over those blocks alone (C ABI of libalora_qkv.so, gfx950).  A step of a layer calls, behind the projection,
 * alora_block_bounds for the rows it wrote, alora_block_select and alora_selected_attention.
 *
 * Conventions and limits are those of alora_qkv.h and alora_attention.h.  All pointers are DEVICE pointers.  block_tables may be NULL where n_seqs or
 * max_blocks is 0.
 */
#ifndef ALORA_SELECT_H
#define ALORA_SELECT_H

#include <stddef.h>
#include <stdint.h>
#include "alora_qkv.h"
#include "alora_attention.h"

#ifdef __cplusplus
extern "C" {
#endif

/* dims of alora_block_bounds */
typedef struct alora_bounds_dims {
    int32_t dtype;
    int32_t n_rows;       /* rows of slot_mapping                                                */
    int32_t n_kv_heads, head_dim, block_size;
    int64_t n_slots;
} alora_bounds_dims;

/*
 * Bounds of the blocks that the rows of slot_mapping lie in.  Rows of one block follow each other; the last of them, at offset o of its
 * block, stands for offsets 0 .. o.  With lo_d, hi_d the smallest and largest component d of these rows' keys, of one head, and
 * a = max_d max(|lo_d|, |hi_d|):
 *     bounds[block, head, 0, d] = ceil(hi_d f),  bounds[block, head, 1, d] = floor(lo_d f)     in [-127, 127],  f = 127 / a in fp32
 *     scales[block, head] = a / 127
 * so that scale * bounds encloses the keys, up to the three roundings to fp32 (2^-22 of a component).  a below 2^-100: bounds 0, which enclose the keys up to a only.  A component that is
 * not finite: bounds 0, scale infinity.
 *   slot_mapping  int64 [n_rows]; rows outside [0, n_slots) are passed over, also between rows of one block
 *   bounds        int8 [n_slots / block_size, n_kv_heads, 2, head_dim], 16-byte aligned; scales fp32 [n_slots / block_size, n_kv_heads]
 * Blocks copied or moved (alora_cache.h) get their bounds from a call with the slot of their last row.
 * n_rows = 0 is a successful no-op.  head_dim in {64, 128}; n_slots <= 2^31 - 1; n_kv_heads <= 2^16; n_rows <= 2^27.
 */
int alora_block_bounds(const void *k_cache, const int64_t *slot_mapping, int8_t *bounds, float *scales, const alora_bounds_dims *dims, void *hip_stream);

/*
 * For every row and K/V head the blocks of its context to be read: the first n_first, the last n_recent, and of the others those with the largest
 *     score(b) = scales[b] * sum_d ( up_d * bounds[b, 0, d] + down_d * bounds[b, 1, d] )
 * up_d and down_d being the sums over the head's query heads of max(q_d, 0) and min(q_d, 0) (in 64 bits, rounded to fp32), scaled by 127 / max_d max(up_d, -down_d) in fp32 and rounded to
 * whole numbers (all 0 where that maximum is below 2^-100 or not finite; a component that is no number counts as 0): with bounds of a block that is a bound of the sum of its keys' scores, up to the rounding of q and of the bounds.  The sum is exact; equal scores go to the
 * lower block.  Scores are clamped to the finite numbers; a block with infinite scale has the largest finite score, one whose table entry is outside the cache
 * a score of minus infinity.
 *   selected  int32 [n_tokens, n_kv_heads, budget]: blocks of the row's table in ascending order, behind the last one -1; all blocks of a context of at
 *             most budget.  A row whose sequence id or position is out of range gets -1 throughout.
 * n_first >= 0, n_recent >= 1, n_first + n_recent <= budget, budget <= 2^20 (ALORA_EINVAL otherwise).  Limits as in alora_attention.h, and
 * n_tokens * n_kv_heads < 2^22, n_kv_heads <= 2^16, max_blocks <= 2^28 (ALORA_ESHAPE).
 *   workspace device, 16-byte aligned, >= alora_block_select_workspace_bytes() bytes (0: may be NULL), contents on entry irrelevant; calls that share
 *             it must be stream-ordered.  ALORA_EWORKSPACE otherwise.  What that function gives is enough for every call of fewer rows too (the other dims alike).
 *             Tables of more than 4352 columns take 4 bytes for every row, K/V head and column: rows do not depend on each other, so a large chunk can be several calls.
 */
int alora_block_select_workspace_bytes(const alora_attn_dims *dims, size_t *out_bytes);
int alora_block_select(const void *q, const int8_t *bounds, const float *scales, const int32_t *block_tables, const int32_t *token_seq_ids,
                       const int32_t *token_positions, int32_t *selected, int32_t budget, int32_t n_first, int32_t n_recent, const alora_attn_dims *dims,
                       void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * alora_paged_attention over the positions 0 .. p of the blocks in `selected` alone (int32 [n_tokens, n_kv_heads, budget], any list of blocks
 * of the row's table in ascending order).  An entry outside the row's context, or not above the entry before it, is left out; a row with
 * nothing left gets zeros.  Limits as above, 1 <= budget <= 2^20 (ALORA_EINVAL), budget * block_size < 2^30 (ALORA_ESHAPE).
 * In bf16 a weight of the softmax is two bf16 numbers in the weighted sum of V, as in alora_tree.h; an infinite value that is read is one in the result.
 *   workspace as above, alora_selected_attention_workspace_bytes() (for one budget): with few rows the lists are cut into parts, combined in a fixed order.
 */
int alora_selected_attention_workspace_bytes(const alora_attn_dims *dims, int32_t budget, size_t *out_bytes);
int alora_selected_attention(const void *q, const void *k_cache, const void *v_cache, const int32_t *block_tables, const int32_t *token_seq_ids,
                             const int32_t *token_positions, const int32_t *selected, int32_t budget, void *out, const alora_attn_dims *dims,
                             void *workspace, size_t workspace_bytes, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* ALORA_SELECT_H */
