/*
 * alora_steps.h -- a step's rows built where the requests' lengths are: block tables, slots and the per-row metadata of
 * alora_qkv_forward and the reader, from lengths on the device (C ABI of libalora_qkv.so, gfx950).  The planner
 * (alora_planner.h) does this on the host, where requests are admitted; a decoding loop whose lengths follow from what the
 * device computed -- how many drafted tokens were accepted, which requests ended -- needs no copy to the host and can be
 * captured into a device graph.
 *
 * Conventions are those of alora_qkv.h.  All pointers are DEVICE pointers.
 */
#ifndef ALORA_STEPS_H
#define ALORA_STEPS_H

#include <stddef.h>
#include <stdint.h>
#include "alora_qkv.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Limits (ALORA_ESHAPE): n_seqs <= 2^20, row_cap and pool_cap <= 2^30, n_slots / block_size <= 2^31 - 1. */
typedef struct alora_step_dims {
    int32_t n_seqs;       /* requests                                                            */
    int32_t max_blocks;   /* columns of block_tables                                             */
    int32_t block_size;
    int32_t row_cap;      /* rows of the four token arrays                                       */
    int32_t pool_cap;     /* entries of pool                                                     */
    int64_t n_slots;      /* rows of the caches                                                  */
} alora_step_dims;

/*
 * Request s has lengths[s] = n tokens in the cache and changes by change[s] = c.
 *   c > 0   it grows: blocks ceil(n / bs) .. ceil((n + c) / bs) - 1 of its table are taken from the pool, and it gets rows for
 *           positions n .. n + c - 1;
 *   c <= 0  it gives its last -c tokens back (rejected drafts; all of them: the request is over): blocks
 *           ceil(n / bs) - 1 down to max(ceil((n + c) / bs), kept_blocks[s]) return to the pool, the last one first.
 * Requests are served in their order.  One whose n or n + c is outside [0, max_blocks * block_size] is refused; of those that grow,
 * one for whose blocks the pool or for whose rows row_cap is too small, and every later one that grows, are refused too.  A refused request stays
 * as it is.  Blocks that return are handed out from the next call on.
 *
 *   lengths, change  [n_seqs]; kept_blocks [n_seqs] or NULL: leading blocks that are someone else's too (a shared prefix)
 *                    and never return; seq_adapters [n_seqs] or NULL (then -1): adapter id of each request
 *   block_tables     [n_seqs, max_blocks], entries of new blocks are written, all others left as they are
 *   pool             [pool_cap], a ring of free block ids: state[1] of them from entry state[0] on; blocks that return are written behind
 *                    them (never more than pool_cap in all)
 *   state            [6], of which the first two are read (outside [0, pool_cap): an empty pool)
 *   lengths_out      [n_seqs] n + c, or n where refused
 *   state_out        [6] the pool's first entry and count behind the call, rows, blocks taken, blocks returned, requests refused
 *   row_offsets      [n_seqs + 1] first row of each request
 *   token_seq_ids, token_positions, token_adapter_ids [row_cap], slot_mapping int64 [row_cap]: request, position, adapter and cache slot of each
 *                    row; rows behind the last one get -1, 0, -1 and -1, which the projection and the reader pass over.
 *                    A pool or table entry outside [0, n_slots / block_size) gives slot -1.
 * lengths_out and state_out may not be lengths and state (ALORA_EINVAL): a call may be repeated with the same inputs and gives the same
 * results.  A loop exchanges them from step to step.
 */
int alora_step_rows(const int32_t *lengths, const int32_t *change, const int32_t *kept_blocks, const int32_t *seq_adapters, int32_t *block_tables,
                    int32_t *pool, const int32_t *state, int32_t *lengths_out, int32_t *state_out, int32_t *row_offsets, int32_t *token_seq_ids,
                    int32_t *token_positions, int32_t *token_adapter_ids, int64_t *slot_mapping, const alora_step_dims *dims, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* ALORA_STEPS_H */
