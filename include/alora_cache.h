/*
 * alora_cache.h -- moving what the paged K/V cache holds: whole blocks (a fork's partial block, a pool made dense,
 * blocks cleared) and single token rows whose positions change, over all layers in one call (C ABI of
 * libalora_qkv.so, gfx950).  alora_planner_fork, _compact and _drop (alora_planner.h) say what to move.
 *
 * Conventions are those of alora_qkv.h.  Caches are dense, [n_slots, n_kv_heads * head_dim] each, slot s being
 * offset s % block_size of block s / block_size, 16-byte aligned.
 */
#ifndef ALORA_CACHE_H
#define ALORA_CACHE_H

#include <stddef.h>
#include <stdint.h>
#include "alora_qkv.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Limits (ALORA_ESHAPE): head_dim a multiple of 8 (bf16) or 4 (fp32), at most 256; n_slots % block_size == 0;
 * n_slots / block_size <= 2^31 - 1; n_layers <= 4096. */
typedef struct alora_cache_dims {
    int32_t dtype;
    int32_t n_layers;               /* 0 is a successful no-op                                               */
    int32_t n_kv_heads, head_dim, block_size;
    int64_t n_slots;
    void *const *k_caches;          /* (host) n_layers device pointers, read during the call only            */
    void *const *v_caches;
} alora_cache_dims;

/*
 * Block src[i] is copied to block dst[i], in the K and V cache of every layer; src[i] = -1 clears block dst[i] to zeros.
 *   src, dst   (host) [n], read during the call only (also where it is captured into a graph: a replay makes the
 *              same copies).  ALORA_EDATA, nothing enqueued: an index outside the pool, a destination
 *              named twice, or a block that is both source and destination (the copies run side by side).
 * n = 0 is a successful no-op.
 */
int alora_cache_copy_blocks(const int32_t *src, const int32_t *dst, int32_t n, const alora_cache_dims *dims, void *hip_stream);

/*
 * Row src[i] of every layer's caches goes to row dst[i]; the key is turned by shift[i] positions on the way:
 *     K[dst[i]] = R(shift[i]) K[src[i]],  V[dst[i]] = V[src[i]]
 * R as in alora_qk_norm_rope, with cos, sin at |shift[i]| and the sine's sign that of the shift.  A key that was stored
 * for position p then stands for p + shift[i], whatever base and scaling the tables have, as long as p and the
 * shift count positions of the same tables.  The tables' magnitude has to be 1 (cached keys hold it already).
 * Limit (ALORA_ESHAPE): n_rows * n_kv_heads <= 2^25.
 * fp32 products, one rounding; keys of rows with shift 0 are copied bit for bit.
 *   src, dst        [n_rows] int64; a row outside [0, n_slots) on either side is left alone
 *   shift           [n_rows] int32, NULL: rows are only copied (then cos and sin are NULL and rotary_dim is 0);
 *                   |shift| beyond the tables uses their last row
 *   cos, sin        fp32 [rope_positions, rotary_dim / 2]
 *   rotary_dim      a multiple of 4, at most head_dim
 * No dst may be another row's src or dst (rows move side by side); dst[i] == src[i] turns a key where it lies.
 */
int alora_cache_move_rows(const int64_t *src, const int64_t *dst, const int32_t *shift, int32_t n_rows, const float *cos,
                          const float *sin, int32_t rope_positions, int32_t rotary_dim, int32_t interleaved,
                          const alora_cache_dims *dims, void *hip_stream);

/* Slow, synchronous check of a move: indexes in range, no dst another row's src or dst, shifts within the tables.
 * ALORA_OK, ALORA_EDATA or an argument error. */
int alora_cache_move_rows_validate(const int64_t *src, const int64_t *dst, const int32_t *shift, int32_t n_rows,
                                   int32_t rope_positions, const alora_cache_dims *dims);

#ifdef __cplusplus
}
#endif
#endif /* ALORA_CACHE_H */
