/*
 * alora_heads.h -- what stands between the projection and the reader of the cache: the norm of every query and
 * key head with the rotary embedding in the same pass, its backward pass, and the cosines and sines it turns by
 * (C ABI of libalora_qkv.so, gfx950).
 *
 * The projection (alora_qkv.h) can turn heads in its store, in halves, over whole heads.  Layers whose query and
 * key heads are normalised first, whose heads are turned in part, or whose pairs are neighbours, project without
 * tables and call alora_qk_norm_rope behind it.
 *
 * Conventions are those of alora_qkv.h: data pointers are DEVICE pointers of buffers that the caller owns,
 * 16-byte aligned unless said otherwise; nothing is allocated, nothing is kept between calls; work is enqueued on
 * `hip_stream` and the call returns; on ALORA_EINVAL, ALORA_ESHAPE and ALORA_EWORKSPACE nothing has been enqueued.
 */
#ifndef ALORA_HEADS_H
#define ALORA_HEADS_H

#include <stddef.h>
#include <stdint.h>
#include "alora_qkv.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Shapes of a call.  Strides are in elements between rows (a row's heads lie behind each other), at least the
 * row's width and a multiple of 16 bytes; views of a fused q | k | v buffer have the buffer's.
 * Limits (ALORA_ESHAPE): head_dim a multiple of 8 (bf16) or 4 (fp32), at most 256; rotary_dim a multiple of 4, at most
 * head_dim; n_tokens * (n_q_heads + 2 * n_kv_heads) <= 2^31 - 1.
 */
typedef struct alora_heads_dims {
    int32_t dtype;            /* ALORA_F32 or ALORA_BF16: of rows, caches and norm weights                   */
    int32_t n_tokens;         /* rows; 0 is a successful no-op                                               */
    int32_t n_q_heads, n_kv_heads, head_dim;
    int32_t rotary_dim;       /* features at the front of each head that are turned; 0 = none                */
    int32_t interleaved;      /* 0: feature i turns with i + rotary_dim / 2;  1: 2i turns with 2i + 1         */
    int32_t norm;             /* 1: heads are normalised first                                               */
    int32_t rope_positions;   /* rows of the tables (>= 1 where rotary_dim > 0)                              */
    float eps;                /* added to the mean square                                                    */
    int64_t n_slots;          /* rows of k_cache and v_cache                                                 */
    int64_t q_stride, q_out_stride;   /* backward: of q, and of q's outputs' gradient                        */
    int64_t k_stride, k_out_stride;   /* k_out: the cache; backward: of k's outputs' gradient                */
    int64_t v_stride, v_out_stride;
    int64_t dq_stride, dk_stride;     /* backward: of the gradients; 0 = q_stride, k_stride                   */
} alora_heads_dims;

/*
 * For every row t, and every query head and key head x of it:
 *     y = x * w / sqrt(mean(x^2) + eps)                    (norm; w = wq or wk, one weight per feature)
 *     out[i] = y[i] c - y[j] s,  out[j] = y[j] c + y[i] s  for the pair (i, j) with c, s = cos, sin[positions[t], pair]
 * and the features from rotary_dim on are y's.  Sums and products are fp32, the result is rounded once.
 * Query heads go from q to q_out.  Key heads go from row t of k to row slot_mapping[t] of k_cache, or, where k is NULL,
 * from that row of k_cache to itself: the projection has stored them there.  Where v is given, its rows are copied to
 * v_cache.  Where slot_mapping[t] is -1 (a padding row), or outside [0, n_slots), keys and values are left alone;
 * the row's query heads are written.
 *   q, q_out       [n_tokens, n_q_heads * head_dim]; q_out may be q
 *   k, v           [n_tokens, n_kv_heads * head_dim] or NULL
 *   k_cache        [n_slots, n_kv_heads * head_dim];  v_cache the same, NULL where v is
 *   wq, wk         [head_dim], NULL exactly where norm is 0
 *   cos, sin       fp32 [rope_positions, rotary_dim / 2], NULL exactly where rotary_dim is 0
 *   positions      [n_tokens] int32; outside [0, rope_positions) the nearest row of the tables is used;
 *                  NULL where rotary_dim is 0
 *   slot_mapping   [n_tokens] int64, the non-negative ones pairwise distinct
 * Buffers other than q and q_out do not overlap.
 */
int alora_qk_norm_rope(const void *q, void *q_out, const void *k, void *k_cache, const void *v, void *v_cache,
                       const void *wq, const void *wk, const float *cos, const float *sin, const int32_t *positions,
                       const int64_t *slot_mapping, const alora_heads_dims *dims, void *hip_stream);

/*
 * Gradients.  With g = the outputs' gradient turned back, r = 1 / sqrt(mean(x^2) + eps), u = g * w:
 *     dx = r u - x r^3 mean(u x)          (norm 0: dx = g)
 *     dw = sum over rows and heads of g x r
 *   q, k             what the forward call read;  dq_out, dk_out: gradients of its outputs, row t at row t
 *   dq, dk           written; dq may be dq_out where strides are equal, dk likewise
 *   dwq, dwk         fp32 [head_dim], written; NULL exactly where norm is 0
 *   workspace        16-byte aligned, alora_qk_norm_rope_workspace_bytes() (0 where norm is 0: then it may be NULL);
 *                    contents on entry irrelevant; calls that share it must be stream-ordered
 * n_tokens = 0 writes dwq and dwk (zeros).  The sums' order is fixed by the sizes: equal calls give equal bits.
 * slot fields and v strides of dims are not looked at.
 */
int alora_qk_norm_rope_workspace_bytes(const alora_heads_dims *dims, size_t *out_bytes);
int alora_qk_norm_rope_backward(const void *q, const void *dq_out, void *dq, const void *k, const void *dk_out, void *dk,
                                const void *wq, const void *wk, float *dwq, float *dwk, const float *cos, const float *sin,
                                const int32_t *positions, const alora_heads_dims *dims, void *workspace,
                                size_t workspace_bytes, void *hip_stream);

/* Slow, synchronous check of a forward call's index data: positions in [0, rope_positions) where heads are turned, slots -1 or in
 * [0, n_slots) and distinct.  ALORA_OK, ALORA_EDATA or an argument error. */
int alora_qk_norm_rope_validate(const int32_t *positions, const int64_t *slot_mapping, const alora_heads_dims *dims);

/* How angles are scaled for contexts longer than the model was trained on. */
#define ALORA_ROPE_PLAIN 0     /* theta_i = base^(-2i / rotary_dim)                                          */
#define ALORA_ROPE_LINEAR 1    /* theta_i / factor: positions pressed together                               */
#define ALORA_ROPE_BY_PARTS 2  /* pairs that turn at least `high` times in `original` positions keep theta_i, those that
                                  turn at most `low` times get theta_i / factor, between them the two are mixed:
                                  with g = clamp((original theta_i / 2 pi - low) / (high - low), 0, 1),
                                  theta_i (g + (1 - g) / factor)                                              */
typedef struct alora_rope_spec {
    int32_t rotary_dim;       /* even, 2 .. 512                                                              */
    int32_t scaling;
    double base;              /* > 0                                                                         */
    double factor;            /* > 0; not looked at by ALORA_ROPE_PLAIN                                      */
    double original, low, high;   /* ALORA_ROPE_BY_PARTS: original > 0, low < high                           */
    double magnitude;         /* multiplies cosines and sines; 1 = none                                      */
} alora_rope_spec;

/*
 * cos[p - first, i] = magnitude cos(p theta_i), sin likewise, for p = first .. first + rows - 1 and every pair i.
 * Angles are held in 64 bits: far positions are as exact as near ones.  A result is off by half a unit in its last place, and by what the angle
 * loses in 64 bits, at most magnitude * position * t * 2^-49: t = 1 where base and factor are at least 1, else
 * max(1, theta) (1 + max(0, -log2 base) / 4) with theta the largest angle of a position; by parts 1 + high / (high - low) times that.  (A position's
 * angle is off by up to 10 half units of itself, a power of two another 2 for every bit of its exponent; every step of the kernel's products
 * adds 4, and there are at most as many as positions.)  0 <= first, first + rows <= 2^24 (ALORA_ESHAPE).  cos, sin: fp32
 * [rows, rotary_dim / 2], 16-byte aligned; with magnitude 1 they are tables for alora_cache_move_rows too, with rotary_dim = head_dim for
 * alora_extras.rope_cos and rope_sin.
 */
int alora_rope_tables(float *cos, float *sin, int64_t first, int64_t rows, const alora_rope_spec *spec, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* ALORA_HEADS_H */
