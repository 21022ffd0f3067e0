/*
 * moe_latent.h -- C ABI of attention with keys and values from one shared latent vector a token: filling the cache, and
 * attending over it, for single tokens, for prompts, and for batches whose sequences share a prefix.
 *
 * Every token leaves one row in the cache: a latent vector c and a part p that carries the position.  Head h's key is
 * (w_k[h] c, p) and its value w_v[h] c, so a cache of any number of heads has the bytes of one.  With a query q = (n, r):
 *     z_j = softmax_scale * (n . w_k c_j + r . p_j),   o = w_v sum_j softmax(z)_j c_j = sum_j softmax(z)_j (w_v c_j)
 * which can be computed two ways:
 *   absorbed: a = w_k^T n once for a query, z_j = softmax_scale * (a . c_j + r . p_j), u = sum_j softmax(z)_j c_j, o = w_v u: all heads
 *     read the same rows, 2 * (2 * latent_dim + rope_dim) operations per head and pair of tokens; for few new tokens.
 *   expanded: keys and values of every head made once for all new tokens, 2 * (nope_dim + rope_dim + v_dim) operations per pair; for
 *     prompts.
 *
 * Conventions: as in moe_kv8.h: status codes, caller-owned device memory and streams, calls enqueue, allocate nothing, keep
 * nothing and never wait (they can be captured); numbers per sequence are read on the device when the kernels run and brought
 * into the bounds the host gives; every tensor on one device, which need not be the current one; workspaces may be used again
 * by the next call on the same stream (not by two graphs that may run at once); a launch has less than 2^32 threads, a call that asks for
 * more is MOE_ERR_SHAPE.  The error text of a failed call is moe_latent_last_error() on the same thread.
 */
#ifndef KLOTSKI_MOE_LATENT_H
#define KLOTSKI_MOE_LATENT_H

#include "moe_kv8.h"
#include "moe_rope.h"

#ifdef __cplusplus
extern "C" {
#endif

/* The cache of one layer: device memory, owned by the caller.  What lies in slots a sequence does not hold is never used,
 * whatever it is. */
typedef struct {
    int32_t n_seq;      /* 1..65536 */
    int32_t latent_dim; /* 128, 256 or 512 */
    int32_t rope_dim;   /* 32 or 64 */
    int32_t max_len;    /* slots of a sequence, 1..2^20 */
    int32_t prefix_len; /* rows of `prefix` that every sequence sees before its own, 0..2^20 */
    int32_t reserved;   /* 0 */
    void* rows;         /* bf16 [n_seq, max_len, latent_dim + rope_dim], 16-byte aligned: c, then p */
    const void* prefix; /* bf16 [prefix_len, latent_dim + rope_dim], 16-byte aligned; null without prefix.  It is read once for the
                           rows of all sequences.  (It is filled as the cache of a batch of one sequence.) */
} moe_latent_cache;

/* The heads of the layer: device memory, bf16, 16-byte aligned. */
typedef struct {
    int32_t n_heads;  /* 1..256 */
    int32_t nope_dim; /* elements of a query that meet the latent's key: 32, 64 or 128 */
    int32_t v_dim;    /* 32, 64 or 128 */
    int32_t reserved; /* 0 */
    const void* w_k;  /* element (head, i, j) at head * w_k_head + i * latent_dim + j, [n_heads, nope_dim, latent_dim]; finite */
    const void* w_v;  /* the same with w_v_head, [n_heads, v_dim, latent_dim]; the two may be parts of one matrix */
    int64_t w_k_head, w_v_head; /* strides, multiples of 8; 0: heads one behind the other */
} moe_latent_heads;

/*
 * moe_latent_append -- writes the rows of the new tokens of `step` (moe_kv8.h; the layers of a model share it): of every
 * row x = (c, p), c * norm / sqrt(mean(c^2) + eps) (c itself if `norm` is null) and p turned by the token's position (p itself if `rope`
 * is null).  Positions count from step->next_position, null: from cache->prefix_len + cached.
 *   x: bf16, element (row, i) at row * x_row_stride + i, 16-byte aligned, the stride a multiple of 8.
 *   norm: bf16 [latent_dim], 16-byte aligned.   rope: first + rot_dim at most rope_dim.
 * Sums and products in 32 bits, rounded once.  Tokens that would take a slot from max_len on do not exist.
 */
moe_status moe_latent_append(void* stream, const moe_latent_cache* cache, const moe_kv8_step* step, const void* x,
                             int64_t x_row_stride, const void* norm, float eps, const moe_rope_config* rope);

/* How moe_latent_attend computes: MOE_LATENT_AUTO takes the form that should be the faster one by the step's bounds, and the other one where
 * that would have too many workgroups. */
typedef enum { MOE_LATENT_AUTO = 0, MOE_LATENT_ABSORBED = 1, MOE_LATENT_EXPANDED = 2 } moe_latent_form;

/*
 * moe_latent_attend -- attention of the new tokens, after moe_latent_append of the same step: token i of sequence s sees
 * the whole prefix and slots 0 .. cached[s] + i of its own.
 *   q: bf16, element (row, head, i) at row * q_row_stride + head * q_head_stride + i: nope_dim elements, then rope_dim that have been
 *     turned already (moe_rope_rotate with first = nope_dim); out: likewise, v_dim elements.  16-byte aligned, strides multiples of 8;
 *     no two (row, head) of out share an element, and q and out share none.
 *   softmax_scale: 0 stands for 1 / sqrt(nope_dim + rope_dim).
 * Rows of no sequence are left as they were.  Scores, the softmax's statistics and sums are kept in 32 bits.  Rounded on
 * the way: in the absorbed form the softmax weights to bf16, a and u to two bf16 (16 bits together; latents below 2^-80 have fewer); in the
 * expanded one the softmax weights, keys, values and the queries' nope_dim elements to fp16 times a power of two, finite ones to finite
 * ones.  The keys, and the values, of 64 slots of a sequence share that power for a head, a query's elements do, and a row's weights:
 * each is off by 2^-11 of itself, or by 2^-19 of the largest of them where that is more.  A latent that is not finite reaches the rows that
 * see it, all their elements, and no others.
 * The result of a sequence does not depend on what the others hold; how its sums are split follows from the numbers in the structs and
 * its own length.
 * workspace: moe_latent_attend_workspace_bytes() of device memory, 256-byte aligned; it depends on sizes and bounds only.
 */
moe_status moe_latent_attend_workspace_bytes(const moe_latent_cache* cache, const moe_kv8_step* step, const moe_latent_heads* heads,
                                             int32_t form, int64_t* bytes_out);
moe_status moe_latent_attend(void* stream, const moe_latent_cache* cache, const moe_kv8_step* step, const moe_latent_heads* heads,
                             const void* q, int64_t q_row_stride, int64_t q_head_stride, float softmax_scale, int32_t form, void* out,
                             int64_t out_row_stride, int64_t out_head_stride, void* workspace, int64_t workspace_bytes);

/* Error text of the last failed call on the calling thread. */
const char* moe_latent_last_error(void);

#ifdef __cplusplus
}
#endif
#endif /* KLOTSKI_MOE_LATENT_H */
